// Products of grouped rows: what their kernels are given (expert.hip), for the calls made of them.
#pragma once
#include "groups.h"
#include "products.h"

// out_q = scale * M x_q per row q of a group, M the group's matrix in the server, or its transpose; zero for rows of no group
struct ExpertArgs {
    RowGroups g;
    const void *x; int64_t x_stride; int32_t x_type; Quotient x_shared;       // row q is row q / x_shared of x; order == NULL there: place p
    const float *w; int64_t L, each;                                         // matrix e's rows are the L numbers from w + (e * each + r) * L on
    int32_t K, N, turned;                                                    // turned: M is the transpose: the sum goes over the K rows
    float scale;
    void *out; int64_t out_stride; int32_t out_type, by_place;               // by_place: the row at place p goes to row p of out
    int32_t precise;                                                         // products of numbers of 32 bits
};
int dpaps_expert_product(dpaps_ps *ps, const ExpertArgs &a, hipStream_t st);

// out_e[i][j] = sum over group e's rows of left[i] right[j]
struct OuterArgs {
    RowGroups g;
    const void *left; int64_t left_stride; int32_t left_type, left_by_place; Quotient left_shared;
    const void *right; int64_t right_stride; int32_t right_type; Quotient right_shared;
    int32_t rows, cols;
    void *out; int32_t out_type;
};
int dpaps_outer_sums(dpaps_ps *ps, const OuterArgs &a, hipStream_t st);

// out_p = M x_p + sum_r low[place of p][r] B_e[r], with a matrix M for all rows (or its transpose), low: fp32, of rows of a group, scaled already
struct AdapterArgs {
    RowGroups g;
    const void *x; int64_t x_stride; int32_t x_type;
    const float *w; int64_t L;
    int32_t K, N, turned;
    const float *low; int64_t low_stride; int32_t rank;
    const float *b;                                                          // group e's rank rows from b + e * rank * L on
    void *out; int64_t out_stride; int32_t out_type;
};
