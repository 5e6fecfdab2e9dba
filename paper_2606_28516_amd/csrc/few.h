// The whole layer for a few tokens (few.hip): internal declarations.
#pragma once

#include "kernels.h"

namespace clearmoe {

// Tokens of one workgroup: the columns of a 16 x 16 MFMA.  More tokens run as
// several groups, each reading the weights again.
constexpr int kFewGroup = 16;

struct FewArgs {
    const void *x, *W1, *US, *Vt, *P, *Q, *Wg;
    const float *b1, *b2, *bg;
    void* y;
    int32_t* idx;             // routing [T, k]: written by the first kernel, or given (routed)
    float* gate;
    float* part;              // [S][T][r + k q] partial sums of t and the u_j over hidden slices
    int T, D, H, E, k, r, q;
    int adaptive, renorm, routed;
    double tau;
};

// Hidden slices (the first kernel's workgroups per token group) and the bytes
// of the partial sums.
int few_slices(int H);
size_t few_part_bytes(int64_t T, int H, int r, int k, int q);
// Two kernels; whole: the rows of every matrix are whole, aligned 16-byte pieces.
hipError_t launch_few_hidden(int dtype, bool whole, const FewArgs& a, hipStream_t st);
hipError_t launch_few_out(int dtype, bool whole, const FewArgs& a, hipStream_t st);

}  // namespace clearmoe
