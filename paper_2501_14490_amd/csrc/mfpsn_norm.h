// Internal interface of the layer-norm kernels (mfpsn_norm.hip) for the C-ABI
// layer.  Not installed; not part of the ABI.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace mfpsn {

// x[M][C][S], normalised over C at every (m, s)
struct NormArgs {
    int64_t M;
    int32_t C, S;
    float eps;
    const void* x;
    const void* gy;      // backward only
    const float* gamma;  // nullable: 1
    const float* beta;   // nullable: 0 (forward only)
    float* mean;         // [M][S]; written by the forward where not NULL, read by the backward
    float* rstd;         // [M][S]; likewise
    void* out;           // y, or grad_x
    float* part;         // backward: [blocks][2][C] partial sums of grad_gamma, grad_beta
    float* grad_gamma;   // nullable
    float* grad_beta;    // nullable
};

// Upper bound of the backward's blocks, and so of its partial rows: the
// partial sums of 2 C floats a block stay below 1/8 of the bytes that the
// block's share of x and grad_y has (see norm_blocks), and 1024 blocks of 4
// waves are 4 waves for each SIMD.
constexpr int kNormMaxBlocks = 1024;

// Blocks of the backward for M rows of C channels and S columns (host; the
// workspace is sized by it)
inline int norm_blocks(int64_t M, int64_t C, int64_t S)
{
    (void)C;
    const int64_t work = (M * S + 15) / 16;  // 16 columns for a block at least
    return (int)(work < 1 ? 1 : (work < kNormMaxBlocks ? work : kNormMaxBlocks));
}

hipError_t launch_norm_forward(const NormArgs& a, int dtype, hipStream_t stream);
hipError_t launch_norm_backward(const NormArgs& a, int dtype, hipStream_t stream);

}  // namespace mfpsn
