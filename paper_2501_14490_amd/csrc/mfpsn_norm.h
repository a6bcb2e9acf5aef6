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

// Blocks of the backward for M rows of C channels and S columns (host; the
// workspace has 2 C floats for each): one for 4 rows (S = 1) or a tile of 64
// columns, up to 4 waves for each SIMD, 8 for few channels, whose tiles are
// short of loads in flight and whose partial sums are small.
constexpr int kNormMaxBlocks = 2048;
inline int norm_blocks(int64_t M, int64_t C, int64_t S)
{
    const int64_t work = S == 1 ? (M + 3) / 4 : (M * S + 63) / 64, most = C <= 256 ? kNormMaxBlocks : kNormMaxBlocks / 2;
    return (int)(work < 1 ? 1 : (work < most ? work : most));
}

hipError_t launch_norm_forward(const NormArgs& a, int dtype, hipStream_t stream);
hipError_t launch_norm_backward(const NormArgs& a, int dtype, hipStream_t stream);

}  // namespace mfpsn
