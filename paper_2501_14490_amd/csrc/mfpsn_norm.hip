// gfx950 kernels of the layer norm over the channels of x[M][C][S] (time-first
// tensors [T][N][C][S] have M = T N; time-last ones [N][C][S][T] have M = N
// and the time inside S).
//
//   forward   mu = mean_c x, var = mean_c (x - mu)^2, r = 1/sqrt(var + eps),
//             y = gamma (x - mu) r + beta
//   backward  xh = (x - mu) r, a = gamma gy,
//             gx = r (a - mean_c a - xh mean_c(a xh)),
//             ggamma = sum_{m,s} gy xh, gbeta = sum_{m,s} gy
//
// Both passes are HBM-bound (one read of each input, one write of each output;
// about 10 flops an element).  A row's values are loaded once and stay in
// registers between its statistics and its outputs, so the variance can be
// the mean of the squared deviations (two passes over registers) instead of a
// difference of two large sums.  All sums are float; ggamma and gbeta are
// summed by each thread over the columns of its block, then over a block's
// threads, then over the blocks by a second kernel in double, each in a fixed
// order, so repeated calls give the same bits.
//
// S = 1: the channels are contiguous; a wave (or the block's four waves, for
// long rows) takes a row, 16 bytes a lane and load where rows are aligned.
// S > 1: a block takes a tile of neighbouring columns (m, s) and all channels;
// lanes run over the columns, and the channels are spread over the lanes'
// rows and the waves.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mfpsn_internal.h"
#include "mfpsn_norm.h"

namespace mfpsn {
namespace {

constexpr int kT = 256;  // threads of a block

struct F32 {
    using T = float;
    __device__ static float get(T v) { return v; }
    __device__ static T put(float v) { return v; }
};
struct BF16 {
    using T = uint16_t;
    __device__ static float get(T v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
    // round to nearest even (the stored result's one rounding to 16 bits)
    __device__ static T put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};

template <typename T, int N> struct alignas(sizeof(T) * N) Vec {
    T v[N];
};

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o);
    return v;
}

// Sum over the WPR waves that share a row; `at` alternates between calls so
// that one barrier a call is enough
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float (*lds)[4], int& at)
{
    v = wave_sum(v);
    if constexpr (WPR > 1) {
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
            lds[at][w] = v;
        __syncthreads();
        v = lds[at][0];
#pragma unroll
        for (int i = 1; i < WPR; ++i)
            v += lds[at][i];
        at ^= 1;
    }
    return v;
}

// ---------------------------------------------------------------------------
// S = 1
// ---------------------------------------------------------------------------

// A lane's elements of a row: NV loads of VE neighbours, LANES lanes a row
template <typename D, int VE, int NV, int WPR>
__global__ __launch_bounds__(kT) void norm_fwd_rows(NormArgs a)
{
    using T = typename D::T;
    using V = Vec<T, VE>;
    constexpr int LANES = 64 * WPR, ROWS = 4 / WPR;
    __shared__ float lds[2][4];
    int at = 0;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    const int C = a.C;
    const float inv = 1.0f / (float)C;
    for (int64_t m = (int64_t)blockIdx.x * ROWS + sub; m < a.M; m += (int64_t)gridDim.x * ROWS) {
        const T* __restrict__ x = (const T*)a.x + m * C;
        T* __restrict__ y = (T*)a.out + m * C;
        float f[NV][VE];
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * LANES + lane) * VE;
            V v = {};
            if (e < C)
                v = *(const V*)(x + e);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                f[i][j] = D::get(v.v[j]);
                s += f[i][j];
            }
        }
        const float mean = row_sum<WPR>(s, lds, at) * inv;
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * LANES + lane) * VE;
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                f[i][j] -= mean;
                q += e < C ? f[i][j] * f[i][j] : 0.0f;
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<WPR>(q, lds, at) * inv + a.eps);
        if (lane == 0 && a.mean) {
            a.mean[m] = mean;
            a.rstd[m] = rstd;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * LANES + lane) * VE;
            if (e < C) {
                V v;
#pragma unroll
                for (int j = 0; j < VE; ++j)
                    v.v[j] = D::put(f[i][j] * rstd * (a.gamma ? a.gamma[e + j] : 1.0f) + (a.beta ? a.beta[e + j] : 0.0f));
                *(V*)(y + e) = v;
            }
        }
    }
}

// rows longer than the registers of a block hold: read three times
template <typename D>
__global__ __launch_bounds__(kT) void norm_fwd_long(NormArgs a)
{
    using T = typename D::T;
    __shared__ float lds[2][4];
    int at = 0;
    const int C = a.C;
    const float inv = 1.0f / (float)C;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* __restrict__ x = (const T*)a.x + m * C;
        T* __restrict__ y = (T*)a.out + m * C;
        float s = 0.0f, q = 0.0f;
        for (int e = threadIdx.x; e < C; e += kT)
            s += D::get(x[e]);
        const float mean = row_sum<4>(s, lds, at) * inv;
        for (int e = threadIdx.x; e < C; e += kT) {
            const float d = D::get(x[e]) - mean;
            q += d * d;
        }
        const float rstd = 1.0f / sqrtf(row_sum<4>(q, lds, at) * inv + a.eps);
        if (threadIdx.x == 0 && a.mean) {
            a.mean[m] = mean;
            a.rstd[m] = rstd;
        }
        for (int e = threadIdx.x; e < C; e += kT)
            y[e] = D::put((D::get(x[e]) - mean) * rstd * (a.gamma ? a.gamma[e] : 1.0f) + (a.beta ? a.beta[e] : 0.0f));
    }
}

template <typename D, int VE, int NV, int WPR>
__global__ __launch_bounds__(kT) void norm_bwd_rows(NormArgs a)
{
    using T = typename D::T;
    using V = Vec<T, VE>;
    constexpr int LANES = 64 * WPR, ROWS = 4 / WPR;
    __shared__ float lds[2][4];
    __shared__ float sums[ROWS > 1 ? (ROWS - 1) * LANES : 1];
    int at = 0;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    const int C = a.C;
    const float inv = 1.0f / (float)C;
    float gg[NV][VE] = {}, gb[NV][VE] = {}, gam[NV][VE];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const int e = (i * LANES + lane) * VE + j;
            gam[i][j] = e < C ? (a.gamma ? a.gamma[e] : 1.0f) : 0.0f;
        }
    for (int64_t m = (int64_t)blockIdx.x * ROWS + sub; m < a.M; m += (int64_t)gridDim.x * ROWS) {
        const T* __restrict__ x = (const T*)a.x + m * C;
        const T* __restrict__ gy = (const T*)a.gy + m * C;
        T* __restrict__ gx = (T*)a.out + m * C;
        const float mean = a.mean[m], rstd = a.rstd[m];
        V vx[NV] = {}, vg[NV] = {};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * LANES + lane) * VE;
            if (e < C) {
                vx[i] = *(const V*)(x + e);
                vg[i] = *(const V*)(gy + e);
            }
        }
        float sa = 0.0f, sh = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float g = D::get(vg[i].v[j]), xh = (D::get(vx[i].v[j]) - mean) * rstd;
                gg[i][j] += g * xh;  // (lanes behind the row: g = 0)
                gb[i][j] += g;
                const float al = g * gam[i][j];
                sa += al;
                sh += al * xh;
            }
        }
        const float ma = row_sum<WPR>(sa, lds, at) * inv;
        const float mh = row_sum<WPR>(sh, lds, at) * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * LANES + lane) * VE;
            if (e < C) {
                V v;
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float g = D::get(vg[i].v[j]), xh = (D::get(vx[i].v[j]) - mean) * rstd;
                    v.v[j] = D::put(rstd * (g * gam[i][j] - ma - xh * mh));
                }
                *(V*)(gx + e) = v;
            }
        }
    }
    if (!a.part)
        return;
    float* __restrict__ part = a.part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j)
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float v = which ? gb[i][j] : gg[i][j];
                if constexpr (ROWS > 1) {
                    __syncthreads();
                    if (sub > 0)
                        sums[(sub - 1) * LANES + lane] = v;
                    __syncthreads();
                    if (sub == 0)
#pragma unroll
                        for (int r = 0; r < ROWS - 1; ++r)
                            v += sums[r * LANES + lane];
                }
                const int e = (i * LANES + lane) * VE + j;
                if (sub == 0 && e < C)
                    part[which * C + e] = v;
            }
}

// rows longer than the registers of a block hold: grad_x here (each input read
// twice), the weights' sums in norm_bwd_long_weights
template <typename D>
__global__ __launch_bounds__(kT) void norm_bwd_long(NormArgs a)
{
    using T = typename D::T;
    __shared__ float lds[2][4];
    int at = 0;
    const int C = a.C;
    const float inv = 1.0f / (float)C;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T* __restrict__ x = (const T*)a.x + m * C;
        const T* __restrict__ gy = (const T*)a.gy + m * C;
        T* __restrict__ gx = (T*)a.out + m * C;
        const float mean = a.mean[m], rstd = a.rstd[m];
        float sa = 0.0f, sh = 0.0f;
        for (int e = threadIdx.x; e < C; e += kT) {
            const float al = D::get(gy[e]) * (a.gamma ? a.gamma[e] : 1.0f);
            sa += al;
            sh += al * (D::get(x[e]) - mean) * rstd;
        }
        const float ma = row_sum<4>(sa, lds, at) * inv;
        const float mh = row_sum<4>(sh, lds, at) * inv;
        for (int e = threadIdx.x; e < C; e += kT) {
            const float al = D::get(gy[e]) * (a.gamma ? a.gamma[e] : 1.0f);
            gx[e] = D::put(rstd * (al - ma - (D::get(x[e]) - mean) * rstd * mh));
        }
    }
}

template <typename D>
__global__ __launch_bounds__(kT) void norm_bwd_long_weights(NormArgs a)
{
    using T = typename D::T;
    const int C = a.C;
    float* __restrict__ part = a.part + (int64_t)blockIdx.y * 2 * C;
    const int64_t e = (int64_t)blockIdx.x * kT + threadIdx.x;
    if (e >= C)
        return;
    float gg = 0.0f, gb = 0.0f;
    for (int64_t m = blockIdx.y; m < a.M; m += gridDim.y) {
        const float g = D::get(((const T*)a.gy)[m * C + e]);
        gg += g * ((D::get(((const T*)a.x)[m * C + e]) - a.mean[m]) * a.rstd[m]);
        gb += g;
    }
    part[e] = gg;
    part[C + e] = gb;
}

// ---------------------------------------------------------------------------
// S > 1
// ---------------------------------------------------------------------------

// A tile: W = LX * VE neighbouring columns j = m S + s, all C channels.  Lane
// (lx, ly) of wave w has columns lx VE .. + VE and channels (p NW + w) LY + ly,
// p = 0, 1, ...; the first NP of them stay in registers (CACHED: all of them).
template <int VE, int LX, int NW> struct Plane {
    static constexpr int LY = 64 / LX, W = LX * VE, STEP = NW * LY, THREADS = NW * 64;
};

// Sums over the channels of VE columns: over the lanes' rows, then the waves
template <int VE, int LX, int NW>
__device__ __forceinline__ void column_sum(float (&v)[VE], float (*lds)[NW][LX * VE])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, lx = lane % LX;
#pragma unroll
    for (int o = LX; o < 64; o <<= 1)
#pragma unroll
        for (int j = 0; j < VE; ++j)
            v[j] += __shfl_xor(v[j], o);
    __syncthreads();
    if (lane < LX)
#pragma unroll
        for (int j = 0; j < VE; ++j)
            (*lds)[w][lx * VE + j] = v[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < VE; ++j) {
        float s = (*lds)[0][lx * VE + j];
        for (int i = 1; i < NW; ++i)
            s += (*lds)[i][lx * VE + j];
        v[j] = s;
    }
}

template <typename D, int VE, int LX, int NW, int NP, bool CACHED>
__global__ __launch_bounds__(NW * 64) void norm_fwd_planes(NormArgs a)
{
    using T = typename D::T;
    using V = Vec<T, VE>;
    using P = Plane<VE, LX, NW>;
    __shared__ float lds[1][NW][P::W];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, lx = lane % LX, ly = lane / LX;
    const int C = a.C, S = a.S, c0 = w * P::LY + ly;
    const float inv = 1.0f / (float)C;
    const int64_t cols = a.M * S, tiles = (cols + P::W - 1) / P::W;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t j = t * P::W + lx * VE;
        const bool live = j < cols;  // (VE divides S: a vector's columns are all live, in one m)
        const int64_t m = live ? j / S : 0;
        const int64_t base = live ? m * C * S + (j - m * S) : 0;
        const T* __restrict__ x = (const T*)a.x + base;
        T* __restrict__ y = (T*)a.out + base;
        V keep[NP];
        float s[VE] = {}, q[VE] = {};
        if constexpr (CACHED) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int c = c0 + p * P::STEP;
                keep[p] = V{};
                if (live && c < C)
                    keep[p] = *(const V*)(x + (int64_t)c * S);
            }
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    s[i] += D::get(keep[p].v[i]);
        } else if (live) {
            for (int c = c0; c < C; c += P::STEP) {
                const V v = *(const V*)(x + (int64_t)c * S);
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    s[i] += D::get(v.v[i]);
            }
        }
        column_sum<VE, LX, NW>(s, lds);
        float mean[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i)
            mean[i] = s[i] * inv;
        if constexpr (CACHED) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (c0 + p * P::STEP < C)
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        const float d = D::get(keep[p].v[i]) - mean[i];
                        q[i] += d * d;
                    }
        } else if (live) {
            for (int c = c0; c < C; c += P::STEP) {
                const V v = *(const V*)(x + (int64_t)c * S);
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const float d = D::get(v.v[i]) - mean[i];
                    q[i] += d * d;
                }
            }
        }
        column_sum<VE, LX, NW>(q, lds);
        float rstd[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i)
            rstd[i] = 1.0f / sqrtf(q[i] * inv + a.eps);
        if (!live)
            continue;
        if (a.mean && w == 0 && ly == 0)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                a.mean[j + i] = mean[i];
                a.rstd[j + i] = rstd[i];
            }
        const auto store = [&](int c, const V& in) {
            const float g = a.gamma ? a.gamma[c] : 1.0f, b = a.beta ? a.beta[c] : 0.0f;
            V v;
#pragma unroll
            for (int i = 0; i < VE; ++i)
                v.v[i] = D::put((D::get(in.v[i]) - mean[i]) * rstd[i] * g + b);
            *(V*)(y + (int64_t)c * S) = v;
        };
        if constexpr (CACHED) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (c0 + p * P::STEP < C)
                    store(c0 + p * P::STEP, keep[p]);
        } else {
            for (int c = c0; c < C; c += P::STEP)
                store(c, *(const V*)(x + (int64_t)c * S));
        }
    }
}

template <typename D, int VE, int LX, int NW, int NP, bool CACHED>
__global__ __launch_bounds__(NW * 64) void norm_bwd_planes(NormArgs a)
{
    using T = typename D::T;
    using V = Vec<T, VE>;
    using P = Plane<VE, LX, NW>;
    __shared__ float lds[1][NW][P::W];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, lx = lane % LX, ly = lane / LX;
    const int C = a.C, S = a.S, c0 = w * P::LY + ly;
    const float inv = 1.0f / (float)C;
    const int64_t cols = a.M * S, tiles = (cols + P::W - 1) / P::W;
    float gg[NP] = {}, gb[NP] = {};
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t j = t * P::W + lx * VE;
        const bool live = j < cols;
        const int64_t m = live ? j / S : 0;
        const int64_t base = live ? m * C * S + (j - m * S) : 0;
        const T* __restrict__ x = (const T*)a.x + base;
        const T* __restrict__ gy = (const T*)a.gy + base;
        T* __restrict__ gx = (T*)a.out + base;
        float mean[VE], rstd[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            mean[i] = live ? a.mean[j + i] : 0.0f;
            rstd[i] = live ? a.rstd[j + i] : 0.0f;
        }
        float sa[VE] = {}, sh[VE] = {};
        const auto add = [&](int c, const V& vx, const V& vg, float& g1, float& g2) {
            const float gam = a.gamma ? a.gamma[c] : 1.0f;
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const float g = D::get(vg.v[i]), xh = (D::get(vx.v[i]) - mean[i]) * rstd[i];
                g1 += g * xh;
                g2 += g;
                sa[i] += g * gam;
                sh[i] += g * gam * xh;
            }
        };
        V kx[NP], kg[NP];
        if constexpr (CACHED) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int c = c0 + p * P::STEP;
                if (live && c < C) {
                    kx[p] = *(const V*)(x + (int64_t)c * S);
                    kg[p] = *(const V*)(gy + (int64_t)c * S);
                }
            }
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (live && c0 + p * P::STEP < C)
                    add(c0 + p * P::STEP, kx[p], kg[p], gg[p], gb[p]);
        } else if (live) {
            for (int c = c0; c < C; c += P::STEP) {
                float g1 = 0.0f, g2 = 0.0f;  // (the weights' sums are norm_bwd_planes_weights' there)
                add(c, *(const V*)(x + (int64_t)c * S), *(const V*)(gy + (int64_t)c * S), g1, g2);
            }
        }
        column_sum<VE, LX, NW>(sa, lds);
        column_sum<VE, LX, NW>(sh, lds);
        if (!live)
            continue;
        const auto store = [&](int c, const V& vx, const V& vg) {
            const float gam = a.gamma ? a.gamma[c] : 1.0f;
            V v;
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const float xh = (D::get(vx.v[i]) - mean[i]) * rstd[i];
                v.v[i] = D::put(rstd[i] * (D::get(vg.v[i]) * gam - sa[i] * inv - xh * (sh[i] * inv)));
            }
            *(V*)(gx + (int64_t)c * S) = v;
        };
        if constexpr (CACHED) {
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (c0 + p * P::STEP < C)
                    store(c0 + p * P::STEP, kx[p], kg[p]);
        } else {
            for (int c = c0; c < C; c += P::STEP)
                store(c, *(const V*)(x + (int64_t)c * S), *(const V*)(gy + (int64_t)c * S));
        }
    }
    if constexpr (CACHED) {
        if (!a.part)
            return;
        float* __restrict__ part = a.part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
#pragma unroll
            for (int o = 1; o < LX; o <<= 1) {
                gg[p] += __shfl_xor(gg[p], o);
                gb[p] += __shfl_xor(gb[p], o);
            }
            const int c = c0 + p * P::STEP;
            if (lx == 0 && c < C) {
                part[c] = gg[p];
                part[C + c] = gb[p];
            }
        }
    }
}

// a wave sums one channel over the columns of its block's share
template <typename D>
__global__ __launch_bounds__(kT) void norm_bwd_planes_weights(NormArgs a)
{
    using T = typename D::T;
    const int C = a.C, S = a.S, lane = threadIdx.x & 63;
    const int64_t c = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (c >= C)
        return;
    const int64_t cols = a.M * S;
    float gg = 0.0f, gb = 0.0f;
    for (int64_t j = (int64_t)blockIdx.y * 64 + lane; j < cols; j += (int64_t)gridDim.y * 64) {
        const int64_t m = j / S, i = (m * C + c) * S + (j - m * S);
        const float g = D::get(((const T*)a.gy)[i]);
        gg += g * ((D::get(((const T*)a.x)[i]) - a.mean[j]) * a.rstd[j]);
        gb += g;
    }
    gg = wave_sum(gg);
    gb = wave_sum(gb);
    if (lane == 0) {
        float* __restrict__ part = a.part + (int64_t)blockIdx.y * 2 * C;
        part[c] = gg;
        part[C + c] = gb;
    }
}

// grad_gamma, grad_beta from the blocks' partial sums: 16 threads a column,
// joined in a fixed order
__global__ __launch_bounds__(kT) void norm_weights_kernel(const float* __restrict__ part, int blocks, int C,
                                                          float* __restrict__ gg, float* __restrict__ gb)
{
    __shared__ double lds[16][16];
    const int col = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int64_t e = (int64_t)blockIdx.x * 16 + col;  // 0 .. 2C-1
    double s = 0.0;
    if (e < 2 * (int64_t)C)
        for (int b = row; b < blocks; b += 16)
            s += (double)part[(int64_t)b * 2 * C + e];
    lds[row][col] = s;
    __syncthreads();
    if (row != 0 || e >= 2 * (int64_t)C)
        return;
    for (int r = 1; r < 16; ++r)
        s += lds[r][col];
    float* __restrict__ out = e < C ? gg : gb;
    if (out)
        out[e < C ? e : e - C] = (float)s;
}

hipError_t last() { return hipGetLastError(); }

template <typename D, int VE, int NV, int WPR>
hipError_t rows(const NormArgs& a, bool bwd, int blocks, hipStream_t s)
{
    if (bwd)
        norm_bwd_rows<D, VE, NV, WPR><<<dim3(blocks), dim3(kT), 0, s>>>(a);
    else
        norm_fwd_rows<D, VE, NV, WPR><<<dim3(blocks), dim3(kT), 0, s>>>(a);
    return last();
}

// the smallest of the kernels whose registers hold a row: a wave of up to
// 32 elements a lane, else four waves; false: none does
template <typename D, int VE>
bool launch_rows(const NormArgs& a, bool bwd, int blocks, hipStream_t s, hipError_t* err)
{
    const int64_t per = ((int64_t)a.C + VE - 1) / VE;  // loads of a row
    constexpr int MAX = 32 / VE < 8 ? 32 / VE : 8;
    const auto fits = [&](int nv, int wpr) { return per <= (int64_t)nv * 64 * wpr; };
    if (fits(1, 1)) *err = rows<D, VE, 1, 1>(a, bwd, blocks, s);
    else if (fits(2, 1)) *err = rows<D, VE, 2, 1>(a, bwd, blocks, s);
    else if (fits(4, 1)) *err = rows<D, VE, 4, 1>(a, bwd, blocks, s);
    else if (MAX == 8 && fits(8, 1)) *err = rows<D, VE, MAX, 1>(a, bwd, blocks, s);
    else if (fits(4, 4)) *err = rows<D, VE, 4, 4>(a, bwd, blocks, s);
    else if (MAX == 8 && fits(8, 4)) *err = rows<D, VE, MAX, 4>(a, bwd, blocks, s);
    else return false;
    return true;
}

template <typename D, int VE, int LX, int NW, int NP, bool CACHED>
hipError_t planes(const NormArgs& a, bool bwd, int blocks, hipStream_t s)
{
    if (bwd)
        norm_bwd_planes<D, VE, LX, NW, NP, CACHED><<<dim3(blocks), dim3(NW * 64), 0, s>>>(a);
    else
        norm_fwd_planes<D, VE, LX, NW, NP, CACHED><<<dim3(blocks), dim3(NW * 64), 0, s>>>(a);
    return last();
}

template <typename D, int VE, int LX>
hipError_t launch_planes(const NormArgs& a, bool bwd, int blocks, hipStream_t s, bool* cached)
{
    constexpr int LY = 64 / LX;
    *cached = a.C <= 16 * 16 * LY;
    if (a.C <= 4 * 16 * LY)
        return planes<D, VE, LX, 4, 16, true>(a, bwd, blocks, s);
    if (*cached)
        return planes<D, VE, LX, 16, 16, true>(a, bwd, blocks, s);
    return planes<D, VE, LX, 16, 1, false>(a, bwd, blocks, s);
}

template <typename D> hipError_t run(const NormArgs& a, bool bwd, hipStream_t s)
{
    constexpr int VE = 16 / sizeof(typename D::T);
    const int blocks = norm_blocks(a.M, a.C, a.S);
    const auto al = [&](size_t n) {
        return (uintptr_t)a.x % n == 0 && (uintptr_t)a.out % n == 0 && (!bwd || (uintptr_t)a.gy % n == 0);
    };
    bool whole = true;  // the kernel sums the weights' gradients too
    hipError_t err = hipSuccess;
    if (a.S == 1) {
        const int grid = bwd ? blocks : (int)((a.M + 3) / 4 < (1 << 20) ? (a.M + 3) / 4 : (1 << 20));
        const bool done = a.C % VE == 0 && al(16) ? launch_rows<D, VE>(a, bwd, grid, s, &err)
                                                  : launch_rows<D, 1>(a, bwd, grid, s, &err);
        if (!done) {
            whole = false;
            const int g = (int)(a.M < (1 << 20) ? a.M : (1 << 20));
            if (bwd)
                norm_bwd_long<D><<<dim3(g), dim3(kT), 0, s>>>(a);
            else
                norm_fwd_long<D><<<dim3(g), dim3(kT), 0, s>>>(a);
            err = last();
        }
    } else {
        const int64_t tiles = (a.M * a.S + 63) / 64;
        const int grid = bwd ? blocks : (int)(tiles < (1 << 20) ? tiles : (1 << 20));
        err = a.S % 4 == 0 && al(4 * sizeof(typename D::T)) ? launch_planes<D, 4, 16>(a, bwd, grid, s, &whole)
                                                            : launch_planes<D, 1, 64>(a, bwd, grid, s, &whole);
    }
    if (err != hipSuccess || !bwd || !a.part)
        return err;
    if (!whole) {
        if (a.S == 1)
            norm_bwd_long_weights<D><<<dim3((a.C + kT - 1) / kT, blocks), dim3(kT), 0, s>>>(a);
        else
            norm_bwd_planes_weights<D><<<dim3((a.C + 3) / 4, blocks), dim3(kT), 0, s>>>(a);
        if ((err = last()) != hipSuccess)
            return err;
    }
    norm_weights_kernel<<<dim3((unsigned)((2 * (int64_t)a.C + 15) / 16)), dim3(kT), 0, s>>>(a.part, blocks, a.C, a.grad_gamma,
                                                                                        a.grad_beta);
    return last();
}

}  // namespace

hipError_t launch_norm_forward(const NormArgs& a, int dtype, hipStream_t s)
{
    return dtype == kBF16 ? run<BF16>(a, false, s) : run<F32>(a, false, s);
}

hipError_t launch_norm_backward(const NormArgs& a, int dtype, hipStream_t s)
{
    return dtype == kBF16 ? run<BF16>(a, true, s) : run<F32>(a, true, s);
}

}  // namespace mfpsn
