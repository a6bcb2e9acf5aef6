// gfx950 kernels of the gated delta rule over whole sequences, forward and
// backward:
//   S_t = e^{g_t} S_{t-1} + beta_t k_t (v_t - e^{g_t} S_{t-1}^T k_t)^T,
//   o_t = scale S_t^T q_t,          S [Dk][Dv] per sequence and value head.
//
// Chunks of 64 steps turn the recurrence into matrix products.  Within a chunk,
// with G_i = g_1 + .. + g_i, M_ij = e^{G_i - G_j} (i >= j), the state S0 before
// it and the residuals r_i = v_i - e^{g_i} S_{i-1}^T k_i:
//   (I + A) r = V - diag(e^G) K S0,      A_ij = M_ij (k_i.k_j) beta_j  (i > j)
//   O  = scale diag(e^G) Q S0 + P r,     P_ij = scale M_ij (q_i.k_j) beta_j  (i >= j)
//   S1 = e^{G_last} S0 + K^T diag(e^{G_last - G} beta) r
// X = (I + A)^-1 and P depend on no state: delta_prep computes them for all
// chunks at once.  delta_scan walks the chunks in order with the state in
// registers.  Exponents are differences of G in double, at most 0 for decays,
// so a step that forgets everything (g = -inf) harms no other.
//
// Backward, with dO and the gradient dS1 of the state behind the chunk:
//   dr' = P^T dO + diag(e^{G_last - G} beta) K dS1,    dV = X^T dr'
//   dS0 = e^{G_last} dS1 + scale Q^T diag(e^G) dO - K^T diag(e^G) dV
// walked in reverse by delta_rscan, and, with both states at hand, for all
// chunks at once in delta_grads (E_ij = scale M_ij beta_j (dO r^T)_ij, i >= j,
// F_ij = -M_ij beta_j (dV r^T)_ij, i > j):
//   dQ = scale diag(e^G) dO S0^T + E K
//   dK = E^T Q + (F + F^T) K + diag(e^{G_last - G} beta) r dS1^T - diag(e^G) dV S0^T
//   dbeta_j = (sum_i E_ij (q_i.k_j) + F_ij (k_i.k_j)) / beta_j + e^{G_last - G_j} k_j.(dS1 r_j)
//   dg_t = sum_{i >= t > j} (E_ij (q_i.k_j) + F_ij (k_i.k_j)) + e^{G_last} <S0, dS1>
//          + sum_{i >= t} e^{G_i} (scale q_i.(S0 dO_i) - k_i.(S0 dV_i))
//          + sum_{j < t} e^{G_last - G_j} beta_j k_j.(dS1 r_j)
// (the quotient by beta_j is taken before the factor goes in).  Value heads that
// share a key head are summed by the block that has the key head.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mfpsn_delta.h"
#include "mfpsn_delta_mat.h"
#include "mfpsn_internal.h"

namespace mfpsn {
namespace {

constexpr int L = kDeltaChunk;
constexpr int LF = L + 4;  // LDS row of a float L x L matrix

__device__ __forceinline__ int length_of(const DeltaArgs& a, int n)
{
    return a.lengths ? min(max(a.lengths[n], 0), a.T) : a.T;
}

// A decay so strong that its exponential is 0 acts as e^-1000 (also 0): sums of
// it stay finite, and so do their differences
__device__ __forceinline__ double decay_of(float g) { return (double)(g < -1000.0f ? -1000.0f : g); }

// Inclusive sums of g over the 64 lanes of a wave
__device__ __forceinline__ double running_sum(double v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double u = __shfl_up(v, o);
        if (lane >= o)
            v += u;
    }
    return v;
}

// The unit (sequence, value head, chunk) of the per-chunk arrays
__device__ __forceinline__ int64_t unit_of(const DeltaArgs& a, int n, int hv, int c)
{
    return ((int64_t)n * a.Hv + hv) * a.nc + c;
}

// X = (I + A)^-1 of the strictly lower triangle A [L][LF] in LDS, by four
// waves: the 16x16 diagonal blocks by substitution (a lane has one column of
// one block), then twice joined, [[X0, 0], [-X1 A10 X0, X1]].  In float
// throughout; substitution and blocks of it stay accurate where the powers of
// A that a product form needs would grow (nearly equal keys).
__device__ void unit_lower_inverse(const float* A, float* X)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4;
    for (int i = tid; i < L * L; i += 256) {
        const int r = i / L, k = i % L;
        if ((r >> 4) != (k >> 4))
            X[r * LF + k] = 0.0f;
    }
    if (wave == 0) {
        const float* a = A + (16 * g) * LF + 16 * g;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == c ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; ++j)
                s = __builtin_fmaf(-a[i * LF + j], x[j], s);
            x[i] = s;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            X[(16 * g + i) * LF + 16 * g + c] = x[i];
    }
    __syncthreads();
    using M = Mat<false>;
    if (wave < 2) {
        const int lo = 32 * wave, hi = lo + 16;
        f32x4 y = {0, 0, 0, 0}, z = {0, 0, 0, 0};
        y = M::mma(M::rows(A + hi * LF + lo, LF, 0), M::cols(X + lo * LF + lo, LF, 0), y);
        z = M::mma(M::rows(X + hi * LF + hi, LF, 0), y, z);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            X[(hi + 4 * g + r) * LF + lo + c] = -z[r];
    }
    __syncthreads();
    {
        const int q = 16 * (wave & 1), p = 32 + 16 * (wave >> 1);
        f32x4 y[2], z = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            y[i] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < 2; ++u)
                y[i] = M::mma(M::rows(A + (32 + 16 * i) * LF, LF, u), M::cols(X + q, LF, u), y[i]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
            z = M::mma(M::rows(X + p * LF + 32, LF, u), y[u], z);
        // (rows 32.. of columns 0..31 are read by no wave here)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            X[(p + 4 * g + r) * LF + q + c] = -z[r];
    }
    __syncthreads();
}

// X, P and the gates of a chunk, for the value heads of one key head
template <typename D, bool BF, int DKP> struct PrepLds {
    using El = typename Mat<BF>::El;
    static constexpr int LDK = DKP + Mat<BF>::PAD;
    El k[L * LDK], q[L * LDK];
    float A[L * LF], X[L * LF];
    double G[L];
    float beta[L];
};

template <typename D, bool BF, int DKP>
__global__ __launch_bounds__(256) void delta_prep(DeltaArgs a)
{
    using T = typename D::T;
    using M = Mat<BF>;
    using El = typename M::El;
    using Lds = PrepLds<D, BF, DKP>;
    __shared__ Lds s;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g4 = 4 * (lane >> 4);
    const int c = blockIdx.x % a.nc;
    const int64_t nh = blockIdx.x / a.nc;
    const int n = (int)(nh / a.Hk), hk = (int)(nh - (int64_t)n * a.Hk), group = a.Hv / a.Hk;
    const int t0 = c * L, live = min(L, length_of(a, n) - t0);
    if (live <= 0)
        return;
    const int64_t row0 = (int64_t)t0 * a.N + n;
    stage<D, El, DKP, 256>(s.k, Lds::LDK, (const T*)a.k + row0 * a.k_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.k_row, live,
                           a.Dk, a.vec_qk);
    stage<D, El, DKP, 256>(s.q, Lds::LDK, (const T*)a.q + row0 * a.q_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.q_row, live,
                           a.Dk, a.vec_qk);
    __syncthreads();
    // (K K^T)[j][i] and (K Q^T)[j][i]: column i = 16 wave + col of every row tile j <= i
    f32x4 kk[4], kq[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
        kk[t] = kq[t] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < DKP / M::KU; ++u) {
        const auto bk = M::rows(s.k + 16 * wave * Lds::LDK, Lds::LDK, u);
        const auto bq = M::rows(s.q + 16 * wave * Lds::LDK, Lds::LDK, u);
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (t <= wave) {
                const auto ak = M::rows(s.k + 16 * t * Lds::LDK, Lds::LDK, u);
                kk[t] = M::mma(ak, bk, kk[t]);
                kq[t] = M::mma(ak, bq, kq[t]);
            }
    }
    const int i = 16 * wave + col;
    for (int r = 0; r < group; ++r) {
        const int hv = hk * group + r;
        const int64_t unit = unit_of(a, n, hv, c);
        if (wave == 0) {
            const int64_t at = (row0 + (int64_t)lane * a.N) * a.Hv + hv;
            const double G = running_sum(lane < live ? decay_of(D::get(((const T*)a.g)[at])) : 0.0);
            s.G[lane] = G;
            s.beta[lane] = lane < live ? D::get(((const T*)a.beta)[at]) : 0.0f;
            float* gate = a.gate + unit * 2 * L;
            gate[lane] = expf((float)G);
            gate[L + lane] = expf((float)(__shfl(G, 63) - G));
        }
        __syncthreads();
        El* P = (El*)a.P + unit * L * L;
        const double Gi = s.G[i];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int j0 = 16 * t + g4;
            f32x4 av = {0, 0, 0, 0}, pv = {0, 0, 0, 0};
            if (t <= wave)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + e;
                    if (j <= i) {
                        const float m = expf((float)(Gi - s.G[j])) * s.beta[j];
                        pv[e] = a.scale * m * kq[t][e];
                        av[e] = j < i ? m * kk[t][e] : 0.0f;
                    }
                }
            *(f32x4*)(s.A + i * LF + j0) = av;
            alignas(16) El e4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                e4[e] = M::put(pv[e]);
            if constexpr (BF)
                *(uint2*)(P + i * L + j0) = *(const uint2*)e4;
            else
                *(uint4*)(P + i * L + j0) = *(const uint4*)e4;
        }
        __syncthreads();
        unit_lower_inverse(s.A, s.X);
        // 16-bit: X as the sum of two numbers of 8 bits each (the scan's products need it as exactly as float)
        El* X = (El*)a.X + unit * L * L * (BF ? 2 : 1);
        for (int e = tid * 4; e < L * L; e += 1024) {
            const f32x4 x = *(const f32x4*)(s.X + (e / L) * LF + e % L);
            if constexpr (BF) {
                bf16x4 hi, lo;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    hi[j] = (__bf16)x[j];
                    lo[j] = (__bf16)(x[j] - (float)hi[j]);
                }
                *(bf16x4*)(X + e) = hi;
                *(bf16x4*)(X + L * L + e) = lo;
            } else {
                *(f32x4*)(X + e) = x;
            }
        }
        __syncthreads();
    }
}

// The chunks of one sequence and value head in order.  A wave has 16 columns
// of the state, all Dk rows, in registers, and everything that is computed from
// them: residuals, outputs and the state itself go from product to product
// without leaving the wave.  The block's waves share the chunk's K, Q, X and P
// in LDS.
template <typename D, bool BF, int DKP> struct ScanLds {
    using El = typename Mat<BF>::El;
    static constexpr int LDK = DKP + Mat<BF>::PAD, LDL = L + Mat<BF>::PAD;
    El k[L * LDK], q[L * LDK];
    El x[BF ? 2 : 1][L * LDL], p[L * LDL];
    float gate[2][L], beta[L];
};

template <typename D, bool BF, int DKP, int NW>
__global__ __launch_bounds__(NW * 64) void delta_scan(DeltaArgs a)
{
    using T = typename D::T;
    using M = Mat<BF>;
    using El = typename M::El;
    using Frag = typename M::Frag;
    using Lds = ScanLds<D, BF, DKP>;
    constexpr int TK = DKP / 16, TH = NW * 64, KU = M::KU, TU = M::TU, UL = L / KU;
    __shared__ Lds s;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g4 = 4 * (lane >> 4);
    const int vblocks = (a.dvp + 16 * NW - 1) / (16 * NW);
    const int64_t head = blockIdx.x / vblocks;
    const int n = (int)(head / a.Hv), hv = (int)(head - (int64_t)n * a.Hv), hk = hv / (a.Hv / a.Hk);
    const int v = ((int)(blockIdx.x % vblocks) * NW + wave) * 16 + col;
    const bool mine = v < a.Dv;          // a column of the tensors
    const bool wide = v - col < a.dvp;   // the wave has columns of the padded arrays
    const int len = length_of(a, n), chunks = (len + L - 1) / L;
    f32x4 S[TK];
#pragma unroll
    for (int t = 0; t < TK; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = 16 * t + g4 + r;
            S[t][r] = a.state_in && mine && d < a.Dk ? a.state_in[(head * a.Dk + d) * a.Dv + v] : 0.0f;
        }
    for (int c = 0; c < chunks; ++c) {
        const int t0 = c * L, live = min(L, len - t0);
        const int64_t row0 = (int64_t)t0 * a.N + n, unit = unit_of(a, n, hv, c);
        __syncthreads();
        stage<D, El, DKP, TH>(s.k, Lds::LDK, (const T*)a.k + row0 * a.k_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.k_row,
                              live, a.Dk, a.vec_qk);
        stage<D, El, DKP, TH>(s.q, Lds::LDK, (const T*)a.q + row0 * a.q_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.q_row,
                              live, a.Dk, a.vec_qk);
        stage_dense<El, L, L, TH>(s.x[0], Lds::LDL, (const El*)a.X + unit * L * L * (BF ? 2 : 1));
        if constexpr (BF)
            stage_dense<El, L, L, TH>(s.x[1], Lds::LDL, (const El*)a.X + unit * L * L * 2 + L * L);
        stage_dense<El, L, L, TH>(s.p, Lds::LDL, (const El*)a.P + unit * L * L);
        for (int i = tid; i < L; i += TH) {
            s.gate[0][i] = a.gate[unit * 2 * L + i];
            s.gate[1][i] = a.gate[unit * 2 * L + L + i];
            s.beta[i] = i < live ? D::get(((const T*)a.beta)[(row0 + (int64_t)i * a.N) * a.Hv + hv]) : 0.0f;
        }
        f32x4 R[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + g4 + r;
                R[t][r] = mine && i < live ? D::get(((const T*)a.v)[(row0 + (int64_t)i * a.N) * a.v_row + (int64_t)hv * a.Dv + v])
                                           : 0.0f;
            }
        __syncthreads();
        if (a.S0 && wide) {  // [v][d], for the backward
            El* S0 = (El*)a.S0 + (unit * a.dvp + v) * DKP;
#pragma unroll
            for (int t = 0; t < TK; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    S0[16 * t + g4 + r] = M::put(S[t][r]);
        }
        // K S0 and Q S0.  16-bit: the state goes in as two numbers of 8 bits each for the residuals (they
        // make the next state, which is kept in float), as one for the outputs (rounded to 8 bits anyway).
        f32x4 KS[4], O[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
            KS[t] = O[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < DKP / KU; ++u) {
            const Frag b = M::pack(S + u * TU);
            Frag rest;
            if constexpr (BF)
                rest = M::pack_rest(S + u * TU, b);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const Frag ak = M::rows(s.k + 16 * t * Lds::LDK, Lds::LDK, u);
                KS[t] = M::mma(ak, b, KS[t]);
                if constexpr (BF)
                    KS[t] = M::mma(ak, rest, KS[t]);
                O[t] = M::mma(M::rows(s.q + 16 * t * Lds::LDK, Lds::LDK, u), b, O[t]);
            }
        }
        f32x4 eG[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            eG[t] = *(const f32x4*)(s.gate[0] + 16 * t + g4);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                R[t][r] = __builtin_fmaf(-eG[t][r], KS[t][r], R[t][r]);
        }
        // residuals r = X R (X is lower triangular)
        f32x4 U[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
            U[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < UL; ++u) {
            const Frag b = M::pack(R + u * TU);
            Frag rest;
            if constexpr (BF)
                rest = M::pack_rest(R + u * TU, b);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (u * KU < 16 * (t + 1)) {
                    const Frag ax = M::rows(s.x[0] + 16 * t * Lds::LDL, Lds::LDL, u);
                    U[t] = M::mma(ax, b, U[t]);
                    if constexpr (BF) {
                        U[t] = M::mma(ax, rest, U[t]);
                        U[t] = M::mma(M::rows(s.x[1] + 16 * t * Lds::LDL, Lds::LDL, u), b, U[t]);
                    }
                }
        }
        if (a.U && wide) {  // [v][i]
            El* pu = (El*)a.U + (unit * a.dvp + v) * L;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    pu[16 * t + g4 + r] = M::put(U[t][r]);
        }
        // outputs
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                O[t][r] *= a.scale * eG[t][r];
#pragma unroll
        for (int u = 0; u < UL; ++u) {
            const Frag b = M::pack(U + u * TU);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (u * KU < 16 * (t + 1))
                    O[t] = M::mma(M::rows(s.p + 16 * t * Lds::LDL, Lds::LDL, u), b, O[t]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + g4 + r;
                if (mine && i < live)
                    ((T*)a.o)[((row0 + (int64_t)i * a.N) * a.Hv + hv) * a.Dv + v] = D::put(O[t][r]);
            }
        // the state behind the chunk
        const float last = s.gate[0][L - 1];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const f32x4 e = *(const f32x4*)(s.gate[1] + 16 * t + g4), b = *(const f32x4*)(s.beta + 16 * t + g4);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                U[t][r] *= e[r] * b[r];
        }
#pragma unroll
        for (int t = 0; t < TK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                S[t][r] *= last;
#pragma unroll
        for (int u = 0; u < UL; ++u) {
            const Frag b = M::pack(U + u * TU);
            Frag rest;
            if constexpr (BF)
                rest = M::pack_rest(U + u * TU, b);
#pragma unroll
            for (int t = 0; t < TK; ++t) {
                const Frag ak = M::cols(s.k + 16 * t, Lds::LDK, u);
                S[t] = M::mma(ak, b, S[t]);
                if constexpr (BF)
                    S[t] = M::mma(ak, rest, S[t]);
            }
        }
    }
    if (!mine)
        return;
    for (int t = len + (lane >> 4); t < a.T; t += 4)  // steps behind the sequence's end
        ((T*)a.o)[(((int64_t)t * a.N + n) * a.Hv + hv) * a.Dv + v] = D::put(0.0f);
    if (a.state_out)
#pragma unroll
        for (int t = 0; t < TK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 16 * t + g4 + r;
                if (d < a.Dk)
                    a.state_out[(head * a.Dk + d) * a.Dv + v] = S[t][r];
            }
}

// The chunks in reverse: the gradient of the state, the values' gradient
template <typename D, bool BF, int DKP> struct RscanLds {
    using El = typename Mat<BF>::El;
    static constexpr int LDK = DKP + Mat<BF>::PAD, LDL = L + Mat<BF>::PAD;
    El k[L * LDK], q[L * LDK], x[L * LDL], p[L * LDL];
    float gate[2][L], beta[L];
};

template <typename D, bool BF, int DKP, int NW>
__global__ __launch_bounds__(NW * 64) void delta_rscan(DeltaArgs a)
{
    using T = typename D::T;
    using M = Mat<BF>;
    using El = typename M::El;
    using Frag = typename M::Frag;
    using Lds = RscanLds<D, BF, DKP>;
    constexpr int TK = DKP / 16, TH = NW * 64, KU = M::KU, TU = M::TU, UL = L / KU;
    __shared__ Lds s;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g4 = 4 * (lane >> 4);
    const int vblocks = (a.dvp + 16 * NW - 1) / (16 * NW);
    const int64_t head = blockIdx.x / vblocks;
    const int n = (int)(head / a.Hv), hv = (int)(head - (int64_t)n * a.Hv), hk = hv / (a.Hv / a.Hk);
    const int v = ((int)(blockIdx.x % vblocks) * NW + wave) * 16 + col;
    const bool mine = v < a.Dv, wide = v - col < a.dvp;
    const int len = length_of(a, n), chunks = (len + L - 1) / L;
    f32x4 S[TK];
#pragma unroll
    for (int t = 0; t < TK; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = 16 * t + g4 + r;
            S[t][r] = a.grad_state_out && mine && d < a.Dk ? a.grad_state_out[(head * a.Dk + d) * a.Dv + v] : 0.0f;
        }
    for (int c = chunks - 1; c >= 0; --c) {
        const int t0 = c * L, live = min(L, len - t0);
        const int64_t row0 = (int64_t)t0 * a.N + n, unit = unit_of(a, n, hv, c);
        __syncthreads();
        stage<D, El, DKP, TH>(s.k, Lds::LDK, (const T*)a.k + row0 * a.k_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.k_row,
                              live, a.Dk, a.vec_qk);
        stage<D, El, DKP, TH>(s.q, Lds::LDK, (const T*)a.q + row0 * a.q_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.q_row,
                              live, a.Dk, a.vec_qk);
        stage_dense<El, L, L, TH>(s.x, Lds::LDL, (const El*)a.X + unit * L * L * (BF ? 2 : 1));
        stage_dense<El, L, L, TH>(s.p, Lds::LDL, (const El*)a.P + unit * L * L);
        for (int i = tid; i < L; i += TH) {
            s.gate[0][i] = a.gate[unit * 2 * L + i];
            s.gate[1][i] = a.gate[unit * 2 * L + L + i];
            s.beta[i] = i < live ? D::get(((const T*)a.beta)[(row0 + (int64_t)i * a.N) * a.Hv + hv]) : 0.0f;
        }
        f32x4 dO[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + g4 + r;
                dO[t][r] = mine && i < live ? D::get(((const T*)a.grad_o)[((row0 + (int64_t)i * a.N) * a.Hv + hv) * a.Dv + v])
                                            : 0.0f;
            }
        __syncthreads();
        if (wide) {  // [v][d], for delta_grads
            El* dS = (El*)a.dS + (unit * a.dvp + v) * DKP;
#pragma unroll
            for (int t = 0; t < TK; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    dS[16 * t + g4 + r] = M::put(S[t][r]);
        }
        // dr' = diag(e^{G_last - G} beta) K dS1 + P^T dO
        f32x4 R[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
            R[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < DKP / KU; ++u) {
            const Frag b = M::pack(S + u * TU);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                R[t] = M::mma(M::rows(s.k + 16 * t * Lds::LDK, Lds::LDK, u), b, R[t]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const f32x4 e = *(const f32x4*)(s.gate[1] + 16 * t + g4), b = *(const f32x4*)(s.beta + 16 * t + g4);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                R[t][r] *= e[r] * b[r];
        }
#pragma unroll
        for (int u = 0; u < UL; ++u) {
            const Frag b = M::pack(dO + u * TU);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if ((u + 1) * KU > 16 * t)
                    R[t] = M::mma(M::cols(s.p + 16 * t, Lds::LDL, u), b, R[t]);
        }
        // dV = X^T dr'
        f32x4 dV[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
            dV[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < UL; ++u) {
            const Frag b = M::pack(R + u * TU);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if ((u + 1) * KU > 16 * t)
                    dV[t] = M::mma(M::cols(s.x + 16 * t, Lds::LDL, u), b, dV[t]);
        }
        const float last = s.gate[0][L - 1];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const f32x4 eG = *(const f32x4*)(s.gate[0] + 16 * t + g4);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + g4 + r;
                if (mine && i < live)
                    ((T*)a.grad_v)[((row0 + (int64_t)i * a.N) * a.Hv + hv) * a.Dv + v] = D::put(dV[t][r]);
                dO[t][r] *= a.scale * eG[r];
                dV[t][r] *= -eG[r];
            }
        }
        // dS0
#pragma unroll
        for (int t = 0; t < TK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                S[t][r] *= last;
#pragma unroll
        for (int u = 0; u < UL; ++u) {
            const Frag bo = M::pack(dO + u * TU), bv = M::pack(dV + u * TU);
#pragma unroll
            for (int t = 0; t < TK; ++t) {
                S[t] = M::mma(M::cols(s.q + 16 * t, Lds::LDK, u), bo, S[t]);
                S[t] = M::mma(M::cols(s.k + 16 * t, Lds::LDK, u), bv, S[t]);
            }
        }
    }
    if (!mine)
        return;
    for (int t = len + (lane >> 4); t < a.T; t += 4)
        ((T*)a.grad_v)[(((int64_t)t * a.N + n) * a.Hv + hv) * a.Dv + v] = D::put(0.0f);
    if (a.grad_state_in)
#pragma unroll
        for (int t = 0; t < TK; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 16 * t + g4 + r;
                if (d < a.Dk)
                    a.grad_state_in[(head * a.Dk + d) * a.Dv + v] = S[t][r];
            }
}

// The gradients of a chunk's queries, keys, decays and write strengths, for
// one key head.  All products are computed transposed: wave w has the columns
// i = 16 w .. 16 w + 15 (steps) of every result, so a step's factors are one
// value a lane, and E^T, F^T in registers are the right operands of E K, F K.
template <typename D, bool BF, int DKP> struct GradsLds {
    using El = typename Mat<BF>::El;
    static constexpr int VB = BF ? 64 : 32;  // values staged at a time
    static constexpr int LDK = DKP + Mat<BF>::PAD, LDL = L + Mat<BF>::PAD, LDV = VB + Mat<BF>::PAD;
    El k[L * LDK], q[L * LDK];
    union {
        struct {
            El dO[L * LDV], dV[L * LDV], r[VB * LDL], S0[VB * LDK], dS[VB * LDK];
        } v;
        struct {
            El E[L * LDL], F[L * LDL];  // [i][j]
        } m;
    };
    double G[L];
    float eG[L], to_end[L], beta[L];
    float sum[4][L];           // over a wave's steps i, of each step j
    float a[L], x[L], row[L];  // of each step
    float z[4];
};

template <typename D, bool BF, int DKP>
__global__ __launch_bounds__(256) void delta_grads(DeltaArgs a)
{
    using T = typename D::T;
    using M = Mat<BF>;
    using El = typename M::El;
    using Frag = typename M::Frag;
    using Lds = GradsLds<D, BF, DKP>;
    constexpr int TK = DKP / 16, KU = M::KU, TU = M::TU, UL = L / KU, VB = Lds::VB;
    __shared__ Lds s;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, g4 = 4 * (lane >> 4);
    const int c = blockIdx.x % a.nc;
    const int64_t nh = blockIdx.x / a.nc;
    const int n = (int)(nh / a.Hk), hk = (int)(nh - (int64_t)n * a.Hk), group = a.Hv / a.Hk;
    const int t0 = c * L, live = max(0, min(L, length_of(a, n) - t0)), steps = min(L, a.T - t0);
    const int64_t row0 = (int64_t)t0 * a.N + n;
    const int i = 16 * wave + col;
    f32x4 dq[TK], dk[TK];
#pragma unroll
    for (int t = 0; t < TK; ++t)
        dq[t] = dk[t] = f32x4{0, 0, 0, 0};
    if (live > 0) {
        stage<D, El, DKP, 256>(s.k, Lds::LDK, (const T*)a.k + row0 * a.k_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.k_row,
                               live, a.Dk, a.vec_qk);
        stage<D, El, DKP, 256>(s.q, Lds::LDK, (const T*)a.q + row0 * a.q_row + (int64_t)hk * a.Dk, (int64_t)a.N * a.q_row,
                               live, a.Dk, a.vec_qk);
        __syncthreads();
        f32x4 kk[4], kq[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
            kk[t] = kq[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < DKP / KU; ++u) {
            const Frag bk = M::rows(s.k + 16 * wave * Lds::LDK, Lds::LDK, u);
            const Frag bq = M::rows(s.q + 16 * wave * Lds::LDK, Lds::LDK, u);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t <= wave) {
                    const Frag ak = M::rows(s.k + 16 * t * Lds::LDK, Lds::LDK, u);
                    kk[t] = M::mma(ak, bk, kk[t]);
                    kq[t] = M::mma(ak, bq, kq[t]);
                }
        }
        for (int h = 0; h < group; ++h) {
            const int hv = hk * group + h;
            const int64_t unit = unit_of(a, n, hv, c);
            if (wave == 0) {
                const int64_t at = (row0 + (int64_t)lane * a.N) * a.Hv + hv;
                const double G = running_sum(lane < live ? decay_of(D::get(((const T*)a.g)[at])) : 0.0);
                s.G[lane] = G;
                s.beta[lane] = lane < live ? D::get(((const T*)a.beta)[at]) : 0.0f;
                s.eG[lane] = expf((float)G);
                s.to_end[lane] = expf((float)(__shfl(G, 63) - G));
            }
            // products over the values
            f32x4 qs[TK], ks[TK], ws[TK], dP[4], dA[4];
#pragma unroll
            for (int t = 0; t < TK; ++t)
                qs[t] = ks[t] = ws[t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < 4; ++t)
                dP[t] = dA[t] = f32x4{0, 0, 0, 0};
            float z = 0.0f;  // <S0, dS1>
            for (int v0 = 0; v0 < a.dvp; v0 += VB) {
                const int rows = min(VB, a.dvp - v0), cols = min(VB, a.Dv - v0);
                __syncthreads();
                const int64_t at = (row0 * a.Hv + hv) * a.Dv + v0;
                stage<D, El, VB, 256>(s.v.dO, Lds::LDV, (const T*)a.grad_o + at, (int64_t)a.N * a.Hv * a.Dv, live, cols,
                                      a.vec_v);
                stage<D, El, VB, 256>(s.v.dV, Lds::LDV, (const T*)a.grad_v + at, (int64_t)a.N * a.Hv * a.Dv, live, cols,
                                      a.vec_v);
                stage_dense<El, VB, L, 256>(s.v.r, Lds::LDL, (const El*)a.U + (unit * a.dvp + v0) * L, rows);
                stage_dense<El, VB, DKP, 256>(s.v.S0, Lds::LDK, (const El*)a.S0 + (unit * a.dvp + v0) * DKP, rows);
                stage_dense<El, VB, DKP, 256>(s.v.dS, Lds::LDK, (const El*)a.dS + (unit * a.dvp + v0) * DKP, rows);
                __syncthreads();
                for (int e = tid; e < VB * DKP; e += 256) {
                    const int at2 = (e / DKP) * Lds::LDK + e % DKP;
                    z = __builtin_fmaf(M::get(s.v.S0[at2]), M::get(s.v.dS[at2]), z);
                }
#pragma unroll
                for (int u = 0; u < VB / KU; ++u) {
                    const Frag bo = M::rows(s.v.dO + 16 * wave * Lds::LDV, Lds::LDV, u);
                    const Frag bv = M::rows(s.v.dV + 16 * wave * Lds::LDV, Lds::LDV, u);
                    const Frag br = M::cols(s.v.r + 16 * wave, Lds::LDL, u);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (t <= wave) {
                            const Frag ar = M::cols(s.v.r + 16 * t, Lds::LDL, u);
                            dP[t] = M::mma(ar, bo, dP[t]);
                            dA[t] = M::mma(ar, bv, dA[t]);
                        }
#pragma unroll
                    for (int t = 0; t < TK; ++t) {
                        const Frag as = M::cols(s.v.S0 + 16 * t, Lds::LDK, u);
                        qs[t] = M::mma(as, bo, qs[t]);
                        ks[t] = M::mma(as, bv, ks[t]);
                        ws[t] = M::mma(M::cols(s.v.dS + 16 * t, Lds::LDK, u), br, ws[t]);
                    }
                }
            }
            __syncthreads();
            // E^T, F^T in place of dP, dA; sums over i and j of their products with q.k and k.k
            const double Gi = s.G[i];
            float row = 0.0f;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                f32x4 y = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = 16 * t + g4 + e;
                    const float m = t <= wave && j <= i ? expf((float)(Gi - s.G[j])) : 0.0f;
                    const float E = a.scale * m * dP[t][e], F = j < i ? -m * dA[t][e] : 0.0f;
                    y[e] = E * kq[t][e] + F * kk[t][e];
                    const float b = s.beta[j];
                    row = __builtin_fmaf(b, y[e], row);
                    dP[t][e] = E * b;
                    dA[t][e] = F * b;
                }
#pragma unroll
                for (int o = 1; o < 16; o <<= 1)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        y[e] += __shfl_xor(y[e], o);
                if (col == 0)
                    *(f32x4*)(s.sum[wave] + 16 * t + g4) = y;
                El* pe = s.m.E + i * Lds::LDL + 16 * t + g4;
                El* pf = s.m.F + i * Lds::LDL + 16 * t + g4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pe[e] = M::put(dP[t][e]);
                    pf[e] = M::put(dA[t][e]);
                }
            }
            row += __shfl_xor(row, 16);
            row += __shfl_xor(row, 32);
            // products with the states, and what the gates take of them
            float ra = 0.0f, rx = 0.0f;
            const float eG = s.eG[i], to_end = s.to_end[i], bi = s.beta[i];
#pragma unroll
            for (int t = 0; t < TK; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int d = 16 * t + g4 + e;
                    const float kd = M::get(s.k[i * Lds::LDK + d]), qd = M::get(s.q[i * Lds::LDK + d]);
                    const float dq1 = a.scale * eG * qs[t][e], dk1 = eG * ks[t][e], dk2 = to_end * ws[t][e];
                    ra += qd * dq1 - kd * dk1;
                    rx += kd * dk2;
                    dq[t][e] += dq1;
                    dk[t][e] += bi * dk2 - dk1;
                }
            ra += __shfl_xor(ra, 16);
            ra += __shfl_xor(ra, 32);
            rx += __shfl_xor(rx, 16);
            rx += __shfl_xor(rx, 32);
            if (lane < 16) {
                s.row[i] = row;
                s.a[i] = ra;
                s.x[i] = rx;
            }
#pragma unroll
            for (int o = 1; o < 64; o <<= 1)
                z += __shfl_xor(z, o);
            if (lane == 0)
                s.z[wave] = z;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < UL; ++u) {
                const Frag bE = M::pack(dP + u * TU), bF = M::pack(dA + u * TU);
                const Frag cE = M::cols(s.m.E + 16 * wave, Lds::LDL, u), cF = M::cols(s.m.F + 16 * wave, Lds::LDL, u);
#pragma unroll
                for (int t = 0; t < TK; ++t) {
                    const Frag ak = M::cols(s.k + 16 * t, Lds::LDK, u);
                    dq[t] = M::mma(ak, bE, dq[t]);
                    dk[t] = M::mma(ak, bF, dk[t]);
                    dk[t] = M::mma(ak, cF, dk[t]);
                    dk[t] = M::mma(M::cols(s.q + 16 * t, Lds::LDK, u), cE, dk[t]);
                }
            }
            if (wave == 0) {
                const float colsum = (s.sum[0][lane] + s.sum[1][lane]) + (s.sum[2][lane] + s.sum[3][lane]);
                const float x = s.x[lane], b = s.beta[lane];
                // sum_{i >= t} of what step i reads, less what it wrote: pairs with both ends behind t cancel
                const double read = (double)s.a[lane] + s.row[lane] - (double)b * colsum, wrote = (double)b * x;
                const double upto = running_sum(read), before = running_sum(wrote) - wrote;
                const double zz = (double)s.eG[L - 1] * (((double)s.z[0] + s.z[1]) + ((double)s.z[2] + s.z[3]));
                const float dg = (float)(__shfl(upto, 63) - upto + read + before + zz);
                const float db = colsum + x;
                if (lane < steps) {
                    const int64_t at = (row0 + (int64_t)lane * a.N) * a.Hv + hv;
                    ((T*)a.grad_g)[at] = D::put(lane < live ? dg : 0.0f);
                    ((T*)a.grad_beta)[at] = D::put(lane < live ? db : 0.0f);
                }
            }
            __syncthreads();
        }
    } else if (tid < steps) {  // a chunk behind the sequence's end
        for (int h = 0; h < group; ++h) {
            const int64_t at = (row0 + (int64_t)tid * a.N) * a.Hv + hk * group + h;
            ((T*)a.grad_g)[at] = D::put(0.0f);
            ((T*)a.grad_beta)[at] = D::put(0.0f);
        }
    }
    if (i < steps) {
        const int64_t at = ((row0 + (int64_t)i * a.N) * a.Hk + hk) * a.Dk;
        const float keep = i < live ? 1.0f : 0.0f;
#pragma unroll
        for (int t = 0; t < TK; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = 16 * t + g4 + e;
                if (d < a.Dk) {
                    ((T*)a.grad_q)[at + d] = D::put(keep * dq[t][e]);
                    ((T*)a.grad_k)[at + d] = D::put(keep * dk[t][e]);
                }
            }
    }
}

template <typename D, bool BF, int DKP> hipError_t forward(const DeltaArgs& a, hipStream_t s)
{
    if (a.nc > 0) {
        delta_prep<D, BF, DKP><<<dim3((unsigned)((int64_t)a.N * a.Hk * a.nc)), dim3(256), 0, s>>>(a);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess)
            return err;
    }
    constexpr int NW = 4;
    const int64_t blocks = (int64_t)a.N * a.Hv * ((a.dvp + 16 * NW - 1) / (16 * NW));
    delta_scan<D, BF, DKP, NW><<<dim3((unsigned)blocks), dim3(NW * 64), 0, s>>>(a);
    return hipGetLastError();
}

template <typename D, bool BF, int DKP> hipError_t backward(const DeltaArgs& a, hipStream_t s)
{
    constexpr int NW = 4;
    const int64_t blocks = (int64_t)a.N * a.Hv * ((a.dvp + 16 * NW - 1) / (16 * NW));
    delta_rscan<D, BF, DKP, NW><<<dim3((unsigned)blocks), dim3(NW * 64), 0, s>>>(a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || a.nc == 0)
        return err;
    delta_grads<D, BF, DKP><<<dim3((unsigned)((int64_t)a.N * a.Hk * a.nc)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_forward(const DeltaArgs& a, int dtype, hipStream_t s)
{
    const bool wide = delta_dkp(a.Dk) == 128;
    if (dtype == kBF16)
        return wide ? forward<StoreBF16, kDeltaBf16Products, 128>(a, s) : forward<StoreBF16, kDeltaBf16Products, 64>(a, s);
    return wide ? forward<StoreF32, false, 128>(a, s) : forward<StoreF32, false, 64>(a, s);
}

hipError_t launch_delta_backward(const DeltaArgs& a, int dtype, hipStream_t s)
{
    const bool wide = delta_dkp(a.Dk) == 128;
    if (dtype == kBF16)
        return wide ? backward<StoreBF16, kDeltaBf16Products, 128>(a, s) : backward<StoreBF16, kDeltaBf16Products, 64>(a, s);
    return wide ? backward<StoreF32, false, 128>(a, s) : backward<StoreF32, false, 64>(a, s);
}

}  // namespace mfpsn
