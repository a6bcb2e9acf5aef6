// 16x16 matrix products of one wave on gfx950's matrix cores, as the
// gated-delta-rule kernels use them: operands from LDS, or a result fed back
// as the next product's right operand without leaving the registers.
//
// A result tile D (16x16) has column lane % 16 in a lane, rows 4 g + r in its
// register r, g = lane / 16.  A right operand needs column lane % 16 too, and
// for its contraction index any fixed order, as long as the left operand has
// the same.  So the order is chosen such that a result's registers are a
// right operand as they are: f32 contracts one tile's 16 rows in four
// v_mfma_f32_16x16x4_f32, number r over the rows {4 g + r}; bf16 contracts two
// tiles' 32 rows in one v_mfma_f32_16x16x32_bf16, lane group g over the rows
// 4 g .. 4 g + 3 of the first tile, then those of the second.  A chain of
// products (state -> residuals -> values -> state) then needs no LDS round
// trip and no barrier.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mfpsn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma_f32(const f32x4 a, const f32x4 b, f32x4 c)
{
#pragma unroll
    for (int r = 0; r < 4; ++r)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
    return c;
}

template <bool BF> struct Mat;

template <> struct Mat<false> {
    using El = float;
    using Frag = f32x4;
    static constexpr int KU = 16;   // rows that one product contracts
    static constexpr int TU = 1;    // result tiles that make one right operand
    static constexpr int PAD = 4;   // elements between the rows of an LDS tile: rows start 4 banks apart
    // operand from LDS [m][k]: rows m0 .. m0 + 15 (p points at row m0), contraction block u
    __device__ static Frag rows(const El* p, int ld, int u)
    {
        const int lane = threadIdx.x & 63;
        return *(const f32x4*)(p + (lane & 15) * ld + 16 * u + 4 * (lane >> 4));
    }
    // operand from LDS [k][m]: columns 0 .. 15 of p
    __device__ static Frag cols(const El* p, int ld, int u)
    {
        const int lane = threadIdx.x & 63;
        const El* s = p + (16 * u + 4 * (lane >> 4)) * ld + (lane & 15);
        return f32x4{s[0], s[ld], s[2 * ld], s[3 * ld]};
    }
    __device__ static Frag pack(const f32x4* t) { return t[0]; }
    __device__ static f32x4 mma(Frag a, Frag b, f32x4 c) { return mfma_f32(a, b, c); }
    __device__ static El put(float v) { return v; }
    __device__ static float get(El v) { return v; }
};

template <> struct Mat<true> {
    using El = __bf16;
    using Frag = bf16x8;
    static constexpr int KU = 32, TU = 2, PAD = 8;
    __device__ static Frag join(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
    __device__ static Frag rows(const El* p, int ld, int u)
    {
        const int lane = threadIdx.x & 63;
        const El* s = p + (lane & 15) * ld + 32 * u + 4 * (lane >> 4);
        return join(*(const bf16x4*)s, *(const bf16x4*)(s + 16));
    }
    // 16 lanes read 4 rows of 16 columns, 8 bytes each, and get a column's 4 rows each
    __device__ static bf16x4 transposed(const El* p)
    {
        const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
        return __builtin_bit_cast(bf16x4, v);
    }
    __device__ static Frag cols(const El* p, int ld, int u)
    {
        const int lane = threadIdx.x & 63, i = lane & 15;
        const El* s = p + (32 * u + 4 * (lane >> 4) + (i >> 2)) * ld + 4 * (i & 3);
        return join(transposed(s), transposed(s + 16 * ld));
    }
    __device__ static Frag pack(const f32x4* t)
    {
        return __builtin_convertvector(__builtin_shufflevector(t[0], t[1], 0, 1, 2, 3, 4, 5, 6, 7), Frag);
    }
    // what pack() left of each value, as the next 8 bits
    __device__ static Frag pack_rest(const f32x4* t, Frag hi)
    {
        const u32x4 h = __builtin_bit_cast(u32x4, hi);
        f32x8 f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = t[i >> 2][i & 3] - __builtin_bit_cast(float, i & 1 ? h[i >> 1] & 0xffff0000u : h[i >> 1] << 16);
        return __builtin_convertvector(f, Frag);
    }
    __device__ static f32x4 mma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    __device__ static El put(float v) { return (__bf16)v; }
    __device__ static float get(El v) { return (float)v; }
};

// Storage types of the tensors
struct StoreF32 {
    using T = float;
    __device__ static float get(T v) { return v; }
    __device__ static T put(float v) { return v; }
};
struct StoreBF16 {
    using T = __bf16;
    __device__ static float get(T v) { return (float)v; }
    __device__ static T put(float v) { return (__bf16)v; }  // to nearest even
};

// Keeps what stands before it before what stands behind it.  The operands of
// several products are read from LDS together, one group ahead of the products
// that use them; left to itself the compiler reads each where it is used and
// waits for it, about 100 cycles a product.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// Address of row r, rows `stride` bytes apart
template <typename T> __device__ __forceinline__ const T* row_at(const T* p, int r, uint32_t stride)
{
    return (const T*)((const char*)p + (uint64_t)(uint32_t)r * stride);
}

// ROWS rows of `cols` elements from memory, `stride` bytes apart, on their way
// into LDS rows of `ld` elements: load() issues every read at once (the values
// wait in registers, so that reads of the next tile run while this one is
// computed with), store() writes them, zeros in rows from `live` on and from
// column `cols` to COLS.  Reads outside that range go to the last row or first
// column instead (live >= 1), never outside the tensor.  VEC: rows are 16-byte
// aligned and cols is a multiple of 16 bytes.  near: ROWS * stride fits 32 bits;
// a whole tile is then read at one 32-bit offset a thread behind scalar row
// addresses, which leaves no address arithmetic to the lanes.
template <typename D, typename El, int COLS, int THREADS, bool VEC, int ROWS = 64> struct Rows {
    using T = typename D::T;
    static_assert(sizeof(El) == sizeof(T));
    static constexpr int VE = 16 / sizeof(T), PER = COLS / VE, STEP = THREADS / PER, NL = (ROWS + STEP - 1) / STEP;
    static_assert(COLS % VE == 0 && THREADS % PER == 0 && ROWS % STEP == 0);
    u32x4 v[NL];

    __device__ __forceinline__ void load(const T* src, uint32_t stride, int live, int cols, bool near)
    {
        const int r0 = threadIdx.x / PER, c = (threadIdx.x % PER) * VE;
        if constexpr (VEC) {
            const int c1 = c < cols ? c : 0;
            if (live >= ROWS && near) {
                const uint32_t off = (uint32_t)r0 * stride + (uint32_t)c1 * (uint32_t)sizeof(T);
#pragma unroll
                for (int n = 0; n < NL; ++n)
                    v[n] = *(const u32x4*)((const char*)src + (uint64_t)(n * STEP) * stride + off);
            } else {
#pragma unroll
                for (int n = 0; n < NL; ++n)
                    v[n] = *(const u32x4*)row_at(src + c1, min(r0 + n * STEP, live - 1), stride);
            }
        } else {
#pragma unroll
            for (int n = 0; n < NL; ++n) {
                const T* p = row_at(src, min(r0 + n * STEP, live - 1), stride);
                alignas(16) T e[VE];
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    e[j] = p[c + j < cols ? c + j : 0];
                    if (c + j >= cols)
                        e[j] = D::put(0.0f);
                }
                v[n] = *(const u32x4*)e;
            }
        }
    }
    __device__ __forceinline__ void store(El* lds, int ld, int live, int cols)
    {
        const int r0 = threadIdx.x / PER, c = (threadIdx.x % PER) * VE;
        El* d = lds + r0 * ld + c;
        if (live >= ROWS && cols == COLS) {
#pragma unroll
            for (int n = 0; n < NL; ++n)
                *(u32x4*)(d + n * STEP * ld) = v[n];
        } else {
#pragma unroll
            for (int n = 0; n < NL; ++n) {
                const bool in = r0 + n * STEP < live && c < cols;
                *(u32x4*)(d + n * STEP * ld) = u32x4{in ? v[n].x : 0, in ? v[n].y : 0, in ? v[n].z : 0, in ? v[n].w : 0};
            }
        }
    }
};

// The same for ROWS x COLS elements that lie densely in one of the kernels' own
// arrays; rows from `live` (>= 1) on become zeros
template <typename El, int ROWS, int COLS, int THREADS> struct Dense {
    static constexpr int VE = 16 / sizeof(El), PER = COLS / VE, STEP = THREADS / PER, NL = (ROWS + STEP - 1) / STEP;
    static_assert(THREADS % PER == 0 && ROWS % STEP == 0);
    u32x4 v[NL];

    __device__ __forceinline__ void load(const El* src, int live = ROWS)
    {
        const int r0 = threadIdx.x / PER, c = (threadIdx.x % PER) * VE;
        if (live >= ROWS) {
            const uint32_t off = (uint32_t)(r0 * COLS + c) * (uint32_t)sizeof(El);
#pragma unroll
            for (int n = 0; n < NL; ++n)
                v[n] = *(const u32x4*)((const char*)(src + n * STEP * COLS) + off);
        } else {
#pragma unroll
            for (int n = 0; n < NL; ++n)
                v[n] = *(const u32x4*)(src + min(r0 + n * STEP, live - 1) * COLS + c);
        }
    }
    __device__ __forceinline__ void store(El* lds, int ld, int live = ROWS)
    {
        const int r0 = threadIdx.x / PER, c = (threadIdx.x % PER) * VE;
        El* d = lds + r0 * ld + c;
        if (live >= ROWS) {
#pragma unroll
            for (int n = 0; n < NL; ++n)
                *(u32x4*)(d + n * STEP * ld) = v[n];
        } else {
#pragma unroll
            for (int n = 0; n < NL; ++n) {
                const bool in = r0 + n * STEP < live;
                *(u32x4*)(d + n * STEP * ld) = u32x4{in ? v[n].x : 0, in ? v[n].y : 0, in ? v[n].z : 0, in ? v[n].w : 0};
            }
        }
    }
};

// A column's values at the steps of four result tiles (row 16 t + 4 g + r in
// [t][r]); steps from `live` on give the last one's, whatever it holds
template <typename T> struct Column {
    T x[4][4];

    __device__ __forceinline__ void load(const T* src, int v, uint32_t stride, int live, bool near)
    {
        const int g4 = 4 * ((threadIdx.x & 63) >> 4);
        if (live >= 64 && near) {
            const uint32_t off = (uint32_t)g4 * stride + (uint32_t)v * (uint32_t)sizeof(T);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[t][r] = *(const T*)((const char*)src + (uint64_t)(16 * t + r) * stride + off);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[t][r] = *row_at(src + v, min(16 * t + g4 + r, live - 1), stride);
        }
    }
};

// The reverse: steps below `live` are written
template <typename D>
__device__ __forceinline__ void store_column(const f32x4* x, typename D::T* dst, int v, uint32_t stride, int live, bool near)
{
    using T = typename D::T;
    const int g4 = 4 * ((threadIdx.x & 63) >> 4);
    if (live >= 64 && near) {
        const uint32_t off = (uint32_t)g4 * stride + (uint32_t)v * (uint32_t)sizeof(T);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *(T*)((char*)dst + (uint64_t)(16 * t + r) * stride + off) = D::put(x[t][r]);
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * t + g4 + r < live)
                    *const_cast<T*>(row_at(dst + v, 16 * t + g4 + r, stride)) = D::put(x[t][r]);
    }
}

// Four consecutive values of a result tile's column
template <bool BF> __device__ __forceinline__ void put4(typename Mat<BF>::El* p, const f32x4 v)
{
    if constexpr (BF)
        *(bf16x4*)p = __builtin_convertvector(v, bf16x4);
    else
        *(f32x4*)p = v;
}

}  // namespace mfpsn
