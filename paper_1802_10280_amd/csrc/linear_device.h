// Device code that the linear layers' kernels share: element types, and what follows the sums.
#pragma once
#include "linear.h"

namespace escoin {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) void* Lds;
typedef __amdgpu_buffer_rsrc_t Buffer;

// Memory by way of a buffer: offsets of 32 bits, zeros where the lane's own one reaches `bytes`.
__device__ inline Buffer buffer(const char* p, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, 0x00020000); }
__device__ inline u4 load16(Buffer from, int lane_offset, int offset) { return __builtin_amdgcn_raw_buffer_load_b128(from, lane_offset, offset, 0); }

// What stands before it in the source is issued before it: a wait that counts the loads on their way goes by their order.
__device__ inline void in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// 16 bytes a lane: 1024 of LDS from `to` on
__device__ inline void copy16(Buffer from, int lane_offset, int offset, char* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (Lds)to, 16, lane_offset, offset, 0, 0);
}

template <int TYPE>
struct Num;
template <>
struct Num<ESCOIN_T_F32> {
    typedef float type;
};
template <>
struct Num<ESCOIN_T_F16> {
    typedef _Float16 type;
};
template <>
struct Num<ESCOIN_T_BF16> {
    typedef __bf16 type;
};

// 16 rows of weights by 16 tokens: a lane's 16 bytes of each are row (token) lane % 16 and the columns from lane / 16 * 16 bytes
// on.  Sums: token lane % 16, rows lane / 16 * 4 + 0..3.
template <int TYPE>
__device__ inline f4 mfma16(u4 w, u4 x, f4 c) {
    if constexpr (TYPE == ESCOIN_T_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, w), __builtin_bit_cast(b8, x), c, 0, 0, 0);
    if constexpr (TYPE == ESCOIN_T_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, w), __builtin_bit_cast(h8, x), c, 0, 0, 0);
    if constexpr (TYPE == ESCOIN_T_F32) {
        // the instruction takes one column a lane: it gets the lanes' first ones, then their second ones, ...
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[j]), __uint_as_float(x[j]), c, 0, 0, 0);
        return c;
    }
}

// The same with 32 rows by 32 tokens: columns from lane / 32 * 16 bytes on; sums of token lane % 32, rows
// i / 4 * 8 + lane / 32 * 4 + i % 4.
template <int TYPE>
__device__ inline f16v mfma32(u4 w, u4 x, f16v c) {
    if constexpr (TYPE == ESCOIN_T_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, w), __builtin_bit_cast(b8, x), c, 0, 0, 0);
    if constexpr (TYPE == ESCOIN_T_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, w), __builtin_bit_cast(h8, x), c, 0, 0, 0);
    if constexpr (TYPE == ESCOIN_T_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[j]), __uint_as_float(x[j]), c, 0, 0, 0);
        return c;
    }
}

// z / (1 + exp(-u)).  For outputs of 16 bits the instructions' own exponential and reciprocal, each a step of fp32 or two off, do; the
// library's forms, some 40 instructions, are an eighth of a long prompt's time.
// Far below zero it is z exp(u), to all of fp32's bits, in two factors that stay in range: exp(-u) passes 2^128, and from 2^126 on the reciprocal
// instruction gives zero, while the result is a number of fp32 and bf16 still.
template <int TYPE, int N>
__device__ inline void logistic(float (&z)[N], const float (&u)[N]) {
    if constexpr (TYPE == ESCOIN_T_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool far = u[i] < -80.0f;
            const float e = expf(far ? 0.5f * u[i] : -u[i]);
            z[i] = far ? z[i] * e * e : z[i] / (1.0f + e);
        }
    } else {
        float p[N];
        bool far = false;
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = -1.44269504088896341f * u[i], far |= p[i] > 120.0f;
        if (__builtin_expect(far, 0)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float e = __builtin_amdgcn_exp2f(p[i] > 120.0f ? 64.0f - p[i] : p[i]);
                z[i] = p[i] > 120.0f ? z[i] * e * 0x1p-64f : z[i] * __builtin_amdgcn_rcpf(1.0f + e);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] *= __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(p[i]));
    }
}

template <int TYPE, int N>
__device__ inline void activate(float (&z)[N], uint32_t flags) {
    if (flags & ESCOIN_F_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] > 0.0f ? z[i] : 0.0f;
    } else if (flags & ESCOIN_F_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = 0.5f * z[i] * erfcf(-0.70710678118654752f * z[i]);
    } else if (flags & (ESCOIN_F_SILU | ESCOIN_F_GELU_TANH)) {
        // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), which keeps its bits where tanh is near -1
        float u[N];
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = flags & ESCOIN_F_SILU ? z[i] : 1.5957691216057308f * (z[i] + 0.044715f * z[i] * z[i] * z[i]);
        logistic<TYPE>(z, u);
    }
}

// What follows the sums of R * 4 neighbouring rows (from `row`, a multiple of R * 4) for one token: bias, activation, gate,
// residual, and the store.  A gated layer's rows are a gate, its partner, the next gate, its partner.
template <int TYPE, bool GATED, int R>
__device__ inline void finish(const LinearArgs& a, const f4 (&z)[R], int row, int token) {
    typedef typename Num<TYPE>::type N;
    if (token >= a.T || row >= a.rows) return;
    constexpr int kOut = GATED ? 2 * R : 4 * R;
    typedef N Nv __attribute__((ext_vector_type(kOut)));
    const int m0 = GATED ? row >> 1 : row;
    const bool whole = m0 + kOut <= a.M;
    // as many neighbours as there are, by element where they end or where they do not start on their size
    const auto get = [&](const char* p, N (&to)[kOut]) {
        if (whole && ((uintptr_t)p & (kOut * sizeof(N) - 1)) == 0) {
            const Nv v = *(const Nv*)p;
#pragma unroll
            for (int i = 0; i < kOut; ++i) to[i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < kOut; ++i) to[i] = m0 + i < a.M ? ((const N*)p)[i] : (N)0.0f;
        }
    };
    float v[kOut];
    N b[kOut];
    if constexpr (GATED) {
        N c[kOut];
        if (a.bias) get(a.bias + m0 * sizeof(N), b), get(a.bias + ((int64_t)a.M + m0) * sizeof(N), c);
        float u[kOut];
#pragma unroll
        for (int i = 0; i < kOut; ++i) {
            v[i] = z[i / 2][i % 2 * 2], u[i] = z[i / 2][i % 2 * 2 + 1];
            if (a.bias) v[i] += (float)b[i], u[i] += (float)c[i];
        }
        activate<TYPE>(v, a.flags);
#pragma unroll
        for (int i = 0; i < kOut; ++i) v[i] *= u[i];
    } else {
        if (a.bias) get(a.bias + m0 * sizeof(N), b);
#pragma unroll
        for (int i = 0; i < kOut; ++i) v[i] = a.bias ? z[i / 4][i % 4] + (float)b[i] : z[i / 4][i % 4];
        activate<TYPE>(v, a.flags);
    }
    if (a.residual) {
        get(a.residual + token * a.ld_residual + m0 * sizeof(N), b);
#pragma unroll
        for (int i = 0; i < kOut; ++i) v[i] += (float)b[i];
    }
    N* const out = (N*)(a.out + token * a.ld_out) + m0;
    if (whole && ((uintptr_t)out & (kOut * sizeof(N) - 1)) == 0) {
        Nv o;
#pragma unroll
        for (int i = 0; i < kOut; ++i) o[i] = (N)v[i];
        *(Nv*)out = o;
    } else {
#pragma unroll
        for (int i = 0; i < kOut; ++i)
            if (m0 + i < a.M) out[i] = (N)v[i];
    }
}

// 16 bytes from any element on
template <int TYPE>
__device__ inline u4 any16(const char* p) {
    struct __attribute__((packed, aligned(sizeof(typename Num<TYPE>::type)))) Raw {
        u4 v;
    };
    return ((const Raw*)p)->v;
}

// 16 bytes of a token's row from byte `at` on, zeros beyond `end`.  WIDE: rows start on 16 bytes and hold a multiple of them.
template <int TYPE, bool WIDE>
__device__ inline u4 input16(const LinearArgs& a, const char* row, int at, int end) {
    if constexpr (WIDE) {
        return *(const u4*)(at < end ? row + at : a.zero);
    } else {
        typedef typename Num<TYPE>::type N;
        constexpr int kN = 16 / sizeof(N);
        if (at + 16 <= end) return any16<TYPE>(row + at);
        typedef N Nv __attribute__((ext_vector_type(kN)));
        Nv v = {};
        if (at < end)
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (at + i * (int)sizeof(N) < end) v[i] = ((const N*)(row + at))[i];
        return __builtin_bit_cast(u4, v);
    }
}

}  // namespace

// Whether inputs come by wide loads: rows on 16 bytes that hold a multiple of them, and a tile's rows within 32 bits of offsets.
inline bool wide_input(const LinearArgs& a, int size) {
    return (((uintptr_t)a.in | (uintptr_t)a.ld_in | (uintptr_t)((int64_t)a.K * size)) & 15) == 0 && a.ld_in < 1 << 23;
}

}  // namespace escoin
