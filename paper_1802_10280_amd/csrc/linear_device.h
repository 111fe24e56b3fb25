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

__device__ inline float activate(float z, uint32_t flags) {
    if (flags & ESCOIN_F_RELU) return z > 0.0f ? z : 0.0f;
    if (flags & ESCOIN_F_SILU) return z / (1.0f + expf(-z));
    if (flags & ESCOIN_F_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
    // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), which keeps its bits where tanh is near -1
    if (flags & ESCOIN_F_GELU_TANH) return z / (1.0f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
    return z;
}

template <int TYPE>
__device__ inline float number(const char* p, int64_t i) {
    return (float)((const typename Num<TYPE>::type*)p)[i];
}

// What follows the sums of four neighbouring rows (from `row`, a multiple of four) for one token: bias, activation, gate,
// residual, and the store.  A gated layer's rows are a gate, its partner, the next gate, its partner.
template <int TYPE, bool GATED>
__device__ inline void finish(const LinearArgs& a, f4 z, int row, int token) {
    typedef typename Num<TYPE>::type N;
    if (token >= a.T || row >= a.rows) return;
    constexpr int kOut = GATED ? 2 : 4;
    const int m0 = GATED ? row >> 1 : row;
    N* const out = (N*)(a.out + token * a.ld_out) + m0;
    const N* const residual = (const N*)(a.residual + token * a.ld_residual) + m0;
    float v[kOut];
#pragma unroll
    for (int i = 0; i < kOut; ++i) {
        if (m0 + i >= a.M) break;
        if constexpr (GATED) {
            float g = z[2 * i], u = z[2 * i + 1];
            if (a.bias) g += number<TYPE>(a.bias, m0 + i), u += number<TYPE>(a.bias, a.M + m0 + i);
            v[i] = activate(g, a.flags) * u;
        } else {
            v[i] = activate(a.bias ? z[i] + number<TYPE>(a.bias, m0 + i) : z[i], a.flags);
        }
        if (a.residual) v[i] += (float)residual[i];
    }
    if (m0 + kOut <= a.M && ((uintptr_t)out & (kOut * sizeof(N) - 1)) == 0) {
        typedef N Nv __attribute__((ext_vector_type(kOut)));
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

// 16 bytes of a token's row from byte `at` on, zeros beyond `end`.  WIDE: rows start on 16 bytes and hold a multiple of them.
template <int TYPE, bool WIDE>
__device__ inline u4 input16(const LinearArgs& a, const char* row, int at, int end) {
    if constexpr (WIDE) {
        return *(const u4*)(at < end ? row + at : a.zero);
    } else {
        typedef typename Num<TYPE>::type N;
        constexpr int kN = 16 / sizeof(N);
        struct __attribute__((packed, aligned(sizeof(N)))) Raw {
            u4 v;
        };
        if (at + 16 <= end) return ((const Raw*)(row + at))->v;
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

inline bool wide_input(const LinearArgs& a, int size) {
    return (((uintptr_t)a.in | (uintptr_t)a.ld_in | (uintptr_t)((int64_t)a.K * size)) & 15) == 0;
}

}  // namespace escoin
