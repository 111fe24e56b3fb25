// The residual stream between two blocks: h = alpha x + beta gate post(y), n = pre(h), one row to a workgroup.
#include "linear_device.h"

namespace escoin {
namespace {

struct NormArgs {
    const void *x, *y, *gate, *post_weight, *post_bias, *pre_weight, *pre_bias;
    void *h, *n;
    int64_t ld_x, ld_y, ld_gate, ld_h, ld_n;  // elements
    int T, D, post, pre, gate_rows;
    float eps, alpha, beta, offset;
};

constexpr int kThreads = 256;

// The sum over a workgroup, the same for each of its threads.
__device__ inline float all_sum(float v, float* lds) {
#pragma unroll
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.0f;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) t += lds[w];
    return t;
}

struct Stats {
    float mean, scale;
};

// Of f(i) over a row: two passes for a layer norm, the squares of the deviations and not a difference of sums.
template <class F>
__device__ inline Stats stats(const NormArgs& a, int kind, float* lds, F f) {
    Stats s = {0.0f, 1.0f};
    if (kind == ESCOIN_NORM_NONE) return s;
    float v = 0.0f;
    if (kind == ESCOIN_NORM_LAYER) {
        for (int i = threadIdx.x; i < a.D; i += blockDim.x) v += f(i);
        s.mean = all_sum(v, lds) / (float)a.D;
    }
    v = 0.0f;
    for (int i = threadIdx.x; i < a.D; i += blockDim.x) {
        const float u = f(i) - s.mean;
        v = fmaf(u, u, v);
    }
    s.scale = 1.0f / sqrtf(all_sum(v, lds) / (float)a.D + a.eps);
    return s;
}

template <class N>
__device__ inline float normed(float v, int kind, const Stats& s, const void* weight, const void* bias, float offset, int i) {
    if (kind == ESCOIN_NORM_NONE) return v;
    v = (v - s.mean) * s.scale;
    if (weight) v *= (float)((const N*)weight)[i] + offset;
    if (bias) v += (float)((const N*)bias)[i];
    return v;
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void norm_kernel(const NormArgs a) {
    typedef typename Num<TYPE>::type N;
    __shared__ float lds[kThreads / 64];
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
        const N* const x = (const N*)a.x + t * a.ld_x;
        const N* const y = (const N*)a.y + t * a.ld_y;
        const N* const gate = (const N*)a.gate + (a.gate_rows ? t * a.ld_gate : 0);
        const Stats post = stats(a, a.y ? a.post : ESCOIN_NORM_NONE, lds, [&](int i) { return (float)y[i]; });
        const auto sum = [&](int i) {
            float v = a.alpha * (float)x[i];
            if (a.y) {
                float b = a.beta * normed<N>((float)y[i], a.post, post, a.post_weight, a.post_bias, a.offset, i);
                if (a.gate) b *= (float)gate[i];
                v += b;
            }
            return v;
        };
        const Stats pre = stats(a, a.n ? a.pre : ESCOIN_NORM_NONE, lds, sum);
        for (int i = threadIdx.x; i < a.D; i += blockDim.x) {
            const float v = sum(i);
            if (a.h) ((N*)a.h)[t * a.ld_h + i] = (N)v;
            if (a.n) ((N*)a.n)[t * a.ld_n + i] = (N)normed<N>(v, a.pre, pre, a.pre_weight, a.pre_bias, a.offset, i);
        }
    }
}

int make_norm_args(const escoin_norm_desc* desc, NormArgs* a) {
    if (!desc) return ESCOIN_EINVAL;
    const escoin_norm_desc& p = *desc;
    const auto kind = [](int k) { return k >= ESCOIN_NORM_NONE && k <= ESCOIN_NORM_LAYER; };
    if (p.T < 0 || p.D < 1 || p.type < ESCOIN_T_F32 || p.type > ESCOIN_T_BF16 || !kind(p.post) || !kind(p.pre) || (p.gate_rows & ~1)) return ESCOIN_EINVAL;
    if (!(p.eps >= 0.0f) || !(fabsf(p.alpha) < INFINITY) || !(fabsf(p.beta) < INFINITY) || !(fabsf(p.weight_offset) < INFINITY) || !(p.eps < INFINITY))
        return ESCOIN_EINVAL;
    const int64_t given[5] = {p.ld_x, p.ld_y, p.ld_gate, p.ld_h, p.ld_n};
    int64_t* const to[5] = {&a->ld_x, &a->ld_y, &a->ld_gate, &a->ld_h, &a->ld_n};
    for (int i = 0; i < 5; ++i) {
        *to[i] = given[i] == 0 ? p.D : given[i];
        if (*to[i] < p.D) return ESCOIN_EINVAL;
        if (*to[i] >= 1ll << 40) return ESCOIN_ERANGE;
    }
    if (p.D >= 1 << 30) return ESCOIN_ERANGE;
    a->T = p.T; a->D = p.D; a->post = p.post; a->pre = p.pre; a->gate_rows = p.gate_rows;
    a->eps = p.eps; a->alpha = p.alpha; a->beta = p.beta; a->offset = p.weight_offset;
    return ESCOIN_OK;
}

}  // namespace
}  // namespace escoin

using namespace escoin;

extern "C" {

int escoin_norm_check_desc(const escoin_norm_desc* desc) {
    NormArgs a;
    return make_norm_args(desc, &a);
}

int escoin_norm_forward(const escoin_norm_desc* desc, const void* d_x, const void* d_y, const void* d_gate, const void* d_post_weight,
                        const void* d_post_bias, const void* d_pre_weight, const void* d_pre_bias, void* d_h, void* d_n, void* hip_stream) {
    NormArgs a;
    const int rc = make_norm_args(desc, &a);
    if (rc != ESCOIN_OK || a.T == 0) return rc;  // tensors without elements may have no address
    if ((!d_y && (a.post != ESCOIN_NORM_NONE || d_gate)) || (a.post == ESCOIN_NORM_NONE && (d_post_weight || d_post_bias)) ||
        (a.pre == ESCOIN_NORM_NONE && (d_pre_weight || d_pre_bias)) || (!d_h && !d_n) || (d_h && d_h == d_n))
        return ESCOIN_EINVAL;
    if (!d_x) return ESCOIN_EINVAL;
    // an output in the place of an input has to lie row upon row
    if ((d_h == d_x && a.ld_h != a.ld_x) || (d_y && d_h == d_y && a.ld_h != a.ld_y) || (d_n == d_x && a.ld_n != a.ld_x) || (d_y && d_n == d_y && a.ld_n != a.ld_y))
        return ESCOIN_EINVAL;
    const void* const all[] = {d_x, d_y, d_gate, d_post_weight, d_post_bias, d_pre_weight, d_pre_bias, d_h, d_n};
    uintptr_t bits = 0;
    for (const void* p : all) bits |= (uintptr_t)p;
    if (bits & (desc->type == ESCOIN_T_F32 ? 3 : 1)) return ESCOIN_EINVAL;
    a.x = d_x; a.y = d_y; a.gate = d_gate; a.post_weight = d_post_weight; a.post_bias = d_post_bias; a.pre_weight = d_pre_weight; a.pre_bias = d_pre_bias;
    a.h = d_h; a.n = d_n;
    const dim3 grid(std::min(a.T, 1 << 20)), block(kThreads);
    hipStream_t stream = (hipStream_t)hip_stream;
    if (desc->type == ESCOIN_T_F32) return launch(norm_kernel<ESCOIN_T_F32>, grid, block, 0, stream, a);
    if (desc->type == ESCOIN_T_F16) return launch(norm_kernel<ESCOIN_T_F16>, grid, block, 0, stream, a);
    return launch(norm_kernel<ESCOIN_T_BF16>, grid, block, 0, stream, a);
}

}  // extern "C"
