// The residual stream between two blocks: h = alpha x + beta gate post(y), n = pre(h), in one pass.  Some twenty instructions an
// element, which memory hides: 8192 rows of 4096 in bf16, x and y read, h and n written, take 71 us (3.76 TB/s of a copy's 4.9; vector
// instructions 69 % of it), 1023 of 5003 in fp32 27.
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

// The sum over a row's WAVES waves (a whole workgroup where there are several), the same for each of its threads.
template <int WAVES>
__device__ inline float all_sum(float v, float* lds) {
#define ESCOIN_SUM(CTRL, ROWS) v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
    ESCOIN_SUM(0x111, 0xf)  // row_shr 1, 2, 4, 8, then over the rows of 16: the last lane has the sum
    ESCOIN_SUM(0x112, 0xf)
    ESCOIN_SUM(0x114, 0xf)
    ESCOIN_SUM(0x118, 0xf)
    ESCOIN_SUM(0x142, 0xa)
    ESCOIN_SUM(0x143, 0xc)
#undef ESCOIN_SUM
    v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    if constexpr (WAVES > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += lds[w];
    }
    return v;
}

struct Stats {
    float mean, scale;
};

// 16 bytes of a row as they lie in memory, at any element.
template <class N>
struct Piece {
    static constexpr int kN = 16 / sizeof(N);
    struct __attribute__((packed, aligned(sizeof(N)))) Raw {
        N v[kN];
    } raw;
    // the elements from `at` on, of which `there` are in the row
    __device__ void load(const void* row, int at, int there) {
        const N* const p = (const N*)row + at;
        if (there >= kN) raw = *(const Raw*)p;
        else
#pragma unroll
            for (int j = 0; j < kN; ++j) raw.v[j] = j < there ? p[j] : (N)0.0f;
    }
    __device__ void store(void* row, int at, int there) const {
        N* const p = (N*)row + at;
        if (there >= kN) *(Raw*)p = raw;
        else
#pragma unroll
            for (int j = 0; j < kN; ++j)
                if (j < there) p[j] = raw.v[j];
    }
};

// A row stays in the registers of its WAVES waves, F elements a thread, in pieces of 16 bytes that follow each other over the threads.
template <int TYPE, int WAVES, int F>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void norm_kernel(const NormArgs a) {
    typedef typename Num<TYPE>::type N;
    typedef Piece<N> P;
    constexpr int kN = P::kN, kPieces = F / kN;
    __shared__ float lds[WAVES];
    const int t = WAVES == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x, lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    if (WAVES == 1 && t >= a.T) return;
    const auto at = [&](int i) { return (i * 64 * WAVES + lane) * kN; };
    const auto there = [&](int i) { return a.D - at(i); };
    const N* const x_row = (const N*)a.x + t * a.ld_x;
    const N* const y_row = (const N*)a.y + t * a.ld_y;
    const N* const gate_row = (const N*)a.gate + (a.gate_rows ? t * a.ld_gate : 0);
    P x[kPieces], y[kPieces];
    float v[F];
    if (a.y)
#pragma unroll
        for (int i = 0; i < kPieces; ++i) y[i].load(y_row, at(i), there(i));
#pragma unroll
    for (int i = 0; i < kPieces; ++i) x[i].load(x_row, at(i), there(i));
    const float count = (float)a.D;
    // of v: two passes for a layer norm, the squares of the deviations and not a difference of sums
    const auto stats = [&](int kind) {
        Stats s = {0.0f, 1.0f};
        if (kind == ESCOIN_NORM_NONE) return s;
        if (kind == ESCOIN_NORM_LAYER) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < F; ++i) sum += v[i];
            s.mean = all_sum<WAVES>(sum, lds) / count;
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const float u = i % kN < there(i / kN) ? v[i] - s.mean : 0.0f;
            sum = fmaf(u, u, sum);
        }
        s.scale = 1.0f / sqrtf(all_sum<WAVES>(sum, lds) / count + a.eps);
        return s;
    };
    const auto norm = [&](int kind, const Stats& s, const void* weight, const void* bias) {
        if (kind == ESCOIN_NORM_NONE) return;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            P w, b;
            if (weight) w.load(weight, at(i), there(i));
            if (bias) b.load(bias, at(i), there(i));
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                float u = (v[i * kN + j] - s.mean) * s.scale;
                if (weight) u *= (float)w.raw.v[j] + a.offset;
                if (bias) u += (float)b.raw.v[j];
                v[i * kN + j] = u;
            }
        }
    };
    const auto put = [&](void* row) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            P o;
#pragma unroll
            for (int j = 0; j < kN; ++j) o.raw.v[j] = (N)v[i * kN + j];
            o.store(row, at(i), there(i));
        }
    };
    if (a.y) {
#pragma unroll
        for (int i = 0; i < F; ++i) v[i] = (float)y[i / kN].raw.v[i % kN];
        norm(a.post, stats(a.post), a.post_weight, a.post_bias);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            P g;
            if (a.gate) g.load(gate_row, at(i), there(i));
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                float u = a.beta * v[i * kN + j];
                if (a.gate) u *= (float)g.raw.v[j];
                v[i * kN + j] = j < there(i) ? a.alpha * (float)x[i].raw.v[j] + u : 0.0f;  // a bias or gate beyond the row does not count
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < F; ++i) v[i] = a.alpha * (float)x[i / kN].raw.v[i % kN];
    }
    if (a.h) put((N*)a.h + t * a.ld_h);
    if (!a.n) return;
    norm(a.pre, stats(a.pre), a.pre_weight, a.pre_bias);
    put((N*)a.n + t * a.ld_n);
}

// Rows too long for that: read from memory again for every pass.
constexpr int kLongWaves = 16;

template <int TYPE>
__global__ __launch_bounds__(64 * kLongWaves) void norm_long_kernel(const NormArgs a) {
    typedef typename Num<TYPE>::type N;
    __shared__ float lds[kLongWaves];
    const int t = blockIdx.x;
    const N* const x = (const N*)a.x + t * a.ld_x;
    const N* const y = (const N*)a.y + t * a.ld_y;
    const N* const gate = (const N*)a.gate + (a.gate_rows ? t * a.ld_gate : 0);
    const auto stats = [&](int kind, auto f) {
        Stats s = {0.0f, 1.0f};
        if (kind == ESCOIN_NORM_NONE) return s;
        float v = 0.0f;
        if (kind == ESCOIN_NORM_LAYER) {
            for (int i = threadIdx.x; i < a.D; i += 64 * kLongWaves) v += f(i);
            s.mean = all_sum<kLongWaves>(v, lds) / (float)a.D;
        }
        v = 0.0f;
        for (int i = threadIdx.x; i < a.D; i += 64 * kLongWaves) {
            const float u = f(i) - s.mean;
            v = fmaf(u, u, v);
        }
        s.scale = 1.0f / sqrtf(all_sum<kLongWaves>(v, lds) / (float)a.D + a.eps);
        return s;
    };
    const auto normed = [&](float v, int kind, const Stats& s, const void* weight, const void* bias, int i) {
        if (kind == ESCOIN_NORM_NONE) return v;
        v = (v - s.mean) * s.scale;
        if (weight) v *= (float)((const N*)weight)[i] + a.offset;
        if (bias) v += (float)((const N*)bias)[i];
        return v;
    };
    const Stats post = stats(a.y ? a.post : ESCOIN_NORM_NONE, [&](int i) { return (float)y[i]; });
    const auto sum = [&](int i) {
        float v = a.alpha * (float)x[i];
        if (a.y) {
            float b = a.beta * normed((float)y[i], a.post, post, a.post_weight, a.post_bias, i);
            if (a.gate) b *= (float)gate[i];
            v += b;
        }
        return v;
    };
    const Stats pre = stats(a.n ? a.pre : ESCOIN_NORM_NONE, sum);
    for (int i = threadIdx.x; i < a.D; i += 64 * kLongWaves) {
        const float v = sum(i);  // both are read before either is written: an output may take an input's place
        if (a.h) ((N*)a.h)[t * a.ld_h + i] = (N)v;
        if (a.n) ((N*)a.n)[t * a.ld_n + i] = (N)normed(v, a.pre, pre, a.pre_weight, a.pre_bias, i);
    }
}

template <int TYPE>
int launch_norm(const NormArgs& a, hipStream_t stream) {
    const int D = a.D;
    const auto go = [&](auto kernel, int waves) {
        const int64_t blocks = waves == 1 ? ((int64_t)a.T + 3) / 4 : a.T;
        const int threads = waves == 1 ? 256 : 64 * waves;
        if (!grid_fits((double)blocks, threads)) return (int)ESCOIN_ERANGE;
        return launch(kernel, dim3((unsigned)blocks), dim3(threads), 0, stream, a);
    };
    // Eight elements a thread: a single row is done soonest.  Sixteen, and fewer waves to a row, where there are rows enough: one wave and no
    // meeting (1000 bf16, 8192 rows: 20.5 us, by four waves 26.8; 1024 rows 7.2 and 6.6), four in place of sixteen (4096 bf16, 8192 rows:
    // 71.9 and 100.6 us, at 3.7 TB/s; 512 rows 8.0 and 8.9; one row 5.6 and 4.9).  Two in place of four and eight in place of sixteen: the same.
    if (D <= 512) return go(norm_kernel<TYPE, 1, 8>, 1);
    if (D <= 1024 && a.T >= 2048) return go(norm_kernel<TYPE, 1, 16>, 1);
    if (D <= 2048) return go(norm_kernel<TYPE, 4, 8>, 4);
    if (D <= 4096 && a.T >= 512) return go(norm_kernel<TYPE, 4, 16>, 4);
    if (D <= 8192) return go(norm_kernel<TYPE, 16, 8>, 16);
    if (D <= 16384) return go(norm_kernel<TYPE, 16, 16>, 16);
    if (D <= 32768) return go(norm_kernel<TYPE, 16, 32>, 16);
    return go(norm_long_kernel<TYPE>, kLongWaves);
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
    hipStream_t stream = (hipStream_t)hip_stream;
    if (desc->type == ESCOIN_T_F32) return launch_norm<ESCOIN_T_F32>(a, stream);
    if (desc->type == ESCOIN_T_F16) return launch_norm<ESCOIN_T_F16>(a, stream);
    return launch_norm<ESCOIN_T_BF16>(a, stream);
}

}  // extern "C"
