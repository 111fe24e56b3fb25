// Pruned linear layers on the host: checks, the plan, and which kernel a call takes.
#include <limits.h>
#include <string.h>

#include <atomic>
#include <memory>
#include <new>
#include <thread>

#include "linear.h"

namespace escoin {

namespace {

bool pitch(int64_t given, int64_t row, int64_t* out) {
    *out = given == 0 ? row : given;
    return *out >= row;
}

uint64_t up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// fp32 -> bf16 / fp16 bits, to nearest even.  NaNs stay NaNs.
inline uint16_t bf16_bits(float f) {
    uint32_t u;
    memcpy(&u, &f, 4);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)(u >> 16 | 0x40);
    return (uint16_t)((u + 0x7fff + (u >> 16 & 1)) >> 16);
}
inline uint16_t fp16_bits(float f) {
    uint32_t u;
    memcpy(&u, &f, 4);
    const uint32_t sign = u >> 16 & 0x8000u, a = u & 0x7fffffffu;
    if (a > 0x7f800000u) return (uint16_t)(sign | 0x7e00u);
    if (a >= 0x477ff000u) return (uint16_t)(sign | 0x7c00u);  // 65520 and more: infinite
    if (a >= 0x38800000u) return (uint16_t)(sign | ((a - 0x38000000u + 0xfff + (a >> 13 & 1)) >> 13));
    if (a <= 0x33000000u) return (uint16_t)sign;  // 2^-25 and less: zero
    // subnormal: a multiple of 2^-24, from 24 bits of significand shifted by 14 to 24 places
    const uint32_t m = (a & 0x7fffffu) | 0x800000u, shift = 126 - (a >> 23), half = 1u << (shift - 1), q = m >> shift, rest = m & (2 * half - 1);
    return (uint16_t)(sign | (q + (rest > half || (rest == half && (q & 1)) ? 1 : 0)));
}

// Up to how many tokens the kept weights are read.  Every workgroup unfolds them for itself, for 64 tokens at a time (fp32: 32): microseconds
// a tile and compute unit, and two more to begin with than the tiled kernel where it is more than 32; inputs whose rows cannot all start on 16 bytes
// cost more.  The tiled kernel's time is its steps (linear_many.hip), but no less than the whole weights take from memory; it
// needs rows enough to be spread over the compute units.  All of it at 50 %: layers with fewer nonzeros, whose kept weights cost less, go by
// the same numbers, and so by the tiled kernel somewhat early.  Measured with 64 tokens, kept against whole: 12288 to 4096 34
// and 33 us, 12288 to 2048 21 and 32, 2560 to 2560 10.7 and 9.4, 4096 to 24576 73 and 34, at 32 tokens 37.7 and 32.1 (41 from memory).
int few_tokens(const LinearDims& d) {
    const bool f32 = d.type == ESCOIN_T_F32;
    const double tiles = (double)d.row_tiles() * d.col_tiles() / 256, steps = d.col_frags() / kStepFrags;
    const double memory = (double)d.row_frags() * d.col_frags() * kFragBytes / 4.9e6, narrow = (int64_t)d.K * d.size() % 16 ? 1.3 : 1.0;
    int most = 16;
    for (int T = 32; T <= 256; T += 32) {
        const double kept = f32 ? 0.61 * (T / 32) : T <= 32 ? 0.18 : 0.30 * ((T + 63) / 64);
        const double rounds = (double)((((d.rows() + 63) / 64) * (int64_t)(T / 32) + 255) / 256);
        if (kept * narrow * tiles + (T > 32 ? 2.0 : 1.0) <= std::max(memory, (f32 ? 0.24 : 0.135) * steps * rounds)) most = T;
    }
    return most;
}

int check_csr(const LinearDims& d, const int32_t* rowptr, const int32_t* colidx) {
    if (!rowptr || rowptr[0] != 0) return ESCOIN_EINVAL;
    const int rows = d.rows();
    for (int m = 0; m < rows; ++m)
        if (rowptr[m + 1] < rowptr[m]) return ESCOIN_EINVAL;
    const int32_t nnz = rowptr[rows];
    if (nnz > 0 && !colidx) return ESCOIN_EINVAL;
    for (int32_t j = 0; j < nnz; ++j)
        if ((uint32_t)colidx[j] >= (uint32_t)d.K) return ESCOIN_EINVAL;
    return ESCOIN_OK;
}

// Where the sections lie, for a layer of so many nonzeros.
LinearHeader layout(const LinearDims& d, int32_t nnz) {
    LinearHeader h;
    memset(&h, 0, sizeof(h));
    h.magic = kLinearMagic;
    h.version = kLinearVersion;
    h.K = d.K; h.M = d.M; h.type = d.type; h.gated = d.gated;
    h.most_tokens = d.T;
    h.few_tokens = few_tokens(d);
    const uint64_t tiles = (uint64_t)d.row_tiles() * d.col_tiles();
    h.off_zero = up(sizeof(h), 256);
    h.off_mask = h.off_zero + 256;
    h.off_start = h.off_mask + tiles * 256;
    h.off_kept = up(h.off_start + (tiles + 1) * 4, 256);
    h.off_whole = up(h.off_kept + (uint64_t)nnz * d.size() + tiles * 15 + 16, 256);  // 16: a lane reads over its tile's end
    h.total_bytes = h.off_whole;
    if (d.T > h.few_tokens) h.total_bytes += (uint64_t)d.row_frags() * d.col_frags() * kFragBytes;
    return h;
}

template <typename V>
V rounded(float f, int type);
template <>
inline float rounded<float>(float f, int) { return f; }
template <>
inline uint16_t rounded<uint16_t>(float f, int type) { return type == ESCOIN_T_BF16 ? bf16_bits(f) : fp16_bits(f); }
inline bool is_zero(float v) { return v == 0.0f; }
inline bool is_zero(uint16_t v) { return (v & 0x7fff) == 0; }

// Blocks of 32 rows that are filled one after the other; such runs of blocks are filled side by side.  A run's values start where they
// would if every one before it took its 15 bytes of padding a tile, so that a plan does not depend on how many threads fill it.
constexpr int kRunFrags = 64;
constexpr int kMostThreads = 8;

uint64_t run_start(const LinearDims& d, const int32_t* rowptr, int frag) {
    const int rows = std::min(frag * kFragRows, d.rows());
    const int64_t before = d.gated ? (int64_t)rowptr[rows / 2] + rowptr[d.M + rows / 2] - rowptr[d.M] : rowptr[rows];
    const int tiles = std::min(frag * (kFragRows / kTileRows), d.row_tiles());
    return ((uint64_t)before * d.size() + (uint64_t)tiles * d.col_tiles() * 15) / 16 * 16;
}

// From the first of a run's blocks on; which are laid out with their zeros first.  Returns the words of the fullest lane, or -1 without memory.
template <typename V>
int fill(const LinearDims& d, const int32_t* rowptr, const int32_t* colidx, const float* value, const LinearHeader& h, char* plan, int from_frag) {
    const int cols = std::max(d.col_tiles() * kTileCols, d.col_frags() * 32 / (int)sizeof(V));
    std::unique_ptr<float[]> sums(new (std::nothrow) float[cols]);
    std::unique_ptr<V[]> dense(new (std::nothrow) V[(size_t)kFragRows * cols]);
    if (!sums || !dense) return -1;
    std::fill_n(sums.get(), cols, 0.0f);
    uint32_t* const mask = (uint32_t*)(plan + h.off_mask);
    uint32_t* const start = (uint32_t*)(plan + h.off_start);
    char* const kept = plan + h.off_kept;
    const bool whole = d.T > h.few_tokens;
    const int to_frag = std::min(from_frag + kRunFrags, d.row_frags());
    uint64_t at = run_start(d, rowptr, from_frag);
    const uint64_t stop = to_frag == d.row_frags() ? h.off_whole - h.off_kept : run_start(d, rowptr, to_frag);
    int most = 0;
    for (int rf = from_frag; rf < to_frag; ++rf) {
        std::fill_n(dense.get(), (size_t)kFragRows * cols, V{});
        for (int i = 0; i < kFragRows; ++i) {
            const int r = rf * kFragRows + i;
            if (r >= d.rows()) break;
            const int m = d.gated ? (r >> 1) + (r & 1) * d.M : r;
            const int32_t begin = rowptr[m], end = rowptr[m + 1];
            V* const row = dense.get() + (size_t)i * cols;
            bool ascending = true;
            for (int32_t j = begin + 1; j < end; ++j) ascending &= colidx[j] > colidx[j - 1];
            if (ascending) {
                for (int32_t j = begin; j < end; ++j) row[colidx[j]] = rounded<V>(value[j], d.type);
            } else {
                // repeated columns are added up before the sum is rounded
                for (int32_t j = begin; j < end; ++j) sums[colidx[j]] += value[j];
                for (int32_t j = begin; j < end; ++j) row[colidx[j]] = rounded<V>(sums[colidx[j]], d.type);
                for (int32_t j = begin; j < end; ++j) sums[colidx[j]] = 0.0f;
            }
        }
        for (int half = 0; half < kFragRows / kTileRows; ++half) {
            const int rt = rf * (kFragRows / kTileRows) + half;
            if (rt >= d.row_tiles()) break;
            for (int ct = 0; ct < d.col_tiles(); ++ct) {
                const size_t tile = (size_t)rt * d.col_tiles() + ct;
                start[tile] = (uint32_t)(at / 16);
                for (int lane = 0; lane < 64; ++lane) {
                    const V* const from = dense.get() + (size_t)(half * kTileRows + lane % 16) * cols + ct * kTileCols + lane / 16 * 8;
                    uint32_t bits = 0;
                    V found[33];
                    int n = 0;
                    for (int b = 0; b < 4; ++b)
                        for (int j = 0; j < 8; ++j) {
                            const V v = from[b * 32 + j];
                            const uint32_t there = !is_zero(v);  // no branch: every other one would be guessed wrong
                            found[n] = v;
                            n += there;
                            bits |= there << (b * 8 + j);
                        }
                    memcpy(kept + at, found, n * sizeof(V));
                    most = std::max(most, (int)((at % 4 + n * sizeof(V) + 3) / 4));
                    at += n * sizeof(V);
                    mask[tile * 64 + lane] = bits;
                }
                while (at % 16) kept[at++] = 0;
            }
        }
        if (!whole) continue;
        char* to = plan + h.off_whole + (size_t)rf * d.col_frags() * kFragBytes;
        constexpr int kHalf = 16 / sizeof(V);  // columns of a lane
        for (int cf = 0; cf < d.col_frags(); ++cf)
            for (int lane = 0; lane < 64; ++lane, to += 16)
                memcpy(to, dense.get() + (size_t)(lane % 32) * cols + (cf * 2 + lane / 32) * kHalf, 16);
    }
    memset(kept + at, 0, (size_t)(stop - at));
    if (to_frag == d.row_frags()) start[(size_t)d.row_tiles() * d.col_tiles()] = (uint32_t)(at / 16);
    return most;
}

// All runs, by as many threads as there are runs (and as the machine gives: at least this one).
template <typename V>
int fill_all(const LinearDims& d, const int32_t* rowptr, const int32_t* colidx, const float* value, LinearHeader* h, char* plan) {
    const int runs = (d.row_frags() + kRunFrags - 1) / kRunFrags;
    std::atomic<int> next{0}, most{0};
    const auto work = [&]() {
        for (int r; (r = next.fetch_add(1)) < runs;) {
            const int words = fill<V>(d, rowptr, colidx, value, *h, plan, r * kRunFrags);
            int seen = most.load();
            while (seen >= 0 && (words < 0 || words > seen) && !most.compare_exchange_weak(seen, words)) {}
        }
    };
    std::thread others[kMostThreads - 1];
    int started = 0;
    const int wanted = std::min(std::min(runs, kMostThreads), (int)std::max(1u, std::thread::hardware_concurrency())) - 1;
    try {
        for (; started < wanted; ++started) others[started] = std::thread(work);
    } catch (...) {
    }
    work();
    for (int i = 0; i < started; ++i) others[i].join();
    h->most_lane_words = most.load();
    return most.load() < 0 ? ESCOIN_ESIZE : ESCOIN_OK;
}

}  // namespace

int make_linear_dims(const escoin_linear_desc* desc, LinearDims* d) {
    if (!desc) return ESCOIN_EINVAL;
    const escoin_linear_desc& p = *desc;
    if (p.T < 0 || p.K < 1 || p.M < 1 || p.type < ESCOIN_T_F32 || p.type > ESCOIN_T_BF16 || (p.gated & ~1)) return ESCOIN_EINVAL;
    if (!pitch(p.ld_in, p.K, &d->ld_in) || !pitch(p.ld_out, p.M, &d->ld_out) || !pitch(p.ld_residual, p.M, &d->ld_residual)) return ESCOIN_EINVAL;
    if (p.K >= 1 << 22 || p.M >= 1 << 29) return ESCOIN_ERANGE;
    if (d->ld_in >= 1ll << 40 || d->ld_out >= 1ll << 40 || d->ld_residual >= 1ll << 40) return ESCOIN_ERANGE;
    d->T = p.T; d->K = p.K; d->M = p.M; d->type = p.type; d->gated = p.gated != 0;
    // tiles are counted in 32 bits, and so are the bytes of 256 rows of whole weights: K stays below 2^22
    if ((double)d->row_tiles() * d->col_tiles() >= 0x1p31) return ESCOIN_ERANGE;
    return ESCOIN_OK;
}

// What a call's kernel goes by: sizes, pitches in bytes and where the input lies.
static LinearArgs linear_sizes(const LinearDims& d, const void* d_in) {
    LinearArgs a = {};
    const int size = d.size();
    a.in = (const char*)d_in;
    a.T = d.T; a.K = d.K; a.M = d.M; a.rows = d.rows();
    a.row_tiles = d.row_tiles(); a.col_tiles = d.col_tiles(); a.row_frags = d.row_frags(); a.col_frags = d.col_frags();
    a.ld_in = d.ld_in * size; a.ld_out = d.ld_out * size; a.ld_residual = d.ld_residual * size;
    return a;
}

static int linear_launch(const LinearDims& d, const LinearHeader& h, const LinearArgs& a, const LinearCall& call) {
    return d.T <= h.few_tokens ? launch_linear_few(d, h, a, call) : launch_linear_many(d, h, a, call);
}

int linear_header(const LinearDims& d, const void* plan, LinearHeader* h) {
    if (!plan) return ESCOIN_EINVAL;
    memcpy(h, plan, sizeof(*h));
    if (h->magic != kLinearMagic || h->version != kLinearVersion || h->K != d.K || h->M != d.M || h->type != d.type || h->gated != (int)d.gated ||
        d.T > h->most_tokens)
        return ESCOIN_EINVAL;
    return ESCOIN_OK;
}

}  // namespace escoin

using namespace escoin;

extern "C" {

int escoin_linear_check_desc(const escoin_linear_desc* desc) {
    LinearDims d;
    return make_linear_dims(desc, &d);
}

int escoin_linear_plan_size(const escoin_linear_desc* desc, const int32_t* rowptr, const int32_t* colidx, size_t* plan_bytes) {
    LinearDims d;
    int rc = make_linear_dims(desc, &d);
    if (rc != ESCOIN_OK) return rc;
    if (!plan_bytes) return ESCOIN_EINVAL;
    rc = check_csr(d, rowptr, colidx);
    if (rc == ESCOIN_OK) *plan_bytes = layout(d, rowptr[d.rows()]).total_bytes;
    return rc;
}

int escoin_linear_plan_build(const escoin_linear_desc* desc, const int32_t* rowptr, const int32_t* colidx, const float* value, void* plan,
                             size_t plan_bytes) {
    LinearDims d;
    int rc = make_linear_dims(desc, &d);
    if (rc != ESCOIN_OK) return rc;
    if (!plan) return ESCOIN_EINVAL;
    rc = check_csr(d, rowptr, colidx);
    if (rc != ESCOIN_OK) return rc;
    if (rowptr[d.rows()] > 0 && !value) return ESCOIN_EINVAL;
    LinearHeader h = layout(d, rowptr[d.rows()]);
    if (plan_bytes < h.total_bytes) return ESCOIN_ESIZE;
    memset(plan, 0, (size_t)h.off_mask);
    memset((char*)plan + h.off_kept - 256, 0, 256);  // what lies between the tables and the values; the table's end is written below
    rc = d.type == ESCOIN_T_F32 ? fill_all<float>(d, rowptr, colidx, value, &h, (char*)plan) : fill_all<uint16_t>(d, rowptr, colidx, value, &h, (char*)plan);
    if (rc == ESCOIN_OK) memcpy(plan, &h, sizeof(h));
    return rc;
}

int escoin_linear_few_tokens(const escoin_linear_desc* desc, const void* plan_host) {
    LinearDims d;
    LinearHeader h;
    int rc = make_linear_dims(desc, &d);
    if (rc == ESCOIN_OK) rc = linear_header(d, plan_host, &h);
    return rc != ESCOIN_OK ? rc : h.few_tokens;
}

int escoin_linear_forward(const escoin_linear_desc* desc, const void* plan_host, const void* d_plan, const void* d_in, void* d_out,
                          const void* d_bias, const void* d_residual, uint32_t flags, void* hip_stream) {
    LinearDims d;
    LinearHeader h;
    int rc = make_linear_dims(desc, &d);
    if (rc == ESCOIN_OK) rc = linear_header(d, plan_host, &h);
    if (rc != ESCOIN_OK) return rc;
    constexpr uint32_t kActs = ESCOIN_F_RELU | ESCOIN_F_SILU | ESCOIN_F_GELU | ESCOIN_F_GELU_TANH;
    if ((flags & ~(kActs | ESCOIN_F_BIAS | ESCOIN_F_RESIDUAL)) || ((flags & kActs) & ((flags & kActs) - 1))) return ESCOIN_EINVAL;
    if (d.T == 0) return ESCOIN_OK;  // tensors without elements may have no address
    if (((flags & ESCOIN_F_BIAS) && !d_bias) || ((flags & ESCOIN_F_RESIDUAL) && !d_residual)) return ESCOIN_EINVAL;
    if (!d_plan || !d_in || !d_out || d_in == d_out) return ESCOIN_EINVAL;
    if ((flags & ESCOIN_F_RESIDUAL) && d_residual == d_out && d.ld_residual != d.ld_out) return ESCOIN_EINVAL;
    const int size = d.size();
    if (((uintptr_t)d_plan & 15) || (((uintptr_t)d_in | (uintptr_t)d_out) & (size - 1)) || ((flags & ESCOIN_F_BIAS) && ((uintptr_t)d_bias & (size - 1))) ||
        ((flags & ESCOIN_F_RESIDUAL) && ((uintptr_t)d_residual & (size - 1))))
        return ESCOIN_EINVAL;
    LinearArgs a = linear_sizes(d, d_in);
    const char* const p = (const char*)d_plan;
    a.out = (char*)d_out;
    a.bias = flags & ESCOIN_F_BIAS ? (const char*)d_bias : nullptr;
    a.residual = flags & ESCOIN_F_RESIDUAL ? (const char*)d_residual : nullptr;
    a.zero = p + h.off_zero;
    a.mask = (const uint32_t*)(p + h.off_mask);
    a.start = (const uint32_t*)(p + h.off_start);
    a.kept = p + h.off_kept;
    a.whole = p + h.off_whole;
    a.flags = flags;
    return linear_launch(d, h, a, {(hipStream_t)hip_stream, nullptr});
}

int escoin_linear_kernel(const escoin_linear_desc* desc, const void* plan_host, const void* d_in, escoin_linear_kernel_info* info) {
    LinearDims d;
    LinearHeader h;
    int rc = make_linear_dims(desc, &d);
    if (rc == ESCOIN_OK) rc = linear_header(d, plan_host, &h);
    if (rc != ESCOIN_OK) return rc;
    if (!info || ((uintptr_t)d_in & (d.size() - 1))) return ESCOIN_EINVAL;
    *info = {};
    return d.T == 0 ? ESCOIN_OK : linear_launch(d, h, linear_sizes(d, d_in), {nullptr, info});
}

}  // extern "C"
