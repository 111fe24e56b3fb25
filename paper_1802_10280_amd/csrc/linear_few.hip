// Pruned linear layers for few tokens: the kept weights, read once.
#include "linear_device.h"
#include "mfma.h"

namespace escoin {
namespace {

constexpr int kMostWaves = 16;

// LDS of a wave: a tile's values; a lane reads up to 12 bytes from where its own end
constexpr int few_buffer(int chunks) { return chunks * 1024 + 16; }

// Exclusive sums over the lanes of a wave.
__device__ inline int lanes_before(int n) {
    int s = n;
#define ESCOIN_SCAN(CTRL, ROWS) s += __builtin_amdgcn_update_dpp(0, s, CTRL, ROWS, 0xf, false);
    ESCOIN_SCAN(0x111, 0xf)  // row_shr 1, 2, 4, 8, then over the rows of 16
    ESCOIN_SCAN(0x112, 0xf)
    ESCOIN_SCAN(0x114, 0xf)
    ESCOIN_SCAN(0x118, 0xf)
    ESCOIN_SCAN(0x142, 0xa)
    ESCOIN_SCAN(0x143, 0xc)
#undef ESCOIN_SCAN
    return s - n;
}

// A tile on its way: its mask, the 16 bytes a lane carries of every 1024 of its values, and (AHEAD) its inputs.
template <int CHUNKS, int PIECES>
struct Load {
    u4 v[CHUNKS], x[PIECES];
    uint32_t mask;
};

// The eight weights of block b, zeros in their places, for a lane whose values start `at` bytes into LDS.
template <int TYPE>
__device__ inline void expand(const char* values, const u2* picks, uint32_t mask, int at, int b, u4 (&w)[TYPE == ESCOIN_T_F32 ? 2 : 1]) {
    at += __popc(mask & ((1u << (8 * b)) - 1)) * (TYPE == ESCOIN_T_F32 ? 4 : 2);
    if constexpr (TYPE == ESCOIN_T_F32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)mask, 8 * b + j, 1);
            w[j / 4][j % 4] = *(const uint32_t*)(values + at) & keep;
            at += 4 & keep;
        }
    } else {
        // four weights are bytes picked from the next eight: which ones depends on their four bits
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const uint32_t nibble = mask >> (8 * b + 4 * n) & 15;
            const u2 pick = picks[nibble];
            // (from whole words: reads at odd halves take LDS a clock a lane)
            const uint32_t* const near = (const uint32_t*)(values + (at & ~3));
            const uint32_t lo = __builtin_amdgcn_alignbyte(near[1], near[0], at), hi = __builtin_amdgcn_alignbyte(near[2], near[1], at);
            w[0][2 * n] = __builtin_amdgcn_perm(hi, lo, pick[0]);
            w[0][2 * n + 1] = __builtin_amdgcn_perm(hi, lo, pick[1]);
            at += 2 * __popc(nibble);
        }
    }
}

// A workgroup has 16 rows and NT * 16 tokens; its waves take the tiles along the columns in turn, and their sums meet in LDS.
template <int TYPE, bool GATED, bool WIDE, int NT, int CHUNKS>
__global__ __launch_bounds__(64 * kMostWaves) void linear_few_kernel(const LinearArgs a) {
    extern __shared__ char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    constexpr int kSize = sizeof(typename Num<TYPE>::type), kParts = kSize == 4 ? 2 : 1, kPieces = 4 * NT * kParts;
    // a tile's inputs are asked for with its weights, a tile ahead, where there are registers for two tiles' inputs
    constexpr bool kAhead = kPieces <= 8;
    constexpr int kBuffer = few_buffer(CHUNKS);
    const int rt = blockIdx.x, token0 = blockIdx.y * NT * 16;
    u2* const picks = (u2*)lds;
    char* const values = lds + 128 + wave * kBuffer;
    if (threadIdx.x < 16) {
        uint32_t p[4], pos = 0;
        for (int j = 0; j < 4; ++j) {
            p[j] = threadIdx.x >> j & 1 ? (2 * pos + 1) << 8 | 2 * pos : 0x0c0cu;  // 0x0c picks a byte of zeros
            pos += threadIdx.x >> j & 1;
        }
        picks[threadIdx.x] = u2{p[0] | p[1] << 16, p[2] | p[3] << 16};
    }
    const int end = a.K * kSize;
    const char* row[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) row[t] = a.in + min(token0 + t * 16 + lane % 16, a.T - 1) * a.ld_in;
    const auto inputs = [&](int ct, u4* x) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int p = 0; p < kParts; ++p)
                    x[(b * NT + t) * kParts + p] = input16<TYPE, WIDE>(a, row[t], (ct * kTileCols + b * 32 + lane / 16 * 8) * kSize + p * 16, end);
    };
    const int64_t first = (int64_t)rt * a.col_tiles;
    Load<CHUNKS, kAhead ? kPieces : 1> next;
    const auto ask = [&](int ct, uint32_t begin, uint32_t stop) {
        const int bytes = (int)(stop - begin) * 16;
        const char* const from = a.kept + (uint64_t)begin * 16;
        next.mask = a.mask[(first + ct) * 64 + lane];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = c * 1024 + lane * 16;
            next.v[c] = *(const u4*)(at < bytes ? from + at : a.zero);
        }
        if constexpr (kAhead) inputs(ct, next.x);
    };
    // where a tile's values lie is known one tile before they are asked for
    uint32_t begin = 0, stop = 0;
    const auto look = [&](int ct) {
        if (ct < a.col_tiles) begin = a.start[first + ct], stop = a.start[first + ct + 1];
    };
    look(wave);
    if (wave < a.col_tiles) ask(wave, begin, stop);
    look(wave + waves);
    __syncthreads();
    f4 sum[NT] = {};
    for (int ct = wave; ct < a.col_tiles; ct += waves) {
        const uint32_t mask = next.mask;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) *(u4*)(values + c * 1024 + lane * 16) = next.v[c];
        // the wave's lanes read what others of them have written: in order, as all LDS accesses of a wave are
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        u4 x[kPieces];
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) x[i] = next.x[i];
        } else {
            inputs(ct, x);  // before the next weights: loads come back in order
        }
        __builtin_amdgcn_sched_barrier(0);
        if (ct + waves < a.col_tiles) ask(ct + waves, begin, stop);
        look(ct + 2 * waves);
        __builtin_amdgcn_sched_barrier(0);
        const int at = lanes_before(__popc(mask)) * kSize;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            u4 w[kParts];
            expand<TYPE>(values, picks, mask, at, b, w);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int p = 0; p < kParts; ++p) sum[t] = mfma16<TYPE>(w[p], x[(b * NT + t) * kParts + p], sum[t]);
        }
    }
    __syncthreads();
    f4* const parts = (f4*)(lds + 128);
#pragma unroll
    for (int t = 0; t < NT; ++t) parts[(t * waves + wave) * 64 + lane] = sum[t];
    __syncthreads();
    for (int t = wave; t < NT; t += waves) {
        f4 z = parts[t * waves * 64 + lane];
        for (int k = 1; k < waves; ++k) z += parts[(t * waves + k) * 64 + lane];
        finish<TYPE, GATED>(a, z, rt * 16 + lane / 16 * 4, token0 + t * 16 + lane % 16);
    }
}

template <int TYPE, bool GATED, bool WIDE, int NT, int CHUNKS>
int launch_one(const LinearArgs& a, int waves, hipStream_t stream) {
    const int lds = 128 + waves * std::max(few_buffer(CHUNKS), NT * 1024);
    const dim3 grid((unsigned)a.row_tiles, (unsigned)((a.T + NT * 16 - 1) / (NT * 16))), block(64 * waves);
    if (!grid_fits((double)grid.x * grid.y, 64 * waves)) return ESCOIN_ERANGE;
    const auto kernel = linear_few_kernel<TYPE, GATED, WIDE, NT, CHUNKS>;
    const int rc = lds > 64 * 1024 ? allow_dynamic_lds((const void*)kernel, lds) : ESCOIN_OK;
    return rc != ESCOIN_OK ? rc : launch(kernel, grid, block, (size_t)lds, stream, a);
}

template <int TYPE, bool GATED, bool WIDE, int NT>
int launch_chunks(const LinearHeader& h, const LinearArgs& a, int waves, hipStream_t stream) {
    const int chunks = (h.most_tile_bytes + 1023) / 1024;
    if constexpr (TYPE == ESCOIN_T_F32) {
        if (chunks > 5) return launch_one<TYPE, GATED, WIDE, NT, 8>(a, waves, stream);
        if (chunks > 4) return launch_one<TYPE, GATED, WIDE, NT, 5>(a, waves, stream);
    }
    if (chunks > 3) return launch_one<TYPE, GATED, WIDE, NT, 4>(a, waves, stream);
    if (chunks > 2) return launch_one<TYPE, GATED, WIDE, NT, 3>(a, waves, stream);
    if (chunks > 1) return launch_one<TYPE, GATED, WIDE, NT, 2>(a, waves, stream);
    return launch_one<TYPE, GATED, WIDE, NT, 1>(a, waves, stream);
}

template <int TYPE, bool GATED, bool WIDE>
int launch_tokens(const LinearHeader& h, const LinearArgs& a, hipStream_t stream) {
    const int token_blocks = (a.T + 63) / 64;
    int waves = kMostWaves;
    while (waves > 4 && (int64_t)a.row_tiles * token_blocks * waves > 256 * 24) waves /= 2;
    if (const char* e = getenv("WAVES")) waves = atoi(e);
    waves = std::min(waves, a.col_tiles);
    if (a.T <= 16) return launch_chunks<TYPE, GATED, WIDE, 1>(h, a, waves, stream);
    if (a.T <= 32) return launch_chunks<TYPE, GATED, WIDE, 2>(h, a, waves, stream);
    if constexpr (TYPE == ESCOIN_T_F32) return launch_chunks<TYPE, GATED, WIDE, 2>(h, a, waves, stream);  // registers for no more inputs
    else return launch_chunks<TYPE, GATED, WIDE, 4>(h, a, waves, stream);
}

template <int TYPE>
int launch_type(const LinearDims& d, const LinearHeader& h, const LinearArgs& a, hipStream_t stream) {
    const bool wide = wide_input(a, d.size());
    if (d.gated) return wide ? launch_tokens<TYPE, true, true>(h, a, stream) : launch_tokens<TYPE, true, false>(h, a, stream);
    return wide ? launch_tokens<TYPE, false, true>(h, a, stream) : launch_tokens<TYPE, false, false>(h, a, stream);
}

}  // namespace

int launch_linear_few(const LinearDims& d, const LinearHeader& h, const LinearArgs& a, hipStream_t stream) {
    if (d.type == ESCOIN_T_F32) return launch_type<ESCOIN_T_F32>(d, h, a, stream);
    if (d.type == ESCOIN_T_F16) return launch_type<ESCOIN_T_F16>(d, h, a, stream);
    return launch_type<ESCOIN_T_BF16>(d, h, a, stream);
}

}  // namespace escoin
