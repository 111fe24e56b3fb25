// Pruned linear layers for few tokens: the kept weights, read once.
#include "linear_device.h"
#include "mfma.h"

namespace escoin {
namespace {

constexpr int kMostWaves = 16;

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

// A tile on its way: its mask and the 16 bytes a lane carries of every 1024 of its values.
template <int CHUNKS>
struct Load {
    u4 v[CHUNKS];
    uint32_t mask;
};

template <int CHUNKS>
__device__ inline void ask(const LinearArgs& a, int64_t tile, int lane, Load<CHUNKS>& l) {
    const uint32_t begin = a.start[tile], end = a.start[tile + 1];
    const int bytes = (int)(end - begin) * 16;
    const char* const from = a.kept + (uint64_t)begin * 16;
    l.mask = a.mask[tile * 64 + lane];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = c * 1024 + lane * 16;
        l.v[c] = *(const u4*)(at < bytes ? from + at : a.zero);
    }
}

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
            struct __attribute__((packed, aligned(2))) Near {
                uint32_t lo, hi;
            };
            const Near near = *(const Near*)(values + at);
            w[0][2 * n] = __builtin_amdgcn_perm(near.hi, near.lo, pick[0]);
            w[0][2 * n + 1] = __builtin_amdgcn_perm(near.hi, near.lo, pick[1]);
            at += 2 * __popc(nibble);
        }
    }
}

// A workgroup has 16 rows and NT * 16 tokens; its waves take the tiles along the columns in turn, and their sums meet in LDS.
template <int TYPE, bool GATED, bool WIDE, int NT, int CHUNKS>
__global__ __launch_bounds__(64 * kMostWaves) void linear_few_kernel(const LinearArgs a, int buffer) {
    extern __shared__ char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    constexpr int kSize = sizeof(typename Num<TYPE>::type), kParts = kSize == 4 ? 2 : 1;
    const int rt = blockIdx.x, token0 = blockIdx.y * NT * 16;
    u2* const picks = (u2*)lds;
    char* const values = lds + 128 + wave * buffer;
    if (threadIdx.x < 16) {
        uint32_t p[4], pos = 0;
        for (int j = 0; j < 4; ++j) {
            p[j] = threadIdx.x >> j & 1 ? (2 * pos + 1) << 8 | 2 * pos : 0x0c0cu;  // 0x0c picks a byte of zeros
            pos += threadIdx.x >> j & 1;
        }
        picks[threadIdx.x] = u2{p[0] | p[1] << 16, p[2] | p[3] << 16};
    }
    __syncthreads();
    f4 sum[NT] = {};
    const int64_t first = (int64_t)rt * a.col_tiles;
    Load<CHUNKS> next;
    if (wave < a.col_tiles) ask(a, first + wave, lane, next);
    const int end = a.K * kSize;
    const char* row[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) row[t] = a.in + min(token0 + t * 16 + lane % 16, a.T - 1) * a.ld_in;
    for (int ct = wave; ct < a.col_tiles; ct += waves) {
        const uint32_t mask = next.mask;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) *(u4*)(values + c * 1024 + lane * 16) = next.v[c];
        // the wave's lanes read what others of them have written: in order, as all LDS accesses of a wave are
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        if (ct + waves < a.col_tiles) ask(a, first + ct + waves, lane, next);
        const int at = lanes_before(__popc(mask)) * kSize;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            u4 w[kParts];
            expand<TYPE>(values, picks, mask, at, b, w);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    const u4 x = input16<TYPE, WIDE>(a, row[t], (ct * kTileCols + b * 32 + lane / 16 * 8) * kSize + p * 16, end);
                    sum[t] = mfma16<TYPE>(w[p], x, sum[t]);
                }
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
    // a lane reads up to 8 bytes from where its values end
    const int buffer = CHUNKS * 1024 + 16, lds = 128 + std::max(waves * buffer, NT * waves * 1024);
    const dim3 grid((unsigned)a.row_tiles, (unsigned)((a.T + NT * 16 - 1) / (NT * 16))), block(64 * waves);
    if (!grid_fits((double)grid.x * grid.y, 64 * waves)) return ESCOIN_ERANGE;
    const auto kernel = linear_few_kernel<TYPE, GATED, WIDE, NT, CHUNKS>;
    const int rc = lds > 64 * 1024 ? allow_dynamic_lds((const void*)kernel, lds) : ESCOIN_OK;
    return rc != ESCOIN_OK ? rc : launch(kernel, grid, block, (size_t)lds, stream, a, buffer);
}

template <int TYPE, bool GATED, bool WIDE, int NT>
int launch_chunks(const LinearHeader& h, const LinearArgs& a, int waves, hipStream_t stream) {
    const int chunks = (h.most_tile_bytes + 1023) / 1024;
    if constexpr (TYPE == ESCOIN_T_F32)
        if (chunks > 4) return launch_one<TYPE, GATED, WIDE, NT, 8>(a, waves, stream);
    if (chunks > 2) return launch_one<TYPE, GATED, WIDE, NT, 4>(a, waves, stream);
    if (chunks > 1) return launch_one<TYPE, GATED, WIDE, NT, 2>(a, waves, stream);
    return launch_one<TYPE, GATED, WIDE, NT, 1>(a, waves, stream);
}

template <int TYPE, bool GATED, bool WIDE>
int launch_tokens(const LinearHeader& h, const LinearArgs& a, hipStream_t stream) {
    const int waves = std::min(kMostWaves, a.col_tiles);
    if (a.T <= 16) return launch_chunks<TYPE, GATED, WIDE, 1>(h, a, waves, stream);
    if (a.T <= 32) return launch_chunks<TYPE, GATED, WIDE, 2>(h, a, waves, stream);
    return launch_chunks<TYPE, GATED, WIDE, 4>(h, a, waves, stream);
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
