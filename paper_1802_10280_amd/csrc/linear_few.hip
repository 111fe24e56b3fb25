// Pruned linear layers for few tokens: the kept weights, read once.
#include "linear_device.h"
#include "mfma.h"

namespace escoin {
namespace {

// Waves of a workgroup: 16, or 8 where the loads on their way (inputs of one tile, values of two) do not fit 128 registers.
constexpr int few_waves(int type, int NT) { return NT > 1 || type == ESCOIN_T_F32 ? 8 : 16; }

// How inputs come: by element, 16 bytes a lane straight to registers, or by way of LDS.  A lane's 16 bytes belong to one token, its
// neighbour's to the next: an access a lane, not one to four lanes, of the cache.  With 16 tokens that bound a call (306 of 337 clocks
// a tile, 24576 by 4096 at 90 %); through LDS, 256 bytes of a token after each other, they take a quarter.  Where the lanes'
// tokens are but a few, they are read together anyway.
enum { kInElements, kInRegisters, kInLds };

// LDS of a wave: a column of words for each lane, and a tile's inputs.  Where its last places are empty, a lane reads behind its last word
// (and drops it): 16-bit values come by three words, fp32 ones by one.
constexpr int few_columns(int type, int chunks) { return (4 * chunks + (type == ESCOIN_T_F32 ? 1 : 3)) * 256; }
constexpr int few_buffer(int type, int in, int NT, int chunks) { return few_columns(type, chunks) + (in == kInLds ? NT * (type == ESCOIN_T_F32 ? 8192 : 4096) : 0); }

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

// A buffer's size
__device__ inline uint32_t all_or_none(bool all) { return (uint32_t)__builtin_amdgcn_readfirstlane(all ? -1 : 0); }

// LDS by its byte address, which 32 bits hold
template <class V>
__device__ inline __attribute__((address_space(3))) V* at_lds(uint32_t address) {
    return (__attribute__((address_space(3))) V*)(uintptr_t)address;
}

// The weights of a lane's half of a tile (two blocks of eight), zeros in their places, from their bits.  column: the LDS address of the
// lane's first word, the next ones follow 256 bytes apart, so that the lanes' reads never meet in a bank.  at: which of its values is next.
template <int TYPE>
__device__ inline void expand(uint32_t picks, uint32_t column, uint32_t bits, uint32_t& at, u4 (&w)[2][TYPE == ESCOIN_T_F32 ? 2 : 1]) {
    if constexpr (TYPE == ESCOIN_T_F32) {
        uint32_t value[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            value[j] = *at_lds<uint32_t>(column + at * 256);
            at += bits >> j & 1;
        }
        __builtin_amdgcn_sched_barrier(0);  // all reads before the first is waited for
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j / 8][j / 4 % 2][j % 4] = value[j] & (uint32_t)__builtin_amdgcn_sbfe((int)bits, j, 1);
    } else {
        // four weights are bytes picked from the next eight: which ones depends on their four bits
        u2 pick[4];
        uint32_t near[4][3], shift[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const uint32_t nibble = bits >> 4 * n & 15;
            pick[n] = *at_lds<u2>(picks + nibble * 8);
            shift[n] = at * 2;
            const auto from = at_lds<uint32_t>(column + (at & ~1u) * 128);
            near[n][0] = from[0], near[n][1] = from[64], near[n][2] = from[128];
            at += __popc(nibble);
        }
        __builtin_amdgcn_sched_barrier(0);  // all reads before the first is waited for
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const uint32_t lo = __builtin_amdgcn_alignbyte(near[n][1], near[n][0], shift[n]), hi = __builtin_amdgcn_alignbyte(near[n][2], near[n][1], shift[n]);
            w[n / 2][0][n % 2 * 2] = __builtin_amdgcn_perm(hi, lo, pick[n][0]);
            w[n / 2][0][n % 2 * 2 + 1] = __builtin_amdgcn_perm(hi, lo, pick[n][1]);
        }
    }
}

// A workgroup has 16 rows and NT * 16 tokens; its waves take the tiles along the columns in turn, and their sums meet in LDS.  A wave's
// next two tiles are on their way while it multiplies one: the values in registers of their own, the inputs, which the L2 has, of one
// tile in the place of those just multiplied.
template <int TYPE, bool GATED, int IN, int NT, int CHUNKS>
__global__ __launch_bounds__(64 * few_waves(TYPE, NT)) void linear_few_kernel(const LinearArgs a) {
    extern __shared__ char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    constexpr int kSize = sizeof(typename Num<TYPE>::type), kParts = kSize == 4 ? 2 : 1, kBlockBytes = 32 * kSize;
    constexpr int kColumns = few_columns(TYPE, CHUNKS), kRowBytes = kTileCols * kSize, kX = IN == kInLds ? 4 * NT * kParts : 0;
    constexpr int kBuffer = kColumns + kX * 1024;
    const int rt = blockIdx.x, token0 = blockIdx.y * NT * 16;
    const uint32_t picks = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds, column = picks + 128 + wave * kBuffer + lane * 4;
    if (threadIdx.x < 16) {
        uint32_t p[4], pos = 0;
        for (int j = 0; j < 4; ++j) {
            p[j] = threadIdx.x >> j & 1 ? (2 * pos + 1) << 8 | 2 * pos : 0x0c0cu;  // 0x0c picks a byte of zeros
            pos += threadIdx.x >> j & 1;
        }
        ((u2*)lds)[threadIdx.x] = u2{p[0] | p[1] << 16, p[2] | p[3] << 16};
    }
    const int end = a.K * kSize, first_byte = lane / 16 * 8 * kSize;
    const char* const in = a.in + token0 * a.ld_in;
    const char* x_row[NT];
    int x_off[NT];
    if constexpr (IN != kInLds) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int token = min(t * 16 + lane % 16, a.T - 1 - token0);
            if constexpr (IN == kInRegisters) x_off[t] = token * (int)a.ld_in + first_byte;
            else x_row[t] = in + token * a.ld_in;
        }
    }
    // By way of LDS: a token's pieces of 16 bytes, turned about by its number so that 16 tokens' reads meet all banks.
    constexpr int kTokenPieces = kRowBytes / 16, kTogether = 64 / kTokenPieces;
    const int piece_token = lane / kTokenPieces, piece_slot = lane % kTokenPieces;
    u4 x[4][NT][kParts];
    // (`there` is not a branch: a buffer without bytes gives zeros at once, and the compiler knows how many loads are on their way)
    const auto inputs = [&](int ct, bool there) {
        const Buffer x_buffer = buffer(in, all_or_none(there));
        const int from = ct * kRowBytes;
        const bool inside = from + kRowBytes <= end;
        if constexpr (IN == kInLds) {
#pragma unroll
            for (int i = 0; i < kX; ++i) {
                const int t = i * kTogether + piece_token, token = min(t, a.T - 1 - token0), at = (piece_slot ^ (t & 15)) * 16;
                // beyond the last column a token's first input of the tile once more: the weights are zeros there
                copy16(x_buffer, token * (int)a.ld_in + (inside || from + at < end ? at : 0), from, lds + 128 + wave * kBuffer + kColumns + i * 1024);
            }
            return;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    const int at = b * kBlockBytes + p * 16;
                    if constexpr (IN == kInElements) x[b][t][p] = input16<TYPE, false>(a, x_row[t], from + at + first_byte, end);
                    else if (inside) x[b][t][p] = load16(x_buffer, x_off[t] + at, from);
                    else x[b][t][p] = load16(x_buffer, x_off[t] + (from + at + first_byte < end ? at : -first_byte), from);
                }
    };
    const int64_t first = (int64_t)rt * a.col_tiles;
    const int tiles = (a.col_tiles - wave + waves - 1) / waves;  // of this wave
    // Where the wave's next 64 tiles start and end is kept a tile a lane.
    uint32_t begins, ends;
    const auto look = [&](int i) {
        const uint32_t* const p = a.start + first + min(wave + (i + lane) * waves, a.col_tiles - 1);
        begins = p[0], ends = p[1];
        asm volatile("" ::"v"(begins), "v"(ends));  // waited for here, and not once a tile
    };
    // A tile's mask is asked for a tile before its values: they start where the lanes before it end.
    u4 v[2][CHUNKS];
    uint32_t at[2], mask[3];
    const char* const masks = (const char*)(a.mask + first * 64);
    const auto ask_mask = [&](int i) -> uint32_t {
        return __builtin_amdgcn_raw_buffer_load_b32(buffer(masks, all_or_none(i < tiles)), lane * 4, (wave + i * waves) * 256, 0);
    };
    const auto ask = [&](int i, uint32_t bits, int to) {
        const uint32_t begin = __builtin_amdgcn_readlane(begins, i & 63), stop = __builtin_amdgcn_readlane(ends, i & 63), all = all_or_none(i < tiles);
        const Buffer from = buffer(a.kept + (uint64_t)begin * 16, ((stop - begin) * 16 + 16) & all);  // a lane's last 16 bytes may reach over the end
        const uint32_t before = lanes_before(__popc(bits));
        at[to] = kSize == 4 ? 0 : before & 1;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) v[to][c] = load16(from, (kSize == 4 ? before : before >> 1) * 4 + c * 16, 0);
    };
    look(0);
#pragma unroll
    for (int i = 0; i < 3; ++i) mask[i] = ask_mask(i);
    ask(0, mask[0], 0);
    if constexpr (IN == kInLds) {
        in_order();
        inputs(wave, true);
        in_order();
    }
    ask(1, mask[1], 1);
    if constexpr (IN != kInLds) inputs(wave, true);
    __syncthreads();
    f4 sum[NT] = {};
    const auto tile = [&](int i, int slot) {
        const uint32_t bits = mask[0];
        uint32_t from = at[slot];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) at_lds<uint32_t>(column)[(c * 4 + j) * 64] = v[slot][c][j];
        if constexpr (IN == kInLds) {
            // the tile's inputs have come once no more is on its way than the next tile's values
            in_order();
            __builtin_amdgcn_s_waitcnt(0x0f70 | CHUNKS);
            in_order();
            const char* const mine = lds + 128 + wave * kBuffer + kColumns + lane % 16 * kRowBytes;
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int p = 0; p < kParts; ++p)
                        x[b][t][p] = *(const u4*)(mine + t * 16 * kRowBytes + (((b * 4 + lane / 16) * kParts + p) ^ (lane & 15)) * 16);
            in_order();
            __builtin_amdgcn_s_waitcnt(0xc07f);  // read, before the next tile's take their place
            in_order();
            inputs(wave + (i + 1) * waves, i + 1 < tiles);
            in_order();
        }
        mask[0] = mask[1], mask[1] = mask[2], mask[2] = ask_mask(i + 3);
        if ((i & 63) == 62) look(i + 2);
        ask(i + 2, mask[1], slot);
        __builtin_amdgcn_sched_barrier(0);
        u4 w[2][2][kParts];
        expand<TYPE>(picks, column, bits, from, w[0]);
        expand<TYPE>(picks, column, bits >> 16, from, w[1]);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int p = 0; p < kParts; ++p) sum[t] = mfma16<TYPE>(w[b / 2][b % 2][p], x[b][t][p], sum[t]);
        if constexpr (IN != kInLds) inputs(wave + (i + 1) * waves, i + 1 < tiles);
    };
    // a tile beyond the last has neither weights nor inputs
    for (int i = 0; i < tiles; i += 2) {
        tile(i, 0);
        tile(i + 1, 1);
    }
    __builtin_amdgcn_s_waitcnt(0);  // the last copies to LDS, of nothing, do not meet the sums
    __syncthreads();
    f4* const parts = (f4*)(lds + 128);
#pragma unroll
    for (int t = 0; t < NT; ++t) parts[(t * waves + wave) * 64 + lane] = sum[t];
    __syncthreads();
    for (int t = wave; t < NT; t += waves) {
        f4 z[1] = {parts[t * waves * 64 + lane]};
        for (int k = 1; k < waves; ++k) z[0] += parts[(t * waves + k) * 64 + lane];
        finish<TYPE, GATED>(a, z, rt * 16 + lane / 16 * 4, token0 + t * 16 + lane % 16);
    }
}

template <int TYPE, bool GATED, int IN, int NT, int CHUNKS>
int launch_one(const LinearArgs& a, const LinearCall& call) {
    const dim3 grid((unsigned)a.row_tiles, (unsigned)((a.T + NT * 16 - 1) / (NT * 16)));
    constexpr int waves_at_most = few_waves(TYPE, NT);
    int waves = waves_at_most;
    constexpr int kWave = std::max(few_buffer(TYPE, IN, NT, CHUNKS), NT * 1024);
    waves = std::min(waves, (160 * 1024 - 128) / kWave);
    // fewer waves of more tiles each once they fill the compute units (the registers are for 12 or 20 on each)
    while (waves > 4 && (int64_t)grid.x * grid.y * waves > 256 * (waves_at_most == 8 ? 12 : 20)) waves /= 2;
    waves = std::min(waves, a.col_tiles);
    const int lds = 128 + waves * kWave;
    if (!grid_fits((double)grid.x * grid.y, 64 * waves)) return ESCOIN_ERANGE;
    if (call.told) {
        *call.told = {1, kTileRows, NT * 16, waves, IN, CHUNKS, few_columns(TYPE, CHUNKS) / 256, 0, 0, lds};
        return ESCOIN_OK;
    }
    const auto kernel = linear_few_kernel<TYPE, GATED, IN, NT, CHUNKS>;
    const int rc = lds > 64 * 1024 ? allow_dynamic_lds((const void*)kernel, lds) : ESCOIN_OK;
    return rc != ESCOIN_OK ? rc : launch(kernel, grid, dim3(64 * waves), (size_t)lds, call.stream, a);
}

template <int TYPE, bool GATED, int IN, int NT>
int launch_chunks(const LinearHeader& h, const LinearArgs& a, const LinearCall& call) {
    const int chunks = (h.most_lane_words + 3) / 4;
    if constexpr (TYPE == ESCOIN_T_F32) {
        if (chunks > 5) return launch_one<TYPE, GATED, IN, NT, 8>(a, call);
        if (chunks > 4) return launch_one<TYPE, GATED, IN, NT, 5>(a, call);
    } else if (chunks > 4) {
        return launch_one<TYPE, GATED, IN, NT, 5>(a, call);
    }
    if (chunks > 3) return launch_one<TYPE, GATED, IN, NT, 4>(a, call);
    if (chunks > 2) return launch_one<TYPE, GATED, IN, NT, 3>(a, call);
    if (chunks > 1) return launch_one<TYPE, GATED, IN, NT, 2>(a, call);
    return launch_one<TYPE, GATED, IN, NT, 1>(a, call);
}

template <int TYPE, bool GATED>
int launch_tokens(const LinearHeader& h, const LinearArgs& a, bool wide, const LinearCall& call) {
    // As many tokens to a workgroup as there are, up to 64: the weights are unfolded once for all of them (64 tokens, 12288 to 4096 at 50 %:
    // 33.8 us, by 32 40.3, by 16 47.2).  But where workgroups of 16 do not outnumber the compute units they are done sooner (1024 to 1024: 5.9, 6.7 by 32).
    const auto blocks = [&](int tokens) { return (int64_t)a.row_tiles * ((a.T + tokens - 1) / tokens); };
    const int nt = blocks(16) <= 256 ? 1 : a.T <= 32 || blocks(32) <= 256 ? 2 : 4;
    if (!wide) return a.T <= 16 || nt == 1 ? launch_chunks<TYPE, GATED, kInElements, 1>(h, a, call) : launch_chunks<TYPE, GATED, kInElements, 2>(h, a, call);
    if (a.T <= 4) return launch_chunks<TYPE, GATED, kInRegisters, 1>(h, a, call);
    if (a.T <= 16 || nt == 1) return launch_chunks<TYPE, GATED, kInLds, 1>(h, a, call);
    if constexpr (TYPE != ESCOIN_T_F32)  // (there are not the registers for more inputs)
        if (nt == 4) return launch_chunks<TYPE, GATED, kInLds, 4>(h, a, call);
    return launch_chunks<TYPE, GATED, kInLds, 2>(h, a, call);
}

template <int TYPE>
int launch_type(const LinearDims& d, const LinearHeader& h, const LinearArgs& a, const LinearCall& call) {
    const bool wide = wide_input(a, d.size());
    return d.gated ? launch_tokens<TYPE, true>(h, a, wide, call) : launch_tokens<TYPE, false>(h, a, wide, call);
}

}  // namespace

int launch_linear_few(const LinearDims& d, const LinearHeader& h, const LinearArgs& a, const LinearCall& call) {
    if (d.type == ESCOIN_T_F32) return launch_type<ESCOIN_T_F32>(d, h, a, call);
    if (d.type == ESCOIN_T_F16) return launch_type<ESCOIN_T_F16>(d, h, a, call);
    return launch_type<ESCOIN_T_BF16>(d, h, a, call);
}

}  // namespace escoin
