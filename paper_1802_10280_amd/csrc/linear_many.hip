// Pruned linear layers for many tokens: the whole weights in tiles on the matrix cores.
#include "linear_device.h"
#include "mfma.h"

namespace escoin {
namespace {

constexpr int kXcds = 8, kGroup = 8;

// The tile of a workgroup.  Workgroups go to the XCDs in turn; each XCD gets tiles that follow one another, and those that run
// together share rows and tokens in its L2.
__device__ inline void place(int n_rows, int n_tokens, int* row, int* token) {
    const int total = n_rows * n_tokens, id = blockIdx.x, per = total / kXcds, more = total % kXcds, xcd = id % kXcds;
    const int i = xcd * per + min(xcd, more) + id / kXcds;
    const int group = i / (kGroup * n_tokens), first = group * kGroup, height = min(kGroup, n_rows - first), in = i - first * n_tokens;
    *row = first + in % height;
    *token = in / height;
}

constexpr int many_pitch(int fragments) { return fragments * 128 + 16; }  // bytes of a token's fp32 sums in LDS

// A workgroup's waves, WM by WN of them, share BM rows and BN tokens.  A step's weights lie in LDS fragment by fragment, its inputs
// token by token, the 16-byte pieces of a token's 128 bytes (SF = 8: 256) turned about by its number so that 16 lanes' reads meet all banks.
// NS steps are in LDS in a ring: while one is multiplied, the next ones come.  WK waves share a tile's columns, fragment by fragment.  A wave reads its next fragments while it multiplies; the
// last of a step are in registers when the waves meet, so that what follows the meeting has work to hide behind.
template <int TYPE, bool GATED, bool WIDE, int BM, int BN, int WM, int WN, int WK, int NS, int SF = kStepFrags>
__global__ __launch_bounds__(64 * WM * WN * WK) void linear_many_kernel(const LinearArgs a, int n_row_tiles, int n_token_tiles) {
    extern __shared__ char lds[];
    constexpr int kWaves = WM * WN * WK, kThreads = 64 * kWaves, kFM = BM / 32 / WM, kFN = BN / 32 / WN;  // fragments of a wave
    constexpr int kStep = SF * 32, kTokenPieces = SF * 2;  // bytes of a row to a step, pieces of 16 of them
    constexpr int kWeightBytes = BM * kStep, kBuffer = (BM + BN) * kStep;
    constexpr int kSize = sizeof(typename Num<TYPE>::type), kPieces = BN * kTokenPieces / kThreads, kFrags = BM / 32 * SF / kWaves;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int row_tile, token_tile;
    place(n_row_tiles, n_token_tiles, &row_tile, &token_tile);
    const int row0 = row_tile * BM, token0 = token_tile * BN, end = a.K * kSize, steps = (a.col_frags + SF - 1) / SF;

    // What a thread copies: of the weights 16 bytes of the wave's share of the fragments, of the inputs a piece of every
    // kThreads / kTokenPieces tokens, by way of buffers: 32-bit offsets leave the registers to the sums, and the compiler waits for every LDS read
    // as long as a copy to LDS by a global address is on its way.
    const auto turned = [](int token) { return SF == 4 ? token >> 1 & 7 : token & 15; };
    const int my_token = tid / kTokenPieces, piece = tid % kTokenPieces ^ turned(my_token);
    const char* const x_base = a.in + token0 * a.ld_in;
    const Buffer w_buffer = buffer(a.whole + (size_t)(row0 / kFragRows) * a.col_frags * kFragBytes, 0xffffffffu), x_buffer = buffer(x_base, 0xffffffffu);
    const int frag_rows = a.row_frags - row0 / kFragRows;  // from the tile's first on
    uint32_t x_off[kPieces];
    const char* x_row[WIDE ? 1 : kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const int token = min(p * (kThreads / kTokenPieces) + my_token, a.T - 1 - token0);
        if constexpr (WIDE) x_off[p] = (uint32_t)token * (uint32_t)a.ld_in + piece * 16;
        else x_row[p] = x_base + token * a.ld_in;
    }
    // Beyond the last column a token's piece is its first one of the last step once more: the weights are zeros there, and the token's
    // own inputs can do no harm to it that they do not do anyway.
    const uint32_t last_back = (steps - 1) * kStep + piece * 16 < end ? 0 : piece * 16;
    static_assert(WIDE || NS > 2, "what is held in registers comes to LDS a step later");
    u4 held[WIDE ? 1 : kPieces];
    const auto ask = [&](int step, char* to) {
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            const int i = f * kWaves + wave, frag = min(i / SF, frag_rows - 1), col = step * SF + i % SF;
            copy16(w_buffer, lane * 16, (frag * a.col_frags + (SF == kStepFrags ? col : min(col, a.col_frags - 1))) * kFragBytes, to + i * kFragBytes);
        }
        if constexpr (WIDE) {
            char* const x_to = to + kWeightBytes + wave * 1024;
            const uint32_t back = step + 1 == steps ? last_back : 0;
#pragma unroll
            for (int p = 0; p < kPieces; ++p) copy16(x_buffer, x_off[p] - back, step * kStep, x_to + p * kThreads * 16);
        } else {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                if ((step + 1) * kStep <= end) held[p] = any16<TYPE>(x_row[p] + step * kStep + piece * 16);
                else held[p] = input16<TYPE, false>(a, x_row[p], step * kStep + piece * 16, end);
            }
        }
    };
    const auto put = [&](char* to) {
        if constexpr (!WIDE)
#pragma unroll
            for (int p = 0; p < kPieces; ++p) *(u4*)(to + kWeightBytes + (p * kThreads + tid) * 16) = held[p];
    };

    f16v sum[kFM][kFN] = {};
    const int wk = wave / (WM * WN), wm = wave / WN % WM, wn = wave % WN;
    const int turn = turned(lane & 31), q = lane >> 5, w_at = (wm * kFM * SF + wk) * kFragBytes + lane * 16;
    const int x_at = kWeightBytes + (wn * kFN * 32 + lane % 32) * kStep;
    u4 w[2][kFM], x[2][kFN];
    const auto read = [&](const char* from, int k, int to) {
#pragma unroll
        for (int n = 0; n < kFN; ++n) x[to][n] = *(const u4*)(from + x_at + n * 32 * kStep + ((((k * WK + wk) * 2 + q) ^ turn) * 16));
#pragma unroll
        for (int m = 0; m < kFM; ++m) w[to][m] = *(const u4*)(from + w_at + (m * SF + k * WK) * kFragBytes);
    };
    const auto multiply = [&](int from, int frag) {
        if (SF > kStepFrags && frag >= a.col_frags) return;  // steps of eight fragments where the last holds four
#pragma unroll
        for (int m = 0; m < kFM; ++m)
#pragma unroll
            for (int n = 0; n < kFN; ++n) sum[m][n] = mfma32<TYPE>(w[from][m], x[from][n], sum[m][n]);
    };
    // The copies of the step after next and later ones may still be on their way when the next one's are needed.
    const auto arrived = [&](bool all) {
        constexpr int kLater = (NS - 2) * (kFrags + kPieces);
        static_assert(kLater < 64, "six bits count the loads on their way");
        in_order();
        if (all || NS == 2) __builtin_amdgcn_s_waitcnt(0);
        else __builtin_amdgcn_s_waitcnt(0x0070 | (kLater & 15) | (kLater >> 4) << 14);  // and for all of LDS
        __builtin_amdgcn_s_barrier();
        in_order();
    };
#pragma unroll
    for (int s = 0; s < NS - 1; ++s)
        if (s < steps) {
            ask(s, lds + s * kBuffer);
            put(lds + s * kBuffer);
            in_order();
        }
    arrived(steps < NS);
    constexpr int kOwn = SF / WK;  // fragments of a step that are a wave's
    static_assert(kOwn % 2 == 0, "a step's first fragments take the registers that its last ones leave alone");
    int at = 0;                   // the step's place in the ring
    read(lds, 0, 0);
    for (int step = 0; step < steps; ++step) {
        const char* const now = lds + at * kBuffer;
        char* const free = lds + (at == 0 ? NS - 1 : at - 1) * kBuffer;
        const bool more = step + NS - 1 < steps;
        // inputs held in registers since the last step, for the one that comes before this step's copies
        if (!WIDE && step > 0 && step + NS - 2 < steps) put(lds + (at >= 2 ? at - 2 : at + NS - 2) * kBuffer);
        if (more) ask(step + NS - 1, free);
        if (++at == NS) at = 0;
#pragma unroll
        for (int k = 0; k < kOwn - 1; ++k) {
            read(now, k + 1, ~k & 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(k & 1, step * SF + k * WK + wk);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (step + 1 < steps) {
            arrived(!more);
            read(lds + at * kBuffer, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        multiply(1, step * SF + (kOwn - 1) * WK + wk);
        __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // The sums go through LDS, in fp32: those of the waves that shared the columns are added up, and rows' outputs are stored side by side.
    // A wave has kOut rows of 32 tokens there at a time; 16 bytes between tokens spread them over the banks.
    constexpr int kOut = kFM * 32, kPitch = many_pitch(kFM), kTurn = 32 * kPitch;
    char* const mine = lds + wave * kTurn;
#pragma unroll
    for (int n = 0; n < kFN; ++n) {
        if (WK > 1 && n) __syncthreads();
#pragma unroll
        for (int m = 0; m < kFM; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f4*)(mine + lane % 32 * kPitch + (m * 32 + i * 8 + q * 4) * 4) = f4{sum[m][n][4 * i], sum[m][n][4 * i + 1], sum[m][n][4 * i + 2], sum[m][n][4 * i + 3]};
        if constexpr (WK > 1) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
        constexpr int kFours = GATED ? 4 : 2, kParts = kOut / (4 * kFours);  // a lane stores 16 bytes of 16-bit outputs
#pragma unroll
        for (int c = 0; c < (kParts + 2 * WK - 1) / (2 * WK); ++c) {
            const int e = (c * WK + wk) * 64 + lane, token = e / kParts, part = e % kParts;
            if (token >= 32) continue;
            f4 z[kFours];
#pragma unroll
            for (int h = 0; h < kFours; ++h) {
                const char* const p = lds + wave % (WM * WN) * kTurn + token * kPitch + (part * kFours + h) * 16;
                z[h] = *(const f4*)p;
#pragma unroll
                for (int k = 1; k < WK; ++k) z[h] += *(const f4*)(p + k * WM * WN * kTurn);
            }
            finish<TYPE, GATED>(a, z, row0 + wm * kOut + part * 4 * kFours, token0 + (wn * kFN + n) * 32 + token);
        }
        if constexpr (WK == 1) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
}

template <int TYPE, bool GATED, bool WIDE, int BM, int BN, int WM, int WN, int WK, int NS, int SF = kStepFrags>
int launch_one(const LinearArgs& a, const LinearCall& call) {
    constexpr int kLds = std::max(NS * (BM + BN) * SF * 32, WM * WN * WK * 32 * many_pitch(BM / 32 / WM)), kThreads = 64 * WM * WN * WK;
    const int64_t rows = (a.rows + BM - 1) / BM, tokens = ((int64_t)a.T + BN - 1) / BN;
    if (!grid_fits((double)rows * tokens, kThreads)) return ESCOIN_ERANGE;
    if (call.told) {
        *call.told = {0, BM, BN, kThreads / 64, WIDE ? 2 : 0, 0, 0, NS, SF * 32, kLds};
        return ESCOIN_OK;
    }
    const auto kernel = linear_many_kernel<TYPE, GATED, WIDE, BM, BN, WM, WN, WK, NS, SF>;
    const int rc = kLds > 64 * 1024 ? allow_dynamic_lds((const void*)kernel, kLds) : ESCOIN_OK;
    return rc != ESCOIN_OK ? rc : launch(kernel, dim3((unsigned)(rows * tokens)), dim3(kThreads), (size_t)kLds, call.stream, a, (int)rows, (int)tokens);
}

// Which tile: the one whose steps take the least time, by how many of its tiles the fullest compute unit gets.  Microseconds a step of 128 bytes a row,
// measured with 256 to 25000 rows and 64 to 4096 tokens: 16-bit types are bound by the copies to LDS with small tiles (a step of 64 by 64
// brings 16 KB for 0.5 MFLOP, of 256 by 256 64 KB for 8), fp32 by the matrix cores with any, so that there the smallest come
// first (64 by 64 take 0.52, never less than the two of 64 by 32 in their place).  Inputs that come through registers have the tiles whose ring holds three steps or more.
template <int TYPE, bool GATED, bool WIDE>
int launch_tile(const LinearArgs& a, const LinearCall& call) {
    const auto tiles = [&](int rows, int tokens) { return ((int64_t)a.rows + rows - 1) / rows * (((int64_t)a.T + tokens - 1) / tokens); };
    const auto rounds = [](int64_t n, int units) { return (double)((n + units - 1) / units); };
    if constexpr (TYPE == ESCOIN_T_F32) {
        const int64_t n32 = tiles(64, 32);
        const double t32 = n32 <= 256 ? 0.24 : 0.255 * rounds(n32, 256), t128 = 1.95 * rounds(tiles(128, 128), 256);
        // (two small tiles to a compute unit or fewer: twice the columns to a step, by more waves; 1001 to 1503, 250 tokens 16.7 us and 18.4)
        if (t32 < t128)
            return n32 <= 512 ? launch_one<TYPE, GATED, WIDE, 64, 32, 2, 1, 4, 3, 8>(a, call) : launch_one<TYPE, GATED, WIDE, 64, 32, 2, 1, 2, 4>(a, call);
        return launch_one<TYPE, GATED, WIDE, 128, 128, 2, 2, 2, WIDE ? 2 : 4>(a, call);
    } else {
        // one tile of 128 by 128 to a compute unit, four steps on their way; or two, a step each
        const int64_t n128 = tiles(128, 128);
        const int64_t n32 = tiles(64, 32), n64 = tiles(64, 64);
        const double t32 = n32 <= 256 ? 0.135 : 0.15 * rounds(n32, 256), t64 = n64 <= 256 ? 0.185 : 0.22 * rounds(n64, 256), small = std::min(t32, t64);
        const double t128 = n128 <= 256 ? 0.46 : WIDE ? 1.05 * rounds(n128, 512) : 0.46 * rounds(n128, 256);
        if constexpr (WIDE) {
            const double tall = 0.97 * rounds(tiles(256, 128), 256), large = 1.6 * rounds(tiles(256, 256), 256);
            if (large < std::min(std::min(small, t128), tall)) return launch_one<TYPE, GATED, WIDE, 256, 256, 2, 4, 1, 2>(a, call);
            if (tall < std::min(small, t128)) return launch_one<TYPE, GATED, WIDE, 256, 128, 2, 2, 2, 3>(a, call);
        }
        // (one small tile to a compute unit: half as many steps of twice the columns, by more waves; 2560 to 2560, 53 tokens 9.4 us and 10.3)
        if (t32 < std::min(t64, t128))
            return n32 <= 256 ? launch_one<TYPE, GATED, WIDE, 64, 32, 2, 1, 4, 3, 8>(a, call) : launch_one<TYPE, GATED, WIDE, 64, 32, 2, 1, 2, 4>(a, call);
        if (t64 < t128)
            return n64 <= 256 ? launch_one<TYPE, GATED, WIDE, 64, 64, 2, 2, 2, 3, 8>(a, call) : launch_one<TYPE, GATED, WIDE, 64, 64, 2, 2, 2, 3>(a, call);
        if constexpr (WIDE)
            if (n128 > 256) return launch_one<TYPE, GATED, WIDE, 128, 128, 2, 2, 2, 2>(a, call);
        return launch_one<TYPE, GATED, WIDE, 128, 128, 2, 2, 2, 4>(a, call);
    }
}

template <int TYPE>
int launch_type(const LinearDims& d, const LinearArgs& a, const LinearCall& call) {
    const bool wide = wide_input(a, d.size());
    if (d.gated) return wide ? launch_tile<TYPE, true, true>(a, call) : launch_tile<TYPE, true, false>(a, call);
    return wide ? launch_tile<TYPE, false, true>(a, call) : launch_tile<TYPE, false, false>(a, call);
}

}  // namespace

int launch_linear_many(const LinearDims& d, const LinearHeader&, const LinearArgs& a, const LinearCall& call) {
    if (d.type == ESCOIN_T_F32) return launch_type<ESCOIN_T_F32>(d, a, call);
    if (d.type == ESCOIN_T_F16) return launch_type<ESCOIN_T_F16>(d, a, call);
    return launch_type<ESCOIN_T_BF16>(d, a, call);
}

}  // namespace escoin
