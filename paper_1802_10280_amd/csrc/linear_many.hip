// Pruned linear layers for many tokens: the whole weights in tiles on the matrix cores.
#include "linear_device.h"
#include "mfma.h"

namespace escoin {
namespace {

constexpr int kStep = kStepFrags * 32;  // bytes of a row to a step
constexpr int kXcds = 8, kGroup = 8;

typedef __attribute__((address_space(3))) void* Lds;
typedef __amdgpu_buffer_rsrc_t Buffer;

__device__ inline Buffer buffer(const char* p) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)0xffffffffu, 0x00020000); }
// 16 bytes a lane: 1024 of LDS from `to` on
__device__ inline void copy(Buffer from, int lane_offset, int offset, char* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (Lds)to, 16, lane_offset, offset, 0, 0);
}

// The tile of a workgroup.  Workgroups go to the XCDs in turn; each XCD gets tiles that follow one another, and those that run
// together share rows and tokens in its L2.
__device__ inline void place(int n_rows, int n_tokens, int* row, int* token) {
    const int total = n_rows * n_tokens, id = blockIdx.x, per = total / kXcds, more = total % kXcds, xcd = id % kXcds;
    const int i = xcd * per + min(xcd, more) + id / kXcds;
    const int group = i / (kGroup * n_tokens), first = group * kGroup, height = min(kGroup, n_rows - first), in = i - first * n_tokens;
    *row = first + in % height;
    *token = in / height;
}

// A workgroup's waves, WM by WN of them, share BM rows and BN tokens.  A step's weights lie in LDS fragment by fragment, its inputs
// token by token, the 16-byte pieces of a token's 128 bytes turned about by its number so that a fragment's reads meet all banks.
// Two steps are in LDS: while one is multiplied, the next one comes.  A wave reads its next fragments while it multiplies; the
// last of a step are in registers when the waves meet, so that what follows the meeting has work to hide behind.
template <int TYPE, bool GATED, bool WIDE, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void linear_many_kernel(const LinearArgs a, int n_row_tiles, int n_token_tiles) {
    extern __shared__ char lds[];
    constexpr int kWaves = WM * WN, kThreads = 64 * kWaves, kFM = BM / 32 / WM, kFN = BN / 32 / WN;  // fragments of a wave
    constexpr int kWeightBytes = BM * kStep, kBuffer = (BM + BN) * kStep;
    constexpr int kSize = sizeof(typename Num<TYPE>::type), kPieces = BN * 8 / kThreads, kFrags = BM / 32 * kStepFrags / kWaves;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int row_tile, token_tile;
    place(n_row_tiles, n_token_tiles, &row_tile, &token_tile);
    const int row0 = row_tile * BM, token0 = token_tile * BN, end = a.K * kSize, steps = a.col_frags / kStepFrags;

    // What a thread copies: of the weights 16 bytes of the wave's share of the fragments, of the inputs a piece of every kThreads / 8
    // tokens, by way of buffers: 32-bit offsets leave the registers to the sums, and the compiler waits for every LDS read
    // as long as a copy to LDS by a global address is on its way.
    const int piece = (tid & 7) ^ (tid >> 3 & 7);
    const char* const x_base = a.in + token0 * a.ld_in;
    const Buffer w_buffer = buffer(a.whole + (size_t)(row0 / kFragRows) * a.col_frags * kFragBytes), x_buffer = buffer(x_base);
    const int frag_rows = a.row_frags - row0 / kFragRows;  // from the tile's first on
    uint32_t x_off[kPieces];
    const char* x_row[WIDE ? 1 : kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const int token = min(p * (kThreads / 8) + (tid >> 3), a.T - 1 - token0);
        if constexpr (WIDE) x_off[p] = (uint32_t)token * (uint32_t)a.ld_in + piece * 16;
        else x_row[p] = x_base + token * a.ld_in;
    }
    // Beyond the last column a token's piece is its first one of the last step once more: the weights are zeros there, and the token's
    // own inputs can do no harm to it that they do not do anyway.
    const uint32_t last_back = (steps - 1) * kStep + piece * 16 < end ? 0 : piece * 16;
    u4 held[WIDE ? 1 : kPieces];
    const auto ask = [&](int step, char* to) {
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
            const int i = f * kWaves + wave, frag = min(i / kStepFrags, frag_rows - 1);
            copy(w_buffer, lane * 16, (frag * a.col_frags + step * kStepFrags + i % kStepFrags) * kFragBytes, to + i * kFragBytes);
        }
        if constexpr (WIDE) {
            char* const x_to = to + kWeightBytes + wave * 1024;
            const uint32_t back = step + 1 == steps ? last_back : 0;
#pragma unroll
            for (int p = 0; p < kPieces; ++p) copy(x_buffer, x_off[p] - back, step * kStep, x_to + p * kThreads * 16);
        } else {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) held[p] = input16<TYPE, false>(a, x_row[p], step * kStep + piece * 16, end);
        }
    };
    const auto put = [&](char* to) {
        if constexpr (!WIDE)
#pragma unroll
            for (int p = 0; p < kPieces; ++p) *(u4*)(to + kWeightBytes + (p * kThreads + tid) * 16) = held[p];
    };

    f16v sum[kFM][kFN] = {};
    const int wm = wave / WN, wn = wave % WN;
    const int turn = lane & 7, q = lane >> 5, w_at = wm * kFM * kStepFrags * kFragBytes + lane * 16, x_at = kWeightBytes + (wn * kFN * 32 + lane % 32) * kStep;
    u4 w[2][kFM], x[2][kFN];
    const auto read = [&](const char* from, int k, int to) {
#pragma unroll
        for (int n = 0; n < kFN; ++n) x[to][n] = *(const u4*)(from + x_at + n * 32 * kStep + (((k * 2 + q) ^ turn) * 16));
#pragma unroll
        for (int m = 0; m < kFM; ++m) w[to][m] = *(const u4*)(from + w_at + (m * kStepFrags + k) * kFragBytes);
    };
    const auto multiply = [&](int from) {
#pragma unroll
        for (int m = 0; m < kFM; ++m)
#pragma unroll
            for (int n = 0; n < kFN; ++n) sum[m][n] = mfma32<TYPE>(w[from][m], x[from][n], sum[m][n]);
    };
    ask(0, lds);
    put(lds);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    read(lds, 0, 0);
    for (int step = 0; step < steps; ++step) {
        char* const now = lds + (step & 1) * kBuffer;
        char* const then = lds + (~step & 1) * kBuffer;
        if (step + 1 < steps) ask(step + 1, then);
#pragma unroll
        for (int k = 0; k < kStepFrags - 1; ++k) {
            read(now, k + 1, ~k & 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(k & 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (step + 1 < steps) put(then);
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (step + 1 < steps) read(then, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        multiply((kStepFrags - 1) & 1);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int m = 0; m < kFM; ++m)
#pragma unroll
        for (int n = 0; n < kFN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f4 z = {sum[m][n][4 * i], sum[m][n][4 * i + 1], sum[m][n][4 * i + 2], sum[m][n][4 * i + 3]};
                finish<TYPE, GATED>(a, z, row0 + (wm * kFM + m) * 32 + i * 8 + q * 4, token0 + (wn * kFN + n) * 32 + lane % 32);
            }
}

template <int TYPE, bool GATED, bool WIDE, int BM, int BN, int WM, int WN>
int launch_one(const LinearArgs& a, hipStream_t stream) {
    constexpr int kLds = 2 * (BM + BN) * kStep, kThreads = 64 * WM * WN;
    const int64_t rows = (a.rows + BM - 1) / BM, tokens = ((int64_t)a.T + BN - 1) / BN;
    if (!grid_fits((double)rows * tokens, kThreads)) return ESCOIN_ERANGE;
    const auto kernel = linear_many_kernel<TYPE, GATED, WIDE, BM, BN, WM, WN>;
    const int rc = kLds > 64 * 1024 ? allow_dynamic_lds((const void*)kernel, kLds) : ESCOIN_OK;
    return rc != ESCOIN_OK ? rc : launch(kernel, dim3((unsigned)(rows * tokens)), dim3(kThreads), (size_t)kLds, stream, a, (int)rows, (int)tokens);
}

template <int TYPE, bool GATED, bool WIDE>
int launch_tile(const LinearArgs& a, hipStream_t stream) {
    const char* e = getenv("TILE");
    if (e && e[0] == 'a') return launch_one<TYPE, GATED, WIDE, 256, 256, 2, 2>(a, stream);
    if (e && e[0] == 'b') return launch_one<TYPE, GATED, WIDE, 256, 256, 2, 4>(a, stream);
    if (e && e[0] == 'c') return launch_one<TYPE, GATED, WIDE, 256, 128, 2, 2>(a, stream);
    if (e && e[0] == 'd') return launch_one<TYPE, GATED, WIDE, 256, 128, 4, 2>(a, stream);
    if (e && e[0] == 's') return launch_one<TYPE, GATED, WIDE, 64, 64, 2, 2>(a, stream);
    return launch_one<TYPE, GATED, WIDE, 128, 128, 2, 2>(a, stream);
}

template <int TYPE>
int launch_type(const LinearDims& d, const LinearArgs& a, hipStream_t stream) {
    // (a tile's rows are offsets of 32 bits)
    const bool wide = wide_input(a, d.size()) && a.ld_in < 1 << 23;
    if (d.gated) return wide ? launch_tile<TYPE, true, true>(a, stream) : launch_tile<TYPE, true, false>(a, stream);
    return wide ? launch_tile<TYPE, false, true>(a, stream) : launch_tile<TYPE, false, false>(a, stream);
}

}  // namespace

int launch_linear_many(const LinearDims& d, const LinearHeader&, const LinearArgs& a, hipStream_t stream) {
    if (d.type == ESCOIN_T_F32) return launch_type<ESCOIN_T_F32>(d, a, stream);
    if (d.type == ESCOIN_T_F16) return launch_type<ESCOIN_T_F16>(d, a, stream);
    return launch_type<ESCOIN_T_BF16>(d, a, stream);
}

}  // namespace escoin
