// Pruned linear layers for many tokens: the whole weights in tiles on the matrix cores.
#include "linear_device.h"
#include "mfma.h"

namespace escoin {
namespace {

constexpr int kThreads = 256, kStep = kStepFrags * 32;  // bytes of a row to a step
constexpr int kXcds = 8, kGroup = 8;

typedef __attribute__((address_space(3))) void* Lds;

__device__ inline void copy16(const void* from, char* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (Lds)lds, 16, 0, 0);
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

// A workgroup's four waves have BM / 2 rows and BN / 2 tokens each.  A step's weights lie in LDS fragment by fragment, its inputs
// token by token, the 16-byte pieces of a token's 128 bytes turned about by its number so that a fragment's reads meet all banks.
template <int TYPE, bool GATED, bool WIDE, int BM, int BN>
__global__ __launch_bounds__(kThreads) void linear_many_kernel(const LinearArgs a, int n_row_tiles, int n_token_tiles) {
    extern __shared__ char lds[];
    constexpr int kFM = BM / 64, kFN = BN / 64;  // fragments of a wave
    constexpr int kWeightBytes = BM * kStep, kBuffer = (BM + BN) * kStep;
    constexpr int kSize = sizeof(typename Num<TYPE>::type), kPieces = BN * 8 / kThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int row_tile, token_tile;
    place(n_row_tiles, n_token_tiles, &row_tile, &token_tile);
    const int row0 = row_tile * BM, token0 = token_tile * BN, end = a.K * kSize, steps = a.col_frags / kStepFrags;

    // what this thread copies: of the weights, 16 bytes of the wave's share of the fragments; of the inputs, a piece of every kThreads / 8 tokens
    const char* w_from[kFM * 2];
#pragma unroll
    for (int f = 0; f < kFM * 2; ++f) {
        const int frag = min(row0 / kFragRows + f, a.row_frags - 1);
        w_from[f] = a.whole + ((size_t)frag * a.col_frags + wave) * kFragBytes + lane * 16;
    }
    const int piece = (tid & 7) ^ (tid >> 3 & 7);
    const char* x_from[kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) x_from[p] = a.in + min(token0 + p * (kThreads / 8) + (tid >> 3), a.T - 1) * a.ld_in;
    u4 held[WIDE ? 1 : kPieces];

    const auto ask = [&](int step, char* to) {
#pragma unroll
        for (int f = 0; f < kFM * 2; ++f) copy16(w_from[f] + (size_t)step * (kStepFrags * kFragBytes), to + (f * kStepFrags + wave) * kFragBytes);
        const int at = step * kStep + piece * 16;
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
            if constexpr (WIDE) copy16(at < end ? x_from[p] + at : a.zero, to + kWeightBytes + (p * kThreads + wave * 64) * 16);
            else held[p] = input16<TYPE, false>(a, x_from[p], at, end);
    };
    const auto put = [&](char* to) {
        if constexpr (!WIDE)
#pragma unroll
            for (int p = 0; p < kPieces; ++p) *(u4*)(to + kWeightBytes + (p * kThreads + tid) * 16) = held[p];
    };

    f16v sum[kFM][kFN] = {};
    const int wm = wave >> 1, wn = wave & 1;
    const int x_at = kWeightBytes + (wn * kFN * 32 + lane % 32) * kStep, turn = lane & 7, q = lane >> 5;
    ask(0, lds);
    put(lds);
    for (int step = 0; step < steps; ++step) {
        char* const now = lds + (step & 1) * kBuffer;
        char* const then = lds + (~step & 1) * kBuffer;
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (step + 1 < steps) ask(step + 1, then);
#pragma unroll
        for (int k = 0; k < kStepFrags; ++k) {
            u4 w[kFM], x[kFN];
#pragma unroll
            for (int m = 0; m < kFM; ++m) w[m] = *(const u4*)(now + ((wm * kFM + m) * kStepFrags + k) * kFragBytes + lane * 16);
#pragma unroll
            for (int n = 0; n < kFN; ++n) x[n] = *(const u4*)(now + x_at + n * 32 * kStep + (((k * 2 + q) ^ turn) * 16));
#pragma unroll
            for (int m = 0; m < kFM; ++m)
#pragma unroll
                for (int n = 0; n < kFN; ++n) sum[m][n] = mfma32<TYPE>(w[m], x[n], sum[m][n]);
        }
        if (step + 1 < steps) put(then);
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

template <int TYPE, bool GATED, bool WIDE, int BM, int BN>
int launch_one(const LinearArgs& a, hipStream_t stream) {
    constexpr int kLds = 2 * (BM + BN) * kStep;
    const int64_t rows = (a.rows + BM - 1) / BM, tokens = ((int64_t)a.T + BN - 1) / BN;
    if (!grid_fits((double)rows * tokens, kThreads)) return ESCOIN_ERANGE;
    const auto kernel = linear_many_kernel<TYPE, GATED, WIDE, BM, BN>;
    const int rc = kLds > 64 * 1024 ? allow_dynamic_lds((const void*)kernel, kLds) : ESCOIN_OK;
    return rc != ESCOIN_OK ? rc : launch(kernel, dim3((unsigned)(rows * tokens)), dim3(kThreads), (size_t)kLds, stream, a, (int)rows, (int)tokens);
}

template <int TYPE, bool GATED, bool WIDE>
int launch_tile(const LinearArgs& a, hipStream_t stream) {
    return launch_one<TYPE, GATED, WIDE, 128, 128>(a, stream);
}

template <int TYPE>
int launch_type(const LinearDims& d, const LinearArgs& a, hipStream_t stream) {
    const bool wide = wide_input(a, d.size());
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
