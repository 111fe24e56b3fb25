// Pruned linear layers: what their plan holds and how a call is checked.
//
// The weights lie twice.  "Kept": for calls of few tokens, which are bound by the bytes of the weights: the nonzeros with a bit for
// each place, tile by tile of 16 rows and 128 columns.  "Whole": for calls of many tokens, which are bound by the matrix cores:
// zeros included, fragment by fragment of 32 rows and 32 bytes of columns.  Rows of a gated layer are taken in turn, a gate's and
// its partner's, so that one lane ends up with both.
#pragma once
#include "common.h"

namespace escoin {

constexpr uint32_t kLinearMagic = 0x4E494C45u;  // "ELIN"
constexpr uint32_t kLinearVersion = 1;

// Kept weights.  A lane of a tile has a row (lane % 16) and, of each 32 columns, eight (from 8 * (lane / 16)): as the
// 16x16 matrix instructions take them.  Its 32 bits of the mask are those in turn; its values follow one another, the
// lanes' after each other; tiles start on 16 bytes.
constexpr int kTileRows = 16, kTileCols = 128;
// A fragment of the whole weights: a lane's 16 bytes are row lane % 32, columns from lane / 32 * 16 bytes on.
constexpr int kFragRows = 32, kFragBytes = 1024;
constexpr int kStepFrags = 4;  // fragments along the columns that a step of the tiled kernel takes: 128 bytes of a row

struct LinearHeader {
    uint32_t magic, version;
    int32_t K, M, type, gated;
    int32_t most_tokens;    // of a call
    int32_t few_tokens;     // up to so many the kept weights are read; most_tokens above it: the whole ones are there too
    int32_t most_lane_words;// 32-bit words that the fullest lane's values of a tile touch
    int32_t reserved;
    uint64_t off_zero;      // 256 bytes of zeros
    uint64_t off_mask;      // [row tile][column tile][lane], 32 bits
    uint64_t off_start;     // [row tile][column tile] and one more: where the tile's values start, in 16 bytes from off_kept
    uint64_t off_kept, off_whole, total_bytes;
};

struct LinearDims {
    int T, K, M, type;
    bool gated;
    int64_t ld_in, ld_out, ld_residual;
    int size() const { return type == ESCOIN_T_F32 ? 4 : 2; }
    int rows() const { return gated ? 2 * M : M; }
    int row_tiles() const { return (rows() + kTileRows - 1) / kTileRows; }
    int col_tiles() const { return (K + kTileCols - 1) / kTileCols; }
    int row_frags() const { return (rows() + kFragRows - 1) / kFragRows; }
    int col_frags() const { return (int)(((int64_t)K * size() + 127) / 128) * kStepFrags; }
};

int make_linear_dims(const escoin_linear_desc* desc, LinearDims* d);
// The header of `plan` if it is a plan of this layer for calls of so many tokens.
int linear_header(const LinearDims& d, const void* plan, LinearHeader* h);

// What the kernels are given.
struct LinearArgs {
    const char* in;
    char* out;
    const char* bias;
    const char* residual;
    const char* zero;       // of the plan, 256 bytes
    const uint32_t* mask;
    const uint32_t* start;
    const char* kept;
    const char* whole;
    int T, K, M, rows;
    int row_tiles, col_tiles, row_frags, col_frags;
    int64_t ld_in, ld_out, ld_residual;  // bytes
    uint32_t flags;
};

// How a call goes out: on a stream, or, with `told`, not at all, and it is told which kernel it would be.
struct LinearCall {
    hipStream_t stream;
    escoin_linear_kernel_info* told;
};

int launch_linear_few(const LinearDims& d, const LinearHeader& h, const LinearArgs& a, const LinearCall& call);
int launch_linear_many(const LinearDims& d, const LinearHeader& h, const LinearArgs& a, const LinearCall& call);

}  // namespace escoin
