// Internal interfaces between the host code of the gated block (gated_block.hip) and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bmgd {

enum { kActSilu = 0, kActGelu = 1, kActRelu = 2 };

// A product that the block is made of.  "Adjacent" operands have the elements of the summed index next to each other in memory,
// "strided" ones a row of the matrix per value of the summed index.
enum GatedOp {
    kOpUp = 0,          // [G | U] = X [Wg | Wu]: left adjacent, right strided; H = act(G) * U leaves the kernel, G and U on request
    kOpMul = 1,         // Y = H Wd: left adjacent, right strided
    kOpDown = 2,        // dH = dY Wd': both adjacent; H, dG and dU leave the kernel
    kOpInput = 3,       // dX = dG Wg' + dU Wu': both adjacent, the sum runs over both halves
    kOpWeight = 4       // dWd = H' dY, [dWg | dWu] = X' [dG | dU]: both strided
};

struct GatedMat {
    void* p;
    int64_t ld;         // elements from one row to the next
};

// How a result is cut into tiles.
struct GatedCut {
    int tile;           // kTile*
    int tiles_m, tiles_n, splits, per_split;    // tiles of the result; workgroups that share a tile's sum, and their share in steps of 64
    int first_counter;
    size_t first_part;  // where its own counters and sums begin among those of a launch
    double us;          // what the launch is expected to take
};

struct GatedProduct : GatedCut {
    GatedMat a;         // left operand
    GatedMat b, b2;     // right operand; its second half for kOpUp and kOpInput
    int64_t M, N, K;    // rows and columns of the result as stored, length of the sum.  kOpUp: N = hidden; kOpInput: K = hidden, the
                        // length of one half; kOpWeight with two halves: N = hidden, the columns of one
    int64_t a_cols, b_cols;             // strided operands: columns that may be read
    bool loose;         // rows of the operands begin anywhere; else at multiples of 16 bytes, and columns and adjacent lengths are multiples of 8
    int64_t half;       // kOpUp, kOpDown: hidden rounded up to 64, the columns of H and of each half of D (zeros behind hidden);
                        // kOpInput: the columns of each half of the left operand; kOpWeight: 0, or the columns of each half of the right operand
    GatedMat out, out2; // result; kOpUp, kOpDown: H in `out`, kOpDown: D = [dG | dU] in `out2`
    GatedMat g, u;      // kOpUp: written unless NULL; kOpDown: read
    // Calls of few rows (kGatedPairRows): H and D have two rows for one, 2 r what row r is rounded to and 2 r + 1 the rest.  kOpUp, kOpDown write both; kOpMul, kOpInput have M of
    // them and add pairs of results; kOpWeight has K of them, and its other operand (twice_a, twice_b: the left, the right one) each row twice.
    int pair, twice_a, twice_b;
    int act;
    float* partial;     // sums of workgroups that share a tile
    unsigned* counter;  // and how many of them have arrived, per tile; zero between launches
    const void* zeros;  // 256 bytes of zeros
    // f16 only, NULL otherwise.  H, dG and dU may leave f16's range: then eight neighbouring elements of a row (a piece) are held as multiples of 2^e, e their byte here, at
    // the offset of the first element over eight.  kOpUp, kOpDown write those of `out` and `out2`, the others read those of their operand.
    unsigned char *scale, *scale2;
    unsigned* scaled;   // three words: [0] some call had an e that is not zero, so all are written from then on; [1 + turn] this call has
    int turn;           // of the call, 0 or 1; its second launch clears the other's word
};

// rows x columns: 256 x 256, 128 x 128 (two workgroups to a unit; one, steps further ahead), 64 x 64; for few rows 32 x 128 and 16 x 128
enum { kTileLarge = 0, kTileMedium = 1, kTileDeep = 2, kTileSmall = 3, kTile32 = 4, kTile16 = 5, kTiles = 6 };

// Bytes of partial sums, and tiles, that a product may use where workgroups share tiles.
constexpr size_t kGatedPartialBytes = size_t(64) << 20;
constexpr int kGatedCounters = 4096;
constexpr int kGatedStep = 64;         // elements of the summed index per step
// Up to so many rows H and D have the rest of their roundings too: two rows each of a tile of 16, or of a step.  There a rounding is shared by all that a row's sums make, and few
// of them make an error: beside a result's own rounding it is 1.3 to 1.8 times as large as with many rows (of 36 draws with one row 14 to 39 % are off by more than 1.5 times their own,
// with eight rows up to 11 %, with 16 up to 3 %, with 64 none).  It takes 1 to 4 % longer (one row, p = 512, hidden 2,048, out 1,000: forward 12.9 us for
// 12.7, backward 17.4 for 16.9; p = out = 4,096, hidden 8,192: 48.6 for 48.2 and 120.2 for 117.5); 9 to 16 rows, whose pairs need the tile of 32, would take up to 32 % (p = 64,
// hidden 8,192, out 64, forward: 16.5 for 12.5).
constexpr int kGatedPairRows = 8;

// Chooses tile and split for the `count` products of one launch, which get one kind of tile.
// tile >= 0: this one and `want` shares of a tile's sum where they fit (tests).
void gated_plan(GatedProduct* const* q, const GatedOp* op, int count, int num_cus, int tile = -1, int64_t want = 0);

// Whether a kind of tile has a form for operands at any address (whose rows have eight elements or more).
inline bool gated_can_be_loose(int tile) { return tile != kTileLarge; }

// Once per process and device: lets the kernels use as much shared memory as they need.
hipError_t gated_prepare_bf16();
hipError_t gated_prepare_f16();
hipError_t gated_launch_bf16(const GatedProduct& q, GatedOp op, hipStream_t stream);
hipError_t gated_launch_f16(const GatedProduct& q, GatedOp op, hipStream_t stream);
// dX (kOpInput), dWd and [dWg | dWu] (kOpWeight) in one launch; NULL leaves one out
hipError_t gated_launch_grads_bf16(const GatedProduct* input, const GatedProduct* down, const GatedProduct* gate, hipStream_t stream);
hipError_t gated_launch_grads_f16(const GatedProduct* input, const GatedProduct* down, const GatedProduct* gate, hipStream_t stream);

// Copies of up to five matrices of 16-bit elements whose rows do not begin at multiples of 16 bytes: rows of `to_ld` elements (a multiple of
// 8), zeros behind the last column.
struct GatedPack {
    struct One { const unsigned short* from; unsigned short* to; int64_t from_ld, to_ld, rows, cols; } m[5];
    int count;
};
hipError_t gated_launch_pack(const GatedPack& q, hipStream_t stream);

}  // namespace bmgd
