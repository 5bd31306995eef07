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
