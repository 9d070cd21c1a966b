// How a call of the loss without logits (asi_head.hip) is laid out: which path, tiles and pieces of the vocabulary it takes, and what lies where
// in its workspace.  Host code alone, without the GPU's headers.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/asi_lm.h"

namespace asi {

constexpr int kStep = 64;                        // k of a step of the products
constexpr int kPlanes = 3, kPairs = 6;           // of an fp32 operand: its planes, and the products of planes

namespace {

// Rows that k_few and its gradients take; more are faster as a part of a tile.  (us so, and in tiles.  fp32 2048 x 32000: values of 64 rows 176
// and 301, of 100 325 and 308, with gradients of 64 541 and 568, of 100 1183 and 622.  bf16 as it lies, 2048 x 32000: values of 16 rows 36 and
// 38, of 32 rows 51 and 40, gradients of 16 rows 112 and 146.  bf16 that tiles cannot take as it lies: values of 64 rows 1000 x 50001 62 and 62,
// 200 x 50001 28 and 36; where rows are no whole vectors, 1001 x 50001, of 32 rows 101 and 91, of 64 165 and 91, 1001 x 3000 of 32 31 and 31;
// gradients of 32 rows 1000 x 50001 163 and 144, 200 x 50001 61 and 92, 1000 x 3000 38 and 58, of 48 rows 317, 110, 52 and 148, 94, 60.
// Gradients of 8 rows 108 by matrix instructions, 114 without.)
constexpr int kFewF32 = 64, kFewBf16 = 16, kFewBf16Whole = 64, kFewBf16Packed = 32, kFewGradVector = 4;
// For bf16 inputs dz is held in two parts of bf16, 2^-16 of itself: rounded to one, it would add as much error as the results' own rounding, and
// where summands cancel, more than is left of them.
constexpr int kFineParts = 2;
constexpr int kKeepSteps = 8;
constexpr int kFewWaves = 4, kFewTokens = 64;        // waves of a workgroup of k_few, 16 tokens each; tokens of a step of k_few_grad
constexpr size_t kPieceBytes = size_t(96) << 20;     // dz of a piece in fp32, each of its three parts; logits that are kept
// dz of a piece in bf16, both parts: a sixteenth of the logits in fp32 between these bounds.  With gradients, us, 96 MiB, 116, 128, 144 and 192:
// 2731 of 4096 rows x 2048 x 32000 2154, 1990, 1978, 1979, 2032; 2000 x 2048 x 32000 1536, 1525, 1394, 1394, 1414; 8190 x 2048 x 100003
// 22129, with 128 19512, 192 18578.
constexpr size_t kFineBytes = size_t(128) << 20, kMostFineBytes = size_t(192) << 20;
// Sums of dH for bf16 (with dz 164 MiB), and for fp32.  (1500 x 512 x 100000 bf16 with gradients, us: 20 MiB 1383, 36 1268, 48 1281; 700 x 1000
// x 32000 382, 353, 354.)
constexpr size_t kFineSums = size_t(36) << 20, kSums = size_t(48) << 20;
// Packed weights of a piece.  Larger than a few rows' dz would ask for, so that a piece has tiles for the whole chip, and a bound between memory
// and time: fp32 with gradients, 150 rows x 2048 x 60000, us: 3054 with 96 MiB, 2396 with 192, 1985 with 384, 1425 with 768, 1420 with 1536; 700
// x 1000 x 32000 1212, 997 with 192 and more; 200 x 5120 x 70000 8475 with 384, 6730, 6140; 512 x 8192 x 70000 19950, 18450, 14720; of values
// alone, 150 x 2048 x 60000, 1168, 816, 610, 628; 1023 x 1000 x 50001 637, 676, 638, 636; 200 x 5120 x 70000 3028, 2132, 1933.
constexpr size_t kPackedBytes = size_t(768) << 20;

// What the gradient needs of a row: p = exp2(scale' (x - top) - log2sum); dz = [target] a - p (a + b (log p + entropy)).  Of the target
// a (1 - p) is -a expm1(log p), which keeps its bits where p is nearly 1.
struct RowInfo {
    float top, log2sum, a, b, entropy;
    int target, pad[2];
};

// What follows from the number of live rows, which the GPU alone knows.
struct Split {
    int rows, piece, splits, pad;                    // live rows; tokens of a piece; parts that the vocabulary of a piece is cut in for dH
};

struct Plan {
    bool f32, few, staged;                           // fp32; rows for k_few; weights are packed by pieces
    int planes, dz_planes, k_steps;                  // of the inputs, and of dz
    long long rows, dim, vocab, packed_dim;
    int tile;                                        // 128 or 256
    bool flexible;
    bool keep;                                       // logits are kept from the values to the gradient
    long long parts;                                 // of the values
    long long piece;                                 // tokens of a piece of the gradient, and of packed weights
    long long most_sums, most_splits;
    int few_blocks;                                  // of the vocabulary for few rows
    size_t logits, kept, split, live, place, hidden, weights, part, target, info, dz, sums, bytes;      // offsets
};
inline long long up(long long x, long long to) { return (x + to - 1) / to * to; }

// Tiles of a packed piece of n tokens: where they are too few to fill half the chip, small ones, which are through sooner (849 tokens of 1023
// rows x 1000 fp32: 68 us, 118 in large ones).
inline int piece_tile(const Plan& p, long long n) { return p.tile == 256 && p.staged && up(p.rows, 256) / 256 * (up(n, 256) / 256) < 128 ? 128 : p.tile; }
// The pieces of the vocabulary that the values are made in, in their order: the first token, how many, the size of the tiles, and which of the
// parts is the first tile's.
template <typename F> void each_piece(const Plan& p, F f) {
    const long long each = p.staged ? p.piece : p.vocab;
    long long part = 0;
    for (long long first = 0; first < p.vocab; first += each) {
        const long long n = p.vocab - first < each ? p.vocab - first : each;
        const int tile = piece_tile(p, n);
        f(first, n, tile, part);
        part += up(n, tile) / tile;
    }
}
inline Plan plan(const asi_linear_logprob_desc* d, bool grad) {
    Plan p{};
    p.f32 = d->dtype == ASI_F32;
    p.planes = p.f32 ? kPlanes : 1;
    p.dz_planes = p.f32 ? kPlanes : kFineParts;
    p.rows = d->rows; p.dim = d->dim; p.vocab = d->vocab;
    p.packed_dim = up(d->dim, kStep);
    p.k_steps = (int)(p.packed_dim / kStep);
    const bool whole = d->weight_stride % 8 == 0 && !d->any_address, as_it_lies = !p.f32 && whole && d->dim % kStep == 0 && d->weight_stride < (1 << 21);
    p.few = d->rows <= (p.f32 ? kFewF32 : as_it_lies ? kFewBf16 : !grad && whole ? kFewBf16Whole : kFewBf16Packed);
    p.staged = !p.few && !as_it_lies;
    // (92000 tokens x 256 bf16 with gradients of 32 rows, us: 124 in tiles of 128, 185 of 256)
    p.tile = d->rows > 128 && up(d->rows, 256) / 256 * (up(d->vocab, 256) / 256) >= 256 ? 256 : 128;
    const long long rows_up = up(d->rows, p.tile);
    size_t dz_bytes = kPieceBytes;
    if (!p.f32) {
        const size_t share = (size_t)rows_up * (size_t)d->vocab * 4 / 16;
        dz_bytes = (share < kFineBytes ? kFineBytes : share < kMostFineBytes ? share : kMostFineBytes) / kFineParts;
    }
    p.piece = (long long)(dz_bytes / 2 / (size_t)rows_up) / 256 * 256;
    if (p.piece < 256) p.piece = 256;
    if (p.piece > up(d->vocab, 256)) p.piece = up(d->vocab, 256);
    // packed weights have a limit of their own, but 4096 of them are taken whatever they need
    const long long most_packed = (long long)(kPackedBytes / (size_t)(p.planes * p.packed_dim * 2)) / 256 * 256;
    if (p.staged && p.piece > most_packed) p.piece = most_packed > 4096 ? most_packed : p.piece < 4096 ? p.piece : 4096;
    p.flexible = !p.staged;
    if (p.few) p.parts = (d->vocab + 16 * kFewWaves - 1) / (16 * kFewWaves);
    else each_piece(p, [&](long long, long long n, int tile, long long first_part) { p.parts = first_part + up(n, tile) / tile; });
    // parts that the vocabulary of a piece may be cut in for dH, and the memory for their sums: twice what fills the chip, but no more than
    // that or twice dH's size in fp32
    const long long tiles = (rows_up / p.tile) * (up(d->dim, p.tile) / p.tile), slots = p.tile == 256 ? 256 : 512;
    const long long memory = (long long)((p.f32 ? kSums : kFineSums) / 4) / (d->rows * d->dim > 0 ? d->rows * d->dim : 1);
    p.most_splits = (2 * slots + tiles - 1) / (tiles > 0 ? tiles : 1);
    if (p.most_splits > (memory > 2 ? memory : 2)) p.most_splits = memory > 2 ? memory : 2;
    if (p.most_splits > 32) p.most_splits = 32;
    if (p.most_splits < 2) p.most_splits = 2;
    p.most_sums = d->rows * p.most_splits;
    // blocks of the vocabulary for few rows' gradients: workgroups for the chip, two to four a CU, each with 64 tokens at least
    const long long few_columns = d->rows <= kFewGradVector ? 2048 : 256, few_want = 1024 / ((d->dim + few_columns - 1) / few_columns);
    const long long few_most = (d->vocab + kFewTokens - 1) / kFewTokens, few_cap = few_want < 1 ? 1 : few_want > 512 ? 512 : few_want;
    p.few_blocks = (int)(few_cap < few_most ? few_cap : few_most);
    // The logits of a vocabulary that is one piece, in fp32, where they are dearer to compute again than to read (3000 rows x 4000 bf16 with
    // gradients, us: dim 256 130 either way, 512 152 and 153 without, 1024 198 and 213, 2048 321 and 359; 700 x 2048 x 32000 570 and 617;
    // fp32 3000 x 256 x 4000 303 and 328, 3000 x 2048 x 4000 986 and 1265)
    const long long kept = 4 * rows_up * up(d->vocab, p.tile);
    p.keep = grad && !p.few && p.piece >= d->vocab && kept <= (long long)kPieceBytes && p.k_steps * (p.f32 ? kPairs : 1) >= kKeepSteps;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (size_t)up((long long)bytes, 256); return here; };
    const size_t rows = (size_t)d->rows;
    if (!p.few) {
        p.split = take(sizeof(Split));
        p.live = take(rows * 4);
        p.place = take(rows * 4);
        p.hidden = take((size_t)p.planes * rows * p.packed_dim * 2);
        if (p.staged) p.weights = take((size_t)p.planes * p.piece * p.packed_dim * 2);
    }
    p.target = take(rows * 4);
    if (grad) p.info = take(rows * sizeof(RowInfo));
    p.part = take((size_t)p.parts * 4 * rows * 4);
    if (grad && p.few) {
        p.logits = take((rows + 15) / 16 * 16 * (size_t)d->vocab * 4);
        p.sums = take((size_t)p.few_blocks * rows * d->dim * 4);
    } else if (grad) {
        // dz lies where the tiles' values were, which are joined by then
        p.dz = p.part;
        const size_t end = p.dz + (size_t)up((long long)p.dz_planes * rows_up * p.piece * 2, 256);
        if (at < end) at = end;
        if (p.keep) p.kept = take((size_t)kept);
        p.sums = take((size_t)p.most_sums * d->dim * 4);
    }
    p.bytes = at;
    return p;
}

}  // namespace
}  // namespace asi
