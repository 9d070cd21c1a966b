// Products of bf16 matrices in tiles for the loss without logits (asi_head.hip): C[m][n] += sum_k A(m, k) B(n, k) with sums in fp32.
//
// A workgroup of 4 waves (2 x 2) has a tile of BM x BN; a step takes 64 k of both operands from memory into LDS without registers in
// between and multiplies what the step before has brought.  Each operand lies in memory in one of two ways:
//   along k      a row is an m (or n), its k next to each other; LDS holds rows of 64 k, a lane reads 8 of them at once
//   across k     a row is a k, its m (or n) next to each other; LDS holds 64 rows, and the transposing LDS read hands each lane 4 k of
//                its column
// so that logits, gradients and weights are read as they lie and nothing is ever stored transposed.  In LDS the 16-byte pieces of a
// row are exchanged by its number, so that the lanes that read together meet different banks: the copy itself writes LDS in order, so
// it is the address in memory that is exchanged.
//
// An fp32 operand comes as three planes of bf16 whose sum it is (8 + 8 + 8 bits); the products of planes that matter to 2^-24 are
// six, the smallest first, and run through the same loop as a sixfold k.
#pragma once
#include "asi_lm_device.h"

namespace asi {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4h __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kTileThreads = 256;
constexpr int kStep = 64;                        // k of a step
constexpr int kPlanes = 3, kPairs = 6;           // of an fp32 operand: its planes, and the products of planes

// `rows` rows of `ld` elements, of which the first `cols` may be read; planes `plane` elements apart
struct Operand {
    const uint16_t* p;
    long long ld, plane;
    long long rows, cols;
};

// Pair number i of `pairs` (1 or 6): which plane of either side.
__device__ __forceinline__ int plane_a(int i, int pairs) { return pairs == 1 ? 0 : (0x001012 >> (4 * i)) & 15; }
__device__ __forceinline__ int plane_b(int i, int pairs) { return pairs == 1 ? 0 : (0x010210 >> (4 * i)) & 15; }

// An operand's side of a tile: N rows (along k) or columns (across k) from `at` on.
template <int N, bool ACROSS> struct Half {
    static constexpr int kBytes = N * kStep * 2;
    static constexpr int kCopies = kBytes / (kTileThreads * 16);          // a wave's copies of 1 KB in a step
    static constexpr int kPieces = ACROSS ? N / 8 : kStep / 8;            // 16-byte pieces of a row in LDS
    static constexpr int kRowsACopy = 64 / kPieces;
    static constexpr int kBlocks = N / 64;                                // blocks of 32 that a wave has

    const char* base;          // of the tile's corner in the present plane, at the present k
    long long left;            // bytes from there to the operand's end
    long long step;            // bytes from a step's k to the next one's
    int off, apart;            // a lane's first piece; from a copy's rows to the next one's
    int read[ACROSS ? kBlocks : kStep / 16];      // a lane's place in LDS: for each block (across k), or each 16 k (along k)

    __device__ __forceinline__ void start(const Operand& o, int plane, long long at) {
        base = reinterpret_cast<const char*>(o.p + (long long)plane * o.plane) + (ACROSS ? at : at * o.ld) * 2;
        left = ((o.rows - 1) * o.ld + o.cols) * 2 - (ACROSS ? at : at * o.ld) * 2;
        step = ACROSS ? kStep * o.ld * 2 : kStep * 2;
    }
    __device__ __forceinline__ void lanes(const Operand& o, int side) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int ld = (int)(o.ld * 2);
        const int row = kRowsACopy * wave * (ACROSS ? 1 : kCopies) + lane / kPieces, piece = lane % kPieces;
        off = row * ld + (piece ^ (ACROSS ? 4 * (row & 3) : row & 7)) * 16;
        apart = kRowsACopy * (ACROSS ? 4 : 1) * ld;
        if constexpr (ACROSS) {
            // 16 lanes read 4 rows of 16 columns, a row by 4 lanes, and get a column each
            const int in16 = lane & 15, k = (lane >> 5) * 8 + (in16 >> 2);
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) {
                const int piece_of = side * (N / 16) + 4 * j + ((lane >> 4) & 1) * 2 + ((in16 & 3) >> 1);
                read[j] = k * (N * 2) + (piece_of ^ (4 * (k & 3))) * 16 + (in16 & 1) * 8;
            }
        } else {
#pragma unroll
            for (int s = 0; s < kStep / 16; ++s)
                read[s] = (side * (N / 2) + (lane & 31)) * (kStep * 2) + ((2 * s + (lane >> 5)) ^ (lane & 7)) * 16;
        }
    }
    // copy number q of this wave's
    __device__ __forceinline__ void copy(char* lds, int q) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int bytes = left > 0x7fffffffLL ? 0x7fffffff : left > 0 ? (int)left : 0;
        copy16_to_lds(base, bytes, off + q * apart, lds + (ACROSS ? wave + 4 * q : wave * kCopies + q) * 1024);
    }
    __device__ __forceinline__ void advance() { base += step; left -= step; }
    // block i's values of the 16 k number s
    __device__ __forceinline__ v8bf frag(const char* lds, int i, int s) const {
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) v4h* Ptr;
            const char* at = lds + read[i] + s * 16 * (N * 2);
            const v4h lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(at + 4 * (N * 2)));
            return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const v8bf*>(lds + read[s] + i * 32 * (kStep * 2));
        }
    }
};

// The sums of a tile: acc[i][j] is the block of 32 x 32 at (m, n) = (at_m() + 32 i, at_n() + 32 j) of the tile; a lane has column
// lane % 32 of it and rows 8 (r / 4) + 4 (lane / 32) + r % 4.
template <int BM, int BN, bool A_ACROSS, bool B_ACROSS> struct Tile {
    static constexpr int kM = BM / 64, kN = BN / 64;
    using HalfA = Half<BM, A_ACROSS>;
    using HalfB = Half<BN, B_ACROSS>;
    static constexpr int kBuffer = HalfA::kBytes + HalfB::kBytes;
    static constexpr int kLds = 2 * kBuffer;
    v16f acc[kM][kN];

    __device__ __forceinline__ static int at_m() { return (threadIdx.x >> 7) * (BM / 2); }
    __device__ __forceinline__ static int at_n() { return ((threadIdx.x >> 6) & 1) * (BN / 2); }
    __device__ __forceinline__ static int row_of(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x >> 5) & 1) + (r & 3); }

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }

    // Adds the products of `pairs` pairs of planes over k_steps steps from k = 64 first on.  The whole workgroup calls it.
    __device__ __forceinline__ void run(const Operand& a, const Operand& b, long long m, long long n, int first, int k_steps, int pairs, char* lds) {
        HalfA ha;
        HalfB hb;
        ha.lanes(a, threadIdx.x >> 7);
        hb.lanes(b, (threadIdx.x >> 6) & 1);
        const int total = k_steps * pairs;
        int at_pair = 0, at_step = 0;            // of the step that is copied next
        auto enter = [&](int pair) {
            ha.start(a, plane_a(pair, pairs), m);
            hb.start(b, plane_b(pair, pairs), n);
            ha.base += ha.step * first; ha.left -= ha.step * first;
            hb.base += hb.step * first; hb.left -= hb.step * first;
        };
        auto moved_on = [&] {
            ha.advance();
            hb.advance();
            if (++at_step == k_steps && ++at_pair < pairs) { at_step = 0; enter(at_pair); }
        };
        enter(0);
#pragma unroll
        for (int q = 0; q < HalfA::kCopies; ++q) ha.copy(lds, q);
#pragma unroll
        for (int q = 0; q < HalfB::kCopies; ++q) hb.copy(lds + HalfA::kBytes, q);
        moved_on();
        wait_copies_and_sync<0>();
        if (total > 1) {
#pragma unroll
            for (int q = 0; q < HalfA::kCopies; ++q) ha.copy(lds + kBuffer, q);
#pragma unroll
            for (int q = 0; q < HalfB::kCopies; ++q) hb.copy(lds + kBuffer + HalfA::kBytes, q);
            moved_on();
        }
        v8bf fa[2][kM], fb[2][kN];
#pragma unroll
        for (int i = 0; i < kM; ++i) fa[0][i] = ha.frag(lds, i, 0);
#pragma unroll
        for (int j = 0; j < kN; ++j) fb[0][j] = hb.frag(lds + HalfA::kBytes, j, 0);
        int at = 0;                              // the buffer that is multiplied
        for (int t = 0; t < total; ++t) {
            char* here = lds + at;
            char* there = lds + (kBuffer - at);
#pragma unroll
            for (int s = 0; s < kStep / 16; ++s) {
                const int now = s & 1, next = now ^ 1;
                if (s + 1 < kStep / 16) {
#pragma unroll
                    for (int i = 0; i < kM; ++i) fa[next][i] = ha.frag(here, i, s + 1);
#pragma unroll
                    for (int j = 0; j < kN; ++j) fb[next][j] = hb.frag(here + HalfA::kBytes, j, s + 1);
                } else if (t + 1 < total) {
                    // every wave has what it needs of this buffer, and the next one is there
                    wait_copies_and_sync<0>();
                    if (t + 2 < total) {
#pragma unroll
                        for (int q = 0; q < HalfA::kCopies; ++q) ha.copy(here, q);
#pragma unroll
                        for (int q = 0; q < HalfB::kCopies; ++q) hb.copy(here + HalfA::kBytes, q);
                        moved_on();
                    }
#pragma unroll
                    for (int i = 0; i < kM; ++i) fa[next][i] = ha.frag(there, i, 0);
#pragma unroll
                    for (int j = 0; j < kN; ++j) fb[next][j] = hb.frag(there + HalfA::kBytes, j, 0);
                }
#pragma unroll
                for (int i = 0; i < kM; ++i)
#pragma unroll
                    for (int j = 0; j < kN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[now][i], fb[now][j], acc[i][j], 0, 0, 0);
            }
            at = kBuffer - at;
        }
    }
};

}  // namespace asi
