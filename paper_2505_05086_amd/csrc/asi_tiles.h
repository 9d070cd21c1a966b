// Products of bf16 matrices in tiles for the loss without logits (asi_head.hip): C[m][n] += sum_k A(m, k) B(n, k) with sums in fp32.
//
// A workgroup of 2 x WN waves has a tile of BM x BN; a step takes 64 k of both operands from memory into LDS without registers in
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
#include "asi_head_plan.h"
#include "asi_lm_device.h"

namespace asi {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4h __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// `rows` rows of `ld` elements, of which the first `cols` may be read; planes `plane` elements apart
struct Operand {
    const uint16_t* p;
    long long ld, plane;
    long long rows, cols;
};

// What a product of planes consists of: one pair; A (or B) in two planes, the smaller first; or the six pairs of three planes a side.
enum Pairs { kOne, kTwoA, kTwoB, kSix };
constexpr int pairs_of(int pairs) { return pairs == kOne ? 1 : pairs == kSix ? kPairs : 2; }
// Pair number i: which plane of either side.
template <int PAIRS> __device__ __forceinline__ int plane_a(int i) { return PAIRS == kSix ? (0x001012 >> (4 * i)) & 15 : PAIRS == kTwoA ? 1 - i : 0; }
template <int PAIRS> __device__ __forceinline__ int plane_b(int i) { return PAIRS == kSix ? (0x010210 >> (4 * i)) & 15 : PAIRS == kTwoB ? 1 - i : 0; }

// copy16_to_lds (asi_device.h) in a form whose end the compiler does not track: it takes any transposing LDS read for one of what the
// newest copies write, and would wait for them at once.  Here it is run() that waits, before the barrier that makes a buffer readable.
// The copy has no register for a result, and what it writes is read behind that wait only.
__device__ __forceinline__ void copy16_unwatched(const void* src, int bytes, int off, uint32_t lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    const uint64_t at = reinterpret_cast<uint64_t>(src);
    const u4 rsrc = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xffffu)),
                     (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00027000u};
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane((int)lds)) : "m0");
#endif
}
__device__ __forceinline__ uint32_t lds_address(const char* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

template <int N> struct Int {
    static constexpr int value = N;
};

// An operand's side of a tile: N rows (along k) or columns (across k) from `at` on, copied by WAVES waves, shared out to PARTS of them.
template <int N, bool ACROSS, int WAVES, int PARTS> struct Half {
    static constexpr int kBytes = N * kStep * 2;
    static constexpr int kCopies = kBytes / (WAVES * 1024);                // a wave's copies of 1 KB in a step
    static constexpr int kPieces = ACROSS ? N / 8 : kStep / 8;            // 16-byte pieces of a row in LDS
    static constexpr int kRowsACopy = 64 / kPieces;
    static constexpr int kBlocks = N / (32 * PARTS);                      // blocks of 32 that a wave has

    const char* base;          // of the tile's corner in the present plane, at the present k
    long long left;            // bytes from there to the operand's end
    const char* corner;        // of the tile, at the first k
    long long all;             // bytes from there to the end of a plane
    long long step, plane;     // bytes from a step's k to the next one's, and from plane to plane
    int off, odd, apart;       // a lane's piece of the first row, in even and odd copies; from a copy's rows to the next one's
    int read[ACROSS ? kBlocks : kStep / 16];      // a lane's place in LDS: for each block (across k), or each 16 k (along k)

    __device__ __forceinline__ void start(const Operand& o, long long at, int first) {
        const long long to = (ACROSS ? at : at * o.ld) * 2;
        step = ACROSS ? kStep * o.ld * 2 : kStep * 2;
        plane = o.plane * 2;
        corner = reinterpret_cast<const char*>(o.p) + to + first * step;
        all = ((o.rows - 1) * o.ld + o.cols) * 2 - to - first * step;
    }
    __device__ __forceinline__ void enter(int in_plane) {
        base = corner + in_plane * plane;
        left = all;
    }
    // on by a step, or, where that was a pair's last one, to the first of a pair whose plane is `planes` further
    __device__ __forceinline__ void move(bool last, int planes, int k_steps) {
        const long long by = last ? planes * plane - (k_steps - 1) * step : step;
        base += by;
        left = last ? all : left - step;
    }
    __device__ __forceinline__ void lanes(const Operand& o, int side) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int ld = (int)(o.ld * 2);
        const int row = kRowsACopy * wave * (ACROSS ? 1 : kCopies) + lane / kPieces, piece = lane % kPieces;
        // along k a copy has 8 rows, so that every second copy's pieces are exchanged by 4 more
        off = row * ld + (piece ^ (ACROSS ? 4 * (row & 3) : (row >> 1) & 7)) * 16;
        odd = row * ld + (piece ^ (ACROSS ? 4 * (row & 3) : ((row >> 1) & 7) ^ 4)) * 16;
        apart = kRowsACopy * (ACROSS ? WAVES : 1) * ld;
        if constexpr (ACROSS) {
            // 16 lanes read 4 rows of 16 columns, a row by 4 lanes, and get a column each
            const int in16 = lane & 15, k = (lane >> 5) * 8 + (in16 >> 2);
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) {
                const int piece_of = side * (N / (8 * PARTS)) + 4 * j + ((lane >> 4) & 1) * 2 + ((in16 & 3) >> 1);
                read[j] = k * (N * 2) + (piece_of ^ (4 * (k & 3))) * 16 + (in16 & 1) * 8;
            }
        } else {
#pragma unroll
            for (int s = 0; s < kStep / 16; ++s)
                read[s] = (side * (N / PARTS) + (lane & 31)) * (kStep * 2) + ((2 * s + (lane >> 5)) ^ ((lane >> 1) & 7)) * 16;
        }
    }
    // copy number q of this wave's
    __device__ __forceinline__ void copy(char* lds, int q) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int bytes = left > 0x7fffffffLL ? 0x7fffffff : left > 0 ? (int)left : 0;
        copy16_unwatched(base, bytes, ((q & 1) ? odd : off) + q * apart, lds_address(lds) + (ACROSS ? wave + WAVES * q : wave * kCopies + q) * 1024);
    }
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
template <int BM, int BN, bool A_ACROSS, bool B_ACROSS, int WN = 2> struct Tile {
    static constexpr int kThreads = 128 * WN, kM = BM / 64, kN = BN / (32 * WN);
    using HalfA = Half<BM, A_ACROSS, 2 * WN, 2>;
    using HalfB = Half<BN, B_ACROSS, 2 * WN, WN>;
    static constexpr int kBuffer = HalfA::kBytes + HalfB::kBytes;
    v16f acc[kM][kN];

    __device__ __forceinline__ static int wave_m() { return threadIdx.x / (64 * WN); }
    __device__ __forceinline__ static int wave_n() { return (threadIdx.x >> 6) % WN; }
    __device__ __forceinline__ static int at_m() { return wave_m() * (BM / 2); }
    __device__ __forceinline__ static int at_n() { return wave_n() * (BN / WN); }
    __device__ __forceinline__ static int row_of(int r) { return 8 * (r >> 2) + 4 * ((threadIdx.x >> 5) & 1) + (r & 3); }

    static constexpr int kFrags = kM * (A_ACROSS ? 2 : 1) + kN * (B_ACROSS ? 2 : 1);      // LDS reads of 16 k
    // The order of what the 16 k before it have: LDS reads and copies between the matrix instructions, each of which keeps its unit busy for
    // as long as eight other instructions take to issue.
    template <int READS, int COPIES, int I = 0> __device__ __forceinline__ static void interleave() {
        constexpr int n = kM * kN, reads = READS * (I + 1) / n - READS * I / n, copies = COPIES * (I + 1) / n - COPIES * I / n;
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
        if constexpr (copies > 0) __builtin_amdgcn_sched_group_barrier(0x010, copies, 0);
        if constexpr (I + 1 < n) interleave<READS, COPIES, I + 1>();
    }

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }

    // Adds the products of PAIRS' pairs of planes over k_steps steps, one at least, from k = 64 first on.  The whole workgroup
    // calls it.
    template <int PAIRS> __device__ __forceinline__ void run(const Operand& a, const Operand& b, long long m, long long n, int first, int k_steps, char* lds) {
        HalfA ha;
        HalfB hb;
        ha.lanes(a, wave_m());
        hb.lanes(b, wave_n());
        const int total = k_steps * pairs_of(PAIRS);
        ha.start(a, m, first);
        hb.start(b, n, first);
        int at_pair = 0, at_step = 0;            // of the step that is copied next
        // without a branch: a step of the loop below is one block, or its last LDS reads would be moved behind its end
        auto moved_on = [&] {
            if constexpr (PAIRS == kOne) {
                ha.move(false, 0, 0);
                hb.move(false, 0, 0);
            } else {
                const bool last = ++at_step == k_steps;
                const int next = at_pair + 1 < pairs_of(PAIRS) ? at_pair + 1 : at_pair;
                ha.move(last, plane_a<PAIRS>(next) - plane_a<PAIRS>(at_pair), k_steps);
                hb.move(last, plane_b<PAIRS>(next) - plane_b<PAIRS>(at_pair), k_steps);
                at_step = last ? 0 : at_step;
                at_pair = last ? next : at_pair;
            }
        };
        ha.enter(plane_a<PAIRS>(0));
        hb.enter(plane_b<PAIRS>(0));
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
        auto frags = [&](const char* from, int s, v8bf* x, v8bf* y) {
#pragma unroll
            for (int i = 0; i < kM; ++i) x[i] = ha.frag(from, i, s);
#pragma unroll
            for (int j = 0; j < kN; ++j) y[j] = hb.frag(from + HalfA::kBytes, j, s);
        };
        auto products = [&](const v8bf* x, const v8bf* y) {
#pragma unroll
            for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int j = 0; j < kN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y[j], acc[i][j], 0, 0, 0);
        };
        frags(lds, 0, fa[0], fb[0]);
        int at = 0;                              // the buffer that is multiplied
        // one step: `more` steps follow it, 2 standing for any more
        auto turn = [&](auto more) {
            constexpr int kMore = decltype(more)::value, kSteps = kStep / 16;
            char* here = lds + at;
            char* there = lds + (kBuffer - at);
#pragma unroll
            for (int s = 0; s + 1 < kSteps; ++s) {
                frags(here, s + 1, fa[(s + 1) & 1], fb[(s + 1) & 1]);
                products(fa[s & 1], fb[s & 1]);
                interleave<kFrags, 0>();
            }
            // every wave has what it needs of this buffer, and the next one is there
            if constexpr (kMore > 0) {
                wait_copies_and_sync<0>();
                frags(there, 0, fa[0], fb[0]);
            }
            constexpr int n = kM * kN, copies = HalfA::kCopies + HalfB::kCopies;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                acc[i / kN][i % kN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[1][i / kN], fb[1][i % kN], acc[i / kN][i % kN], 0, 0, 0);
                if constexpr (kMore > 1) {
#pragma unroll
                    for (int q = copies * i / n; q < copies * (i + 1) / n; ++q) {
                        if (q < HalfA::kCopies) ha.copy(here, q);
                        else hb.copy(here + HalfA::kBytes, q - HalfA::kCopies);
                    }
                }
            }
            if constexpr (kMore > 0) interleave<kFrags, 0>();
            at = kBuffer - at;
        };
        for (int t = 0; t + 2 < total; ++t) {
            turn(Int<2>());
            moved_on();
        }
        if (total > 1) turn(Int<1>());
        if (total > 0) turn(Int<0>());
    }
};

}  // namespace asi
