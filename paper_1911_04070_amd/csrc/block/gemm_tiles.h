// Tiles of a matrix product C[m][n] = sum_k A[m][k] B[k][n] on the matrix cores, for the feed-forward block: bf16 operands,
// fp32 sums.  A workgroup computes BM x BN of C in WR x WC wavefronts; both operands go through LDS in slabs of 32 to 128 k,
// two to four slabs deep, loaded straight into LDS (no registers in between).
//
// An operand lies in memory with either k or its own index (m or n) contiguous, and is kept that way in LDS:
//   k contiguous     [W][SLAB]  read 16 bytes per lane (8 k of one row)
//   index contiguous [SLAB][W]  read with the transposing LDS reads, which hand a lane 4 k of one column
// Either image is permuted within a row (16-byte pieces by the row's low bits, 32-byte pieces by the k's) so that the
// lanes of one read fall into different banks; direct loads write LDS in lane order, so the permutation is applied to
// the addresses they read from.
//
// Pieces outside the matrices (rows past m or n, k past K) are requested at an offset that the buffer descriptor's
// bound refuses, which reads as zero.
//
// Long sums run at what a large library product reaches on the same device (8192 x 4096 x 8192 of both: 1.22 and 1.20
// PFLOP/s); short ones pay for a tile's start and end, 4 us of a 256 x 256 tile's 18 at k = 512.
#pragma once

#include "row_device.h"

namespace bpt {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef short i16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) unsigned char* lds_bytes_t;

// 16 bytes per lane from the buffer `r` at byte offset `off` straight to LDS, lane after lane from `to` on.  Written out
// because the compiler waits for such a load before any LDS read behind it, whatever the two touch; who reads the slab waits
// with slab_barrier.  (M0 holds the LDS address; a wait state lies between its write and its use.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // (M0 as a clobber: it is the compiler's own, set right before each use)
__device__ __forceinline__ void load_to_lds(i32x4_t r, int off, lds_bytes_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"((int)(uintptr_t)to), "v"(off), "s"(r) : "memory", "m0");
}
#pragma clang diagnostic pop
// All but the last PENDING loads of this wavefront have arrived, its LDS reads are through, and so are those of the others
template <int PENDING>
__device__ __forceinline__ void slab_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(PENDING) : "memory");
}

constexpr int kBound = 0x7FFFFFF0;              // bytes an operand's descriptor covers from its tile's first element
constexpr int kOutside = (int)0x80000000;       // an offset behind it

// permutation of the 32-byte pieces of a row of W elements (index contiguous): the 4 k of a transposing read fall into
// different pairs of pieces
template <int W>
__device__ __forceinline__ int piece_swap(int k) {
    return W >= 128 ? 2 * (k & 3) : W == 64 ? (k & 3) : (k & 1);
}

// the same for the 16-byte pieces of a row of SLAB k (k contiguous): 16 neighbouring rows, read at once, fall into the 16
// different pieces of 256 bytes (the banks' width)
template <int SLAB>
__device__ __forceinline__ int row_swap(int row) {
    return SLAB == 128 ? (row & 15) : SLAB == 64 ? ((row >> 1) & 7) : ((row >> 2) & 3);
}

// Loads a slab of an operand of W rows (or columns) into LDS with WAVES wavefronts.
template <int W, int WAVES, bool KFIRST, int SLAB>   // KFIRST: k contiguous
struct SlabLoader {
    static constexpr int kBytes = W * SLAB * 2;
    static constexpr int kLoads = kBytes / 1024 / WAVES;   // 1 KB per wavefront and instruction
    static_assert(kLoads * 1024 * WAVES == kBytes, "the wavefronts share the slab evenly");
    int off[kLoads];

    // position of a lane's piece: its index within the W and its first k
    static __device__ __forceinline__ void place(int i, int wave, int lane, int& index, int& k) {
        const int q = (i * WAVES + wave) * 64 + lane;
        if (KFIRST) {
            constexpr int kPieces = SLAB / 8;
            index = q / kPieces;
            k = ((q % kPieces) ^ row_swap<SLAB>(index)) * 8;
        } else {
            constexpr int kPieces = W / 8;
            k = q / kPieces;
            const int p = q % kPieces;
            index = ((((p >> 1) ^ piece_swap<W>(k)) << 1) | (p & 1)) * 8;
        }
    }
    // ld: elements between rows as stored; valid: how many of the W indexes exist
    __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int64_t valid) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int index, k;
            place(i, wave, lane, index, k);
            const int at = KFIRST ? index * (int)ld + k : k * (int)ld + index;
            off[i] = index < valid ? at * 2 : kOutside;
        }
    }
    // p: the tile's first element of this slab; k_left: k that exist from there on
    __device__ __forceinline__ void load(const bf16_t* p, int64_t k_left, lds_bytes_t lds, int wave, int lane) const {
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        const i32x4_t r = {__builtin_amdgcn_readfirstlane((int)at), __builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xFFFF), kBound, 0x00020000};
        if (k_left >= SLAB) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load_to_lds(r, off[i], lds + (i * WAVES + wave) * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                int index, k;
                place(i, wave, lane, index, k);
                load_to_lds(r, k < k_left ? off[i] : kOutside, lds + (i * WAVES + wave) * 1024);
            }
        }
    }
};

// Operand of v_mfma_f32_32x32x16_bf16: lane l holds k = 16 kk + 8 (l / 32) .. + 7 of index first + l % 32.
template <int W, bool KFIRST, int SLAB>
__device__ __forceinline__ bf16x8_t fragment(lds_bytes_t slab, int first, int kk, int lane) {
    if constexpr (KFIRST) {
        typedef __attribute__((address_space(3))) const bf16x8_t* ptr_t;
        return *(ptr_t)(slab + (first + (lane & 31)) * (SLAB * 2) + (((kk * 2 + (lane >> 5)) ^ row_swap<SLAB>(lane & 31)) * 16));
    } else {
        typedef __attribute__((address_space(3))) i16x4_t* ptr_t;
        const int k = kk * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
        const int piece = ((first >> 4) + ((lane >> 4) & 1)) ^ piece_swap<W>((lane & 15) >> 2);
        lds_bytes_t p = slab + k * (W * 2) + piece * 32 + (lane & 3) * 8;
        const i16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr_t)p);
        const i16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr_t)(p + 4 * W * 2));
        const i16x8_t xy = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        return __builtin_bit_cast(bf16x8_t, xy);
    }
}

// One operand pair of a tile.  PAIR: B is two matrices of BN / 2 columns each, whose slabs lie one behind the other; a
// wavefront then computes the same columns of both (the first half of its column blocks are of the first).
template <int BM, int BN, int WR, int WC, int SLAB, int STAGES, bool A_KFIRST, bool B_KFIRST, bool PAIR>
struct Tile {
    static constexpr int kSlab = SLAB;                         // k per slab
    static constexpr int kWaves = WR * WC, kThreads = 64 * kWaves;
    static constexpr int kRows = BM / WR / 32;                 // 32-row blocks of a wavefront
    static constexpr int kCols = BN / WC / 32;                 // 32-column blocks
    static constexpr int kBlocks = kRows * kCols;
    static constexpr int kBM = BM, kBN = BN;
    static constexpr int kBWidth = PAIR ? BN / 2 : BN;
    using LoadA = SlabLoader<BM, kWaves, A_KFIRST, SLAB>;
    using LoadB = SlabLoader<kBWidth, kWaves, B_KFIRST, SLAB>;
    static constexpr int kStage = LoadA::kBytes + LoadB::kBytes * (PAIR ? 2 : 1);
    static constexpr int kLds = STAGES * kStage;
    static constexpr int kWavesPerSimd = kWaves == 8 || 2 * kLds <= 160 * 1024 ? 2 : 1;
    static_assert(STAGES >= 2 && STAGES <= 4, "run() has waits for these");
    static constexpr int kPending = (LoadA::kLoads + LoadB::kLoads * (PAIR ? 2 : 1));   // loads of a slab, per wavefront
    typedef f32x16_t Acc[kRows][kCols];

    LoadA la;
    LoadB lb;
    lds_bytes_t lds;
    int wave, lane, wr, wc;

    __device__ __forceinline__ void init(unsigned char* shared, int64_t lda, int64_t rows_valid, int64_t ldb, int64_t cols_valid) {
        place(shared);
        la.init(wave, lane, lda, rows_valid);
        lb.init(wave, lane, ldb, cols_valid);
    }
    __device__ __forceinline__ void place(unsigned char* shared) {
        lds = (lds_bytes_t)shared;
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wr = wave / WC;
        wc = wave % WC;
    }
    // first column, within the tile's BN (PAIR: within either half), of a column block of this wavefront
    __device__ __forceinline__ int col_of(int j) const {
        if constexpr (PAIR) return (wc * (kCols / 2) + j % (kCols / 2)) * 32;
        return (wc * kCols + j) * 32;
    }
    __device__ __forceinline__ int row_of(int i) const { return (wr * kRows + i) * 32; }

    __device__ __forceinline__ void load(const bf16_t* a, const bf16_t* b0, const bf16_t* b1, int64_t k_left, int stage) const {
        lds_bytes_t p = lds + stage * kStage;
        la.load(a, k_left, p, wave, lane);
        lb.load(b0, k_left, p + LoadA::kBytes, wave, lane);
        if (PAIR) lb.load(b1, k_left, p + LoadA::kBytes + LoadB::kBytes, wave, lane);
    }
    __device__ __forceinline__ void read(bf16x8_t (&a)[kRows], bf16x8_t (&b)[kCols], lds_bytes_t pa, int kk) const {
        lds_bytes_t pb = pa + LoadA::kBytes;
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            lds_bytes_t p = PAIR && j >= kCols / 2 ? pb + LoadB::kBytes : pb;
            b[j] = fragment<kBWidth, B_KFIRST, SLAB>(p, col_of(j), kk, lane);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) a[i] = fragment<BM, A_KFIRST, SLAB>(pa, row_of(i), kk, lane);
    }
    // The operands of the next 16 k are read while the matrix instructions of these run.  (For 8 wavefronts that order is
    // enforced: 65 532 x 512 x 4096, 263 -> 255 us; for 4 the compiler's own is as good or better.)
    __device__ __forceinline__ void multiply(Acc& acc, int stage) const {
        lds_bytes_t pa = lds + stage * kStage;
        bf16x8_t a[2][kRows], b[2][kCols];
        read(a[0], b[0], pa, 0);
#pragma unroll
        for (int kk = 0; kk < kSlab / 16; ++kk) {
            if (kk + 1 < kSlab / 16) read(a[(kk + 1) & 1], b[(kk + 1) & 1], pa, kk + 1);
            if constexpr (kWaves == 8) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kRows; ++i)
#pragma unroll
                for (int j = 0; j < kCols; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[kk & 1][j], a[kk & 1][i], acc[i][j], 0, 0, 0);
            if constexpr (kWaves == 8) __builtin_amdgcn_sched_barrier(0);
        }
    }
    // Sum over `slabs` slabs; from(t, a, b0, b1, k_left) says where slab t lies.  All threads call it; on return the
    // slabs' memory is free.  STAGES - 1 slabs are on their way while one is worked on, one barrier per slab.
    template <typename From>
    __device__ __forceinline__ void run(Acc& acc, int slabs, From from) const {
        const bf16_t *a, *b0, *b1 = nullptr;
        int64_t k_left;
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t)
            if (t < slabs) {
                from(t, a, b0, b1, k_left);
                load(a, b0, b1, k_left, t);
            }
        int stage = 0, next = STAGES - 1;
        for (int t = 0; t < slabs; ++t) {
            const int behind = min(STAGES - 2, slabs - 1 - t);   // slabs that may still be on their way
            if (STAGES > 3 && behind == 2) slab_barrier<(STAGES > 3 ? 2 : 0) * kPending>();
            else if (STAGES > 2 && behind == 1) slab_barrier<(STAGES > 2 ? 1 : 0) * kPending>();
            else slab_barrier<0>();
            if (t + STAGES - 1 < slabs) {
                from(t + STAGES - 1, a, b0, b1, k_left);
                load(a, b0, b1, k_left, next);
            }
            multiply(acc, stage);
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            next = next + 1 == STAGES ? 0 : next + 1;
        }
        slab_barrier<0>();
    }
};
// For few rows: 32 x 32 of C in a workgroup, whose WAVES wavefronts each take a part of k with slabs, loads and waits of their own,
// so that all of them keep loads of the weights in flight; their sums meet in LDS at the end.  A and B as in a Tile with k
// contiguous in A and n in B.  BS = 2: of two products A B[0], A B[1]; AS = 2: of (A[0] + A[1]) B, A in two parts.
template <int WAVES, int STAGES, int AS, int BS>
struct Strip {
    static constexpr int kSlab = 32, kThreads = 64 * WAVES;
    using LoadA = SlabLoader<32, 1, true, kSlab>;
    using LoadB = SlabLoader<32, 1, false, kSlab>;
    static constexpr int kStage = AS * LoadA::kBytes + BS * LoadB::kBytes;
    static constexpr int kPending = AS * LoadA::kLoads + BS * LoadB::kLoads;
    static constexpr int kLds = WAVES * STAGES * kStage;
    static_assert((STAGES == 3 || STAGES == 4) && WAVES >= 4 && kLds >= WAVES * BS * 4096 && kLds <= 160 * 1024,
                  "waits and the final sums are written for these");

    // On return wavefront w < 4 holds in sum[mat] C[lane % 32][8 w + 4 (lane / 32) ..+ 3].  a: first row's k = 0; b: first column's.
    static __device__ __forceinline__ void run(unsigned char* shared, int wave, int lane, const bf16_t* const* a, int64_t lda, int64_t rows,
                                               const bf16_t* const* b, int64_t ldb, int cols, int k_all, float4* sum) {
        lds_bytes_t all = (lds_bytes_t)shared, mine = all + wave * STAGES * kStage;
        LoadA la;
        LoadB lb;
        la.init(0, lane, lda, rows);
        lb.init(0, lane, ldb, cols);
        const int slabs = (k_all + kSlab - 1) / kSlab, each = (slabs + WAVES - 1) / WAVES;
        const int count = max(min(each, slabs - wave * each), 0), k0 = wave * each * kSlab;
        auto load = [&](int t, int stage) {
            const int k = k0 + t * kSlab;
            lds_bytes_t p = mine + stage * kStage;
#pragma unroll
            for (int m = 0; m < AS; ++m) la.load(a[m] + k, k_all - k, p + m * LoadA::kBytes, 0, lane);
#pragma unroll
            for (int m = 0; m < BS; ++m) lb.load(b[m] + (int64_t)k * ldb, k_all - k, p + AS * LoadA::kBytes + m * LoadB::kBytes, 0, lane);
        };
        f32x16_t acc[BS] = {};
#pragma unroll
        for (int t = 0; t < STAGES - 1; ++t)
            if (t < count) load(t, t);
        int stage = 0, next = STAGES - 1;
        for (int t = 0; t < count; ++t) {
            // this slab has arrived (those behind it may be on their way), and the reads of the one before are through
            const int behind = min(STAGES - 2, count - 1 - t);
            if (STAGES > 3 && behind == 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(2 * kPending) : "memory");
            else if (behind == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kPending) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            if (t + STAGES - 1 < count) load(t + STAGES - 1, next);
            lds_bytes_t pa = mine + stage * kStage, pb = pa + AS * LoadA::kBytes;
#pragma unroll
            for (int kk = 0; kk < kSlab / 16; ++kk) {
                bf16x8_t x[AS], y[BS];
#pragma unroll
                for (int m = 0; m < AS; ++m) x[m] = fragment<32, true, kSlab>(pa + m * LoadA::kBytes, 0, kk, lane);
#pragma unroll
                for (int m = 0; m < BS; ++m) y[m] = fragment<32, false, kSlab>(pb + m * LoadB::kBytes, 0, kk, lane);
#pragma unroll
                for (int u = 0; u < AS; ++u)
#pragma unroll
                    for (int m = 0; m < BS; ++m) acc[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[m], x[u], acc[m], 0, 0, 0);
            }
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            next = next + 1 == STAGES ? 0 : next + 1;
        }
        slab_barrier<0>();   // (the sums take the slabs' place)
        typedef __attribute__((address_space(3))) f32x4_t* ptr_t;
#pragma unroll
        for (int m = 0; m < BS; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4_t v = {acc[m][4 * q], acc[m][4 * q + 1], acc[m][4 * q + 2], acc[m][4 * q + 3]};
                *(ptr_t)(all + ((wave * BS + m) * 4 + q) * 1024 + lane * 16) = v;
            }
        __syncthreads();
        if (wave < 4)
#pragma unroll
            for (int m = 0; m < BS; ++m) {
                f32x4_t v = {};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v += *(ptr_t)(all + ((w * BS + m) * 4 + wave) * 1024 + lane * 16);
                sum[m] = make_float4(v[0], v[1], v[2], v[3]);
            }
    }
};

// Rounds 32 rows of a wavefront's COLS columns to bf16 and writes them, through LDS of its own, in 16-byte pieces along the
// rows (from the accumulators' order a store would touch 32 rows for 16 bytes each).  A wavefront's LDS accesses are in
// order, so nothing is waited for between blocks of rows.
template <int COLS>
struct RowBlock {
    static constexpr int kPitch = COLS * 2 + 16, kBytes = 32 * kPitch;
    lds_bytes_t lds;
    int lane;
    __device__ __forceinline__ RowBlock(lds_bytes_t all, int wave, int lane_) : lds(all + wave * kBytes), lane(lane_) {}
    // four neighbours of row lane % 32: columns col + 4 (lane / 32) ..
    __device__ __forceinline__ void put(int col, float a, float b, float c, float d) const {
        typedef __attribute__((address_space(3))) i32x2_t* ptr_t;
        const i32x2_t v = {(int)bf16_pair(a, b), (int)bf16_pair(c, d)};
        *(ptr_t)(lds + (lane & 31) * kPitch + (col + 4 * (lane >> 5)) * 2) = v;
    }
    // out: the block's first element; rows, cols: how many of them exist
    __device__ __forceinline__ void write(bf16_t* out, int64_t ld, int64_t rows, int cols) const {
        typedef __attribute__((address_space(3))) const i32x4_t* ptr_t;
        constexpr int kPieces = COLS / 8, kRows = 64 / kPieces;
        const int r = lane / kPieces, c = lane % kPieces * 8;
        const uint32_t at = (uint32_t)(r * (int)ld + c) * 2;   // (the rest of the address is the wavefront's)
        const int last = c < cols ? (int)min((int64_t)32, rows) - r : 0;
#pragma unroll
        for (int i = 0; i < 32; i += kRows) {
            const i32x4_t v = *(ptr_t)(lds + (i + r) * kPitch + c * 2);
            if (i < last) *reinterpret_cast<i32x4_t*>(reinterpret_cast<unsigned char*>(out + i * ld) + at) = v;
        }
    }
};

// acc[i][j] register r of lane l is C[row_of(i) + l % 32][col_of(j) + 8 (r / 4) + 4 (l / 32) + r % 4]: the matrix
// instruction is given B as its first operand, so that a lane holds four neighbours of a row of C.

}  // namespace
}  // namespace bpt
