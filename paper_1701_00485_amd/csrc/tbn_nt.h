// tbn_nt.h -- the inner loop that products of two row-major operands share: C[m][n] = sum over k of A[m][k] B[n][k],
// both operands' rows contiguous along k, for 8-bit integers and for 32-bit values held as two 16-bit halves.
//
//   * A stage is 128 bytes of every row of the tile, whatever the type: 128 8-bit values, or 32 values as 32 leading
//     and 32 trailing halves.  It goes from memory into LDS by buffer loads in LDS-DMA mode, 16-byte segments
//     XOR-swizzled by (row / 2) % 8 on the way, so that the operand reads meet no bank twice.
//   * Rows past the operand's end lie outside its buffer resource and arrive as zeros; so do segments past the end of A's
//     row, and then it does not matter what B holds there.
//   * Of a block's waves each owns (BM / WAVES_M) x (BN / WAVES_N) outputs.  The second operand goes first into the matrix
//     instruction, so that lane l of 32x32 tile (i, t) holds row 32 i + l % 32 and, for each v / 4, the four consecutive
//     columns 32 t + 8 (v / 4) + 4 (l / 32) + 0..3.
//   * Operands of a step are read from LDS while the matrix instructions of the step before run, those of a stage's first step too: the
//     barrier between two stages lies before the last step of the earlier one, whose operands are in registers by then.
#pragma once

#include "tbn_device.h"
#include "tbn_dma.h"

namespace tbn {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
// 16 bytes that begin at any 16-bit value, at any 32-bit value: rows of odd lengths are read and written as wide as others, as
// global memory takes such addresses (8-bit products 4000 x 4096 x 4097: 91 us, a value at a time 107).
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef f32x4 f32x4_at4 __attribute__((aligned(4)));

// 8-bit integers: four steps of 32 a stage, exact 32-bit sums.
struct NtI8 {
    typedef i32x16 Acc;
    static constexpr int STEPS = 4, PARTS = 1, PRODUCTS = 1;
    static __device__ __forceinline__ int seg(int u, int, int half) { return 2 * u + half; }
    static constexpr __device__ int part_a(int) { return 0; }
    static constexpr __device__ int part_b(int) { return 0; }
    static __device__ __forceinline__ i32x16 mul(u32x4 b, u32x4 a, i32x16 c) {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, b), __builtin_bit_cast(i32x4, a), c, 0, 0, 0);
    }
};

// 32-bit values x = hi + lo in two fp16 halves (22 bits of x): two steps of 16 a stage, three products each (hi lo, lo hi, hi hi); lo lo,
// 2^-22 of the product, is left out.
struct NtF16x2 {
    typedef f32x16 Acc;
    static constexpr int STEPS = 2, PARTS = 2, PRODUCTS = 3;
    static __device__ __forceinline__ int seg(int u, int part, int half) { return 4 * part + 2 * u + half; }
    static constexpr __device__ int part_a(int p) { return p == 1; }
    static constexpr __device__ int part_b(int p) { return p == 0; }
    static __device__ __forceinline__ f32x16 mul(u32x4 b, u32x4 a, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
    }
};

// The rows of an operand that a block's waves copy: row 8 (wave + WAVES j) + lane / 8 of the tile is this lane's of copy j.
template <int ROWS, int WAVES>
struct NtRows {
    static constexpr int COPIES = ROWS / 8 / WAVES;
    static_assert(ROWS % (8 * WAVES) == 0 && WAVES % 2 == 0, "whole copies");
    v4i rsrc;
    uint32_t off[COPIES];
    // `row0` < rows; ROWS * pitch < 2^31 and pitch % 16 == 0 (checked by the host)
    __device__ __forceinline__ void init(const void* p, int64_t row0, int64_t rows, uint32_t pitch, int wave, int lane, int seg) {
        const int64_t left = rows - row0 < ROWS ? rows - row0 : ROWS;
        rsrc = make_rsrc(reinterpret_cast<const uint8_t*>(p) + row0 * pitch, (uint32_t)(left * pitch));
#pragma unroll
        for (int j = 0; j < COPIES; ++j) off[j] = (uint32_t)(8 * (wave + WAVES * j) + (lane >> 3)) * pitch + 16u * seg;
    }
    // copy j of the stage at byte `at` of the rows (bit 31 set in lanes whose segment is past the row's end)
    __device__ __forceinline__ void issue(int j, uint32_t lds, uint32_t at, int wave) const {
        dma_b128(rsrc, lds + (uint32_t)(8 * (wave + WAVES * j)) * 128u, off[j] + at);
    }
};

template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, class Op>
struct NtLoop {
    static constexpr int WAVES = WAVES_M * WAVES_N;
    static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 32, TN = WN / 32;
    static constexpr int STAGE = (BM + BN) * 128, BYTES = STAGES * STAGE;
    typedef typename Op::Acc Acc;
    typedef NtRows<BM, WAVES> RowsA;
    typedef NtRows<BN, WAVES> RowsB;
    static constexpr int COPIES = RowsA::COPIES + RowsB::COPIES;

    // Logical 16-byte segment that a lane copies of its row.
    static __device__ __forceinline__ int copy_seg(int wave, int lane) { return (lane & 7) ^ ((4 * (wave & 1)) | ((lane >> 4) & 3)); }

    // Adds the products of stages s0 .. s1 - 1 to acc.  `row_bytes`: of A's rows.  Every wave of the block calls it, with the same
    // `rounds` (of barriers), at least s1 - s0; it ends behind a barrier, after which the LDS is free.
    static __device__ __forceinline__ void run(const RowsA& ra, const RowsB& rb, uint8_t* smem, int s0, int s1, int rounds, uint32_t row_bytes,
                                               int wave, int lane, Acc (&acc)[TM][TN]) {
        const int wm = wave / WAVES_N, wn = wave % WAVES_N;
        const int half = lane >> 5, l32 = lane & 31;
        const int sw = (l32 >> 1) & 7;
        const uint32_t base = lds_addr(smem);
        const uint32_t my = 16u * copy_seg(wave, lane);
        const int n = s1 - s0;
        int islot = 0;
        uint32_t copy_lds = 0, copy_at = 0, copy_at_a = 0;  // of the stage whose copies are issued
        auto aim = [&](int s) {
            copy_lds = base + (uint32_t)(islot * STAGE);
            // past the last stage nothing is read and zeros are written, so that every stage issues and waits for the same copies
            copy_at = (uint32_t)(s0 + s) * 128u | (s < n ? 0u : 0x80000000u);
            copy_at_a = copy_at + my < row_bytes ? copy_at : copy_at | 0x80000000u;
            islot = islot + 1 == STAGES ? 0 : islot + 1;
        };
        auto copy = [&](int j) {
            if (j < RowsA::COPIES)
                ra.issue(j, copy_lds, copy_at_a, wave);
            else
                rb.issue(j - RowsA::COPIES, copy_lds + BM * 128, copy_at, wave);
        };
        const int arow = (wm * WM + l32) * 128, brow = (wn * WN + l32) * 128 + BM * 128;
        u32x4 a[2][Op::PARTS][TM], b[2][Op::PARTS][TN];
        constexpr int READS = Op::PARTS * (TM + TN), MUL = TM * TN * Op::PRODUCTS;
        auto read = [&](const uint8_t* st, int u, int r) {  // operand r of step u
            const int p = r / (TM + TN), i = r % (TM + TN), so = 16 * (Op::seg(u, p, half) ^ sw);
            if (i < TN)
                b[u & 1][p][i] = *reinterpret_cast<const u32x4*>(st + brow + 32 * 128 * i + so);
            else
                a[u & 1][p][i - TN] = *reinterpret_cast<const u32x4*>(st + arow + 32 * 128 * (i - TN) + so);
        };
        auto multiply = [&](int u, int k) {  // instruction k of step u
            const int p = k / (TM * TN), i = k / TN % TM, t = k % TN;
            acc[i][t] = Op::mul(b[u & 1][Op::part_b(p)][t], a[u & 1][Op::part_a(p)][i], acc[i][t]);
        };
        // Step u, while the operands of step v of the stage at `st` are read and, in a stage's last step, copies issued: each between two
        // instructions where a step has many (256 x 256 tiles of four waves 4096 x 8192 x 4096: 620 us, in a row 690), in a row where
        // it has few (64 x 64 tiles 512 x 512 x 512: 7.6 us, between them 8.3).
        auto step = [&](int u, const uint8_t* st, int v, bool copies) {
            constexpr bool MANY = MUL >= 12;
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!MANY) {
#pragma unroll
                for (int r = 0; r < READS; ++r) read(st, v, r);
            }
#pragma unroll
            for (int k = 0; k < MUL; ++k) {
                multiply(u, k);
                if constexpr (MANY) {
#pragma unroll
                    for (int r = k * READS / MUL; r < (k + 1) * READS / MUL; ++r) read(st, v, r);
#pragma unroll
                    for (int j = k * COPIES / MUL; j < (k + 1) * COPIES / MUL; ++j)
                        if (copies) copy(j);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (!MANY) {
#pragma unroll
                for (int j = 0; j < COPIES; ++j)
                    if (copies) copy(j);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        constexpr int LAST = Op::STEPS - 1;
        static_assert(LAST & 1, "a stage begins with the first operand registers");

#pragma unroll
        for (int s = 0; s < STAGES; ++s) {
            aim(s);
#pragma unroll
            for (int j = 0; j < COPIES; ++j) copy(j);
        }
        wait_vmcnt((STAGES - 1) * COPIES);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < READS; ++r) read(smem, 0, r);
        pin(acc);
        int slot = 0;
        for (int s = 0; s < rounds; ++s) {
            const uint8_t* st = smem + slot * STAGE;
            slot = slot + 1 == STAGES ? 0 : slot + 1;
            if (s < n) {
#pragma unroll
                for (int u = 0; u < LAST; ++u) {
                    step(u, st, u + 1, false);
                }
            }
            // this wave's copies of the next stage have landed, its reads of this one are done, and so are the other waves'
            wait_vmcnt((STAGES - 2) * COPIES);
            __syncthreads();
            if (s >= n) continue;
            const uint8_t* next = smem + slot * STAGE;
            aim(s + STAGES);  // into this stage's place
            step(LAST, next, 0, true);
        }
        pin(acc);
        wait_vmcnt(0);
        __syncthreads();
    }

    // 256 sums a lane stay in accumulation registers throughout (else the compiler moves a third of them at every step).
    static __device__ __forceinline__ void pin(Acc (&acc)[TM][TN]) {
        if constexpr (TM * TN >= 16) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int t = 0; t < TN; ++t) asm volatile("" : "+a"(acc[i][t]));
        }
    }
};

// A block of GROUPS groups of waves, each with a part of the stages and an LDS ring of its own, for tiles that are too few to fill the
// GPU: the first group's sums plus the others', in order.  Each group brings at most BYTES of LDS; ends behind a barrier.
template <int GROUPS, class Loop>
__device__ __forceinline__ void nt_join(uint8_t* smem, int group, int wave, int lane, typename Loop::Acc (&acc)[Loop::TM][Loop::TN]) {
    if constexpr (GROUPS > 1) {
        constexpr int QUADS = Loop::TM * Loop::TN * 4;
        static_assert((GROUPS - 1) * QUADS * 16 * 64 * Loop::WAVES <= GROUPS * Loop::BYTES, "sums fit in the rings");
        typedef typename Loop::Acc Acc;
        typedef decltype(Acc{}[0] + Acc{}[0]) T;
        typedef T Quad __attribute__((ext_vector_type(4)));
        Quad* const at = reinterpret_cast<Quad*>(smem) + wave * 64 + lane;
        if (group) {
#pragma unroll
            for (int i = 0; i < Loop::TM; ++i)
#pragma unroll
                for (int t = 0; t < Loop::TN; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        at[(((group - 1) * Loop::TM + i) * Loop::TN * 4 + t * 4 + g) * Loop::WAVES * 64] =
                            Quad{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
        }
        __syncthreads();
        if (!group) {
#pragma unroll
            for (int k = 0; k < GROUPS - 1; ++k)
#pragma unroll
                for (int i = 0; i < Loop::TM; ++i)
#pragma unroll
                    for (int t = 0; t < Loop::TN; ++t)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const Quad v = at[((k * Loop::TM + i) * Loop::TN * 4 + t * 4 + g) * Loop::WAVES * 64];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][t][4 * g + e] += v[e];
                        }
        }
        __syncthreads();
    }
}

// Tile (m, n) of the work index w: bands of 8 tile rows, so that the blocks that an XCD runs side by side share rows of
// both operands in its L2.
__device__ __forceinline__ void nt_tile(uint32_t w, uint32_t tiles_m, uint32_t tiles_n, uint32_t* m, uint32_t* n) {
    constexpr uint32_t BAND = 8;
    const uint32_t band = w / (BAND * tiles_n), first = band * BAND;
    const uint32_t rows = tiles_m - first < BAND ? tiles_m - first : BAND;
    const uint32_t in = w - first * tiles_n;
    *n = in / rows;
    *m = first + (in - *n * rows);
}

}  // namespace tbn
