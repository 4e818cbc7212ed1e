// tbn_muon.hip -- Muon's step on the real weights: momentum, the update made orthogonal by Newton-Schulz products, and the
// weights moved along it, for many matrices in the launches of one.
//
// With X the update over its Frobenius norm, m x n, m <= n (a taller matrix is taken transposed), each step is
//   A = X X^T,  P = a I + b A + c A A,  X = P X,   (a, b, c) = (3.4445, -4.7750, 2.0315),
// which moves every singular value s to a s + b s^3 + c s^5 and, five times, into the neighbourhood of 1.
//
//   * Two steps share one product with X on either side: the next A is P A P, as P and A are polynomials of the same
//     matrix, and X is multiplied once, by the product of the two P.  Five steps as two, two and one take, in products of m^3
//     (a symmetric one is half a product of m x m x m), 9 n / m + 11 against 15 n / m + 5.  What rounding put into A grows by a^2
//     in the second step, where singular values are small: against 64 bits the result is as far off as that of elementary
//     fp32 products, or twice as far (random, low-rank and decaying spectra).  Three steps at once would be ten times.
//   * Every factor is held as two fp16 halves (22 bits) and multiplied on the matrix cores with three products (tbn_nt.h), at a
//     third of the matrix rate; sums are fp32.  One fp16 or bf16 product in place of the three would leave 2^-9 to 2^-12 of X,
//     which small singular values carry through five steps that each multiply them by 3.4.  The halves are scaled by powers of
//     two so that both keep their bits and none overflows: X by 2^12 (|X| <= 1.21), A by 2^14 (1.47), P and P A by 2^13 (3.45),
//     a product of two P by 2^12 (11.9).
//   * Rows are groups of 32 values, 64 bytes of leading and 64 of trailing halves, zeros behind the last: the 128 bytes of
//     a stage.
//   * A, P and their products are symmetric: tiles on and below the diagonal are computed and written to both places.
//   * What a launch has to do for which matrix stands in tables in the workspace, written there by a launch of their own: read
//     from kernel arguments, in host memory, they cost each of 17 launches up to 15 us for 21 matrices.
//   * P X needs the rows of X^T: every X is written in both layouts, by the epilogue that has the tile in LDS anyway.
#include <algorithm>
#include <cmath>

#include "tbn_kernels.h"
#include "tbn_nt.h"

namespace tbn {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kXScale = 0x1p12f;

// Eight values at byte `p` (64 bytes before their trailing halves).
__device__ __forceinline__ void put8(uint8_t* p, const float (&v)[8]) {
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        hi[e] = (_Float16)v[e];
        lo[e] = (_Float16)(v[e] - (float)hi[e]);
    }
    *reinterpret_cast<f16x8*>(p) = hi;
    *reinterpret_cast<f16x8*>(p + 64) = lo;
}
// ... the leading halves alone, or the trailing.
__device__ __forceinline__ void put_half8(uint8_t* p, const float (&v)[8], bool trailing) {
    f16x8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const _Float16 hi = (_Float16)v[e];
        h[e] = trailing ? (_Float16)(v[e] - (float)hi) : hi;
    }
    *reinterpret_cast<f16x8*>(p + (trailing ? 64 : 0)) = h;
}
__device__ __forceinline__ void get8(const uint8_t* p, float (&v)[8]) {
    const f16x8 hi = *reinterpret_cast<const f16x8*>(p), lo = *reinterpret_cast<const f16x8*>(p + 64);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)hi[e] + (float)lo[e];
}
// Byte of value c (a multiple of 8) in a row.
__device__ __forceinline__ int64_t place(int64_t c) { return c / 32 * 128 + c % 32 * 2; }

// ---- tables ------------------------------------------------------------------------------
static_assert(kMuonMatrices <= 64, "a lane finds a matrix");

// A matrix: m <= n, transposed if `tall`; its arrays in the workspace.
struct Matrix {
    float* w;
    float* mom;
    const void* g;
    uint8_t *x[2], *xt[2], *a, *t, *p[3];
    double* norm;          // partial sums of squares, `parts` of them
    int32_t m, n;
    uint32_t mp, np;       // bytes of a row of m (n) values
    uint32_t parts, tall;
    float weight_decay, scale;
};

// What the launches are: A = X X^T; P of A; P A; P A P; the product of both P; P X.
enum Kind { GRAM, POLY, TIMES, BOTH, PAIR, APPLY };
struct Step {
    int32_t kind;
    int32_t second;  // of a chain's two steps
    int32_t two;     // APPLY: by the product of two P
    int32_t now;     // which X
    int32_t last;    // APPLY: into w
};

// v = p (a b^T) + q aux + diag on the diagonal
struct Job {
    const uint8_t* a;    // rows of M and of N, `pitch` bytes each
    const uint8_t* b;
    const uint8_t* aux;  // rows of pitch_o bytes, or null
    uint8_t* direct;     // v by rows, or null
    uint8_t* turned;     // v by columns, or null
    uint32_t pitch, pitch_o, pitch_t;
    int32_t M, N;
    bool symmetric, to_w;
    float p, q, diag;
};

// Scales of the halves: X 2^12, A 2^14, P and P A 2^13, a product of two P 2^12.  `x`: a Matrix, here or in constant memory.
template <typename X>
__host__ __device__ __forceinline__ Job job_of(X x, const Step& s) {
    const int kind = s.kind;
    const bool apply = kind == APPLY, poly = kind == POLY, gram = kind == GRAM;
    const bool turn = apply && s.last && x->tall;  // along the rows of w
    const uint8_t* const p = s.second ? x->p[1] : x->p[0];
    const uint8_t *const by = s.two ? x->p[2] : x->p[0], *const xt = s.now ? x->xt[1] : x->xt[0];
    uint8_t* const to = gram || kind == BOTH ? x->a : kind == TIMES ? x->t : kind == PAIR ? x->p[2] : s.second ? x->p[1] : x->p[0];
    Job j;
    j.a = gram ? (s.now ? x->x[1] : x->x[0]) : poly ? x->a : !apply ? p : turn ? xt : by;
    j.b = gram ? (s.now ? x->x[1] : x->x[0]) : poly || kind == TIMES ? x->a : kind == BOTH ? x->t : kind == PAIR ? x->p[0] : turn ? by : xt;
    j.aux = poly ? x->a : nullptr;
    j.direct = !apply ? to : s.last ? nullptr : s.now ? x->x[0] : x->x[1];
    j.turned = !apply ? to : s.last ? nullptr : s.now ? x->xt[0] : x->xt[1];
    j.pitch = gram ? x->np : x->mp;
    j.pitch_o = apply ? x->np : x->mp;
    j.pitch_t = x->mp;
    j.M = turn ? x->n : x->m;
    j.N = apply && !turn ? x->n : x->m;
    j.symmetric = !apply;
    j.to_w = apply && s.last;
    j.p = gram ? 0x1p-10f : poly ? kC * 0x1p-15f : kind == BOTH ? 0x1p-12f : apply ? (s.two ? 0x1p-12f : 0x1p-13f) : 0x1p-14f;
    j.q = poly ? kB * 0x1p-1f : 0.0f;
    j.diag = poly ? kA * 0x1p13f : 0.0f;
    return j;
}

// The matrices, and for every launch the first blocks (tiles) of each and its first divided stages.
struct Table {
    const uint32_t* first;    // round_up(n, 8) words
    const uint32_t* divided;  // ... behind them
    const Matrix* matrix;
    int32_t n;
};
// What no kernel that reads it writes: scalar loads.
template <typename T>
__device__ __forceinline__ const __attribute__((address_space(4))) T* constant(const T* p) {
    return (const __attribute__((address_space(4))) T*)(uintptr_t)p;
}
// The matrix that `at` falls to.
__device__ __forceinline__ int find(const uint32_t* first, int n, uint32_t at) {
    const int lane = threadIdx.x & 63;
    const uint32_t f = lane < n ? first[lane] : 0xFFFFFFFFu;
    return __popcll(__ballot(f <= at)) - 1;
}

struct Start {
    Table table;
    int32_t nesterov;
    float momentum, eps;
};
struct Products {
    Table table;
    Step step;
    const float* lr_dev;
    f32x4* part;      // two sums of a tile for every block that divides stages
    float lr;
    uint32_t whole;   // tiles with a block of their own
    uint32_t stages;  // of the others
    uint32_t blocks;  // that divide them
};

constexpr int kWords = 1000;
struct Words {
    uint32_t* to;
    int32_t n;
    uint32_t word[kWords];
};
static_assert(sizeof(Words) <= 4096, "kernel arguments");

__global__ __launch_bounds__(256) void muon_table_kernel(const Words w) {
    for (int i = threadIdx.x; i < w.n; i += 256) w.to[i] = w.word[i];
}

// ---- momentum and the update's norm ------------------------------------------------------
// m = momentum m + g; the sum of the squares of u = g + momentum m (or of m), in 64 bits, a partial sum a block.  Bound by memory:
// ResNet-18's 11.7 M values with fp32 gradients in 28 us, 5.0 TB/s; 4096 x 8192 with bf16 ones in 93 us, 3.6 TB/s.
template <bool BF16>
__device__ __forceinline__ float grad_at(const void* g, int64_t i) {
    return BF16 ? bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(g)[i]) : reinterpret_cast<const float*>(g)[i];
}

// Four from the i-th four on.
template <bool BF16>
__device__ __forceinline__ f32x4 grad4(const void* g, int64_t i) {
    if constexpr (BF16) {
        const u32x2 r = reinterpret_cast<const u32x2*>(g)[i];
        return f32x4{bf16_bits_to_f32(r.x & 0xFFFFu), __uint_as_float(r.x & 0xFFFF0000u), bf16_bits_to_f32(r.y & 0xFFFFu),
                     __uint_as_float(r.y & 0xFFFF0000u)};
    } else {
        return reinterpret_cast<const f32x4*>(g)[i];
    }
}
__device__ __forceinline__ bool wide(const Matrix& j) {
    return ((reinterpret_cast<uintptr_t>(j.mom) | reinterpret_cast<uintptr_t>(j.g)) & 15) == 0;
}

template <bool BF16>
__global__ __launch_bounds__(256) void muon_momentum_kernel(const Start a) {
    __shared__ double sums[4];
    const int at = find(a.table.first, a.table.n, blockIdx.x);
    const Matrix& j = a.table.matrix[at];
    const uint32_t block = blockIdx.x - a.table.first[at];
    const int64_t count = (int64_t)j.m * j.n;
    double sum = 0.0;
    const int64_t vecs = wide(j) ? count / 4 : 0, stride = (int64_t)j.parts * 256;
    constexpr int U = 4;  // pieces in flight a thread
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < vecs; i += U * stride) {
        f32x4 m[U], g[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t at = i + k * stride < vecs ? i + k * stride : i;
            m[k] = reinterpret_cast<const f32x4*>(j.mom)[at];
            g[k] = grad4<BF16>(j.g, at);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (i + k * stride >= vecs) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[k][e] = a.momentum * m[k][e] + g[k][e];
                const double u = a.nesterov ? g[k][e] + a.momentum * m[k][e] : m[k][e];
                sum += u * u;
            }
            reinterpret_cast<f32x4*>(j.mom)[i + k * stride] = m[k];
        }
    }
    for (int64_t i = vecs * 4 + (int64_t)block * 256 + threadIdx.x; i < count; i += stride) {
        const float g = grad_at<BF16>(j.g, i), m = a.momentum * j.mom[i] + g;
        j.mom[i] = m;
        const double u = a.nesterov ? g + a.momentum * m : m;
        sum += u * u;
    }
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) j.norm[block] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// ---- X and its transpose -----------------------------------------------------------------
// A block takes 64 x 64 values of the update over its norm: rows of `direct` as they lie, rows of `turned` from LDS.  Bound by memory:
// 4096 x 8192 in 100 us, 4.7 TB/s.
template <bool BF16>
__global__ __launch_bounds__(256) void muon_start_kernel(const Start a) {
    __shared__ float tile[64][65];
    __shared__ double sums[4];
    const int at = find(a.table.divided, a.table.n, blockIdx.x);
    const Matrix& j = a.table.matrix[at];
    const uint32_t block = blockIdx.x - a.table.divided[at];
    // w is rows x cols: `direct` has its rows, `turned` its columns
    const int32_t rows = j.tall ? j.n : j.m, cols = j.tall ? j.m : j.n;
    uint8_t *const direct = j.tall ? j.xt[0] : j.x[0], *const turned = j.tall ? j.x[0] : j.xt[0];
    const uint32_t pitch_d = j.tall ? j.mp : j.np, pitch_t = j.tall ? j.np : j.mp;
    const int tid = threadIdx.x;
    double sum = tid < (int)j.parts ? j.norm[tid] : 0.0;
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d, 64);
    if ((tid & 63) == 0) sums[tid >> 6] = sum;
    __syncthreads();
    const float inv = (float)((double)kXScale / (sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + (double)a.eps));
    const uint32_t tiles = (uint32_t)(cols + 63) / 64;
    const int32_t r0 = (int32_t)(block / tiles) * 64, c0 = (int32_t)(block % tiles) * 64;
    const bool fours = cols % 4 == 0 && wide(j);
    // thread (r, 8 values): two passes of 32 rows
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int r = 32 * p + tid / 8, c = tid % 8 * 8;
        const int64_t i = (int64_t)(r0 + r) * cols + c0 + c;
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 m = {0.0f, 0.0f, 0.0f, 0.0f}, g = m;
            if (fours) {
                if (r0 + r < rows && c0 + c + 4 * h < cols) {
                    m = *reinterpret_cast<const f32x4*>(j.mom + i + 4 * h);
                    if (a.nesterov) g = grad4<BF16>(j.g, i / 4 + h);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (r0 + r < rows && c0 + c + 4 * h + e < cols) {
                        m[e] = j.mom[i + 4 * h + e];
                        if (a.nesterov) g[e] = grad_at<BF16>(j.g, i + 4 * h + e);
                    }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[4 * h + e] = (a.nesterov ? g[e] + a.momentum * m[e] : m[e]) * inv;
                tile[r][c + 4 * h + e] = v[4 * h + e];
            }
        }
        if (r0 + r < rows && c0 + c < (cols + 31) / 32 * 32) put8(direct + (r0 + r) * (int64_t)pitch_d + place(c0 + c), v);
    }
    __syncthreads();
    // eight lanes write the 128 bytes of 32 values: leading halves of 8 each, then trailing ones
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int c = 32 * (p & 1) + tid / 8, r = 32 * (p >> 1) + tid % 4 * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[r + e][c];
        if (c0 + c < cols && r0 + r < (rows + 31) / 32 * 32)
            put_half8(turned + (c0 + c) * (int64_t)pitch_t + place(r0 + r), v, tid & 4);
    }
}

// ---- products ----------------------------------------------------------------------------
// Tile w of those on and below the diagonal, row after row.
__device__ __forceinline__ void lower_tile(uint32_t w, uint32_t* i, uint32_t* j) {
    uint32_t r = (uint32_t)((sqrtf(8.0f * (float)w + 1.0f) - 1.0f) * 0.5f);
    while (r * (r + 1) / 2 > w) --r;
    while ((r + 1) * (r + 2) / 2 <= w) ++r;
    *i = r;
    *j = w - r * (r + 1) / 2;
}

// A block a tile for as many tiles as fill the GPU whole times; the stages of the tiles that are left, in a row, are divided evenly
// over as many blocks again.  A tile whose stages lie in more than one block is left as sums, two at most for a block, and FINISH,
// a block a tile, adds them in order and ends it.  (All tiles divided so: of 4096 x 4096 x 8192 578 us against 388, because blocks
// at different places of the rows share nothing in the L2s.)
// The matrix instructions bound large ones: P X of 4096 x 8192 in 640 us (256 x 256 tiles by four waves, 1.29 PFLOP/s of the three
// products; 128 x 128 683 where those took 610 by themselves), a symmetric 4096 x 4096 product in 191 + 10 (1.03).  512 x 512 x 512 take
// 9.8 us: a launch, 16 stages at 0.25 (copies alone 0.13, operands and products alone 0.16: a wave issues both in turn), the tile's end.
// Sixteen waves on a tile in place of four: 9.4 us, and 15 in place of 12 where every compute unit has a tile; waves that only copy take
// 0.9 from it, and add 9% where 128 x 128 tiles lie side by side.
template <int BT, int WAVES_M, int WAVES_N, int STAGES, bool FINISH>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, BT >= 256 ? 1 : BT >= 128 ? 2 : 3) void muon_product_kernel(const Products a) {
    typedef NtLoop<BT, BT, WAVES_M, WAVES_N, STAGES, NtF16x2> Loop;
    constexpr int TM = Loop::TM, TN = Loop::TN, PITCH = Loop::WN + 4;
    static_assert(Loop::BYTES >= Loop::WAVES * 32 * PITCH * 4, "staging fits in the ring");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[Loop::BYTES];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int QUADS = TM * TN * 4, UNROLL = 4;
    // blocks below a.whole: a tile each; those behind them: an even part of the stages of the other tiles
    const bool whole = !FINISH && blockIdx.x < a.whole;
    uint32_t block, u = 0, end = 1;
    const int strip = FINISH ? (int)(blockIdx.x % TM) : 0;  // of 32 rows of every wave
    if (FINISH) {
        block = a.whole + blockIdx.x / TM;
    } else if (whole) {
        block = (uint32_t)xcd_remap(blockIdx.x, a.whole);
    } else {
        block = (uint32_t)xcd_remap(blockIdx.x - a.whole, a.blocks);
        u = (uint32_t)((uint64_t)block * a.stages / a.blocks);
        end = (uint32_t)((uint64_t)(block + 1) * a.stages / a.blocks);
    }
    while (u < end) {
        const int at = FINISH || whole ? find(a.table.first, a.table.n, block) : find(a.table.divided, a.table.n, u);
        const auto* const x = constant(a.table.matrix + at);
        const Job j = job_of(x, a.step);
        const uint32_t first_tile = *constant(a.table.first + at), first_stage = *constant(a.table.divided + at);
        const uint32_t stages = j.pitch / 128;
        const uint32_t skip = a.whole > first_tile ? a.whole - first_tile : 0;  // of its tiles, those with a block of their own
        uint32_t tile, s0 = 0, s1 = stages;
        if (FINISH || whole) {
            tile = block - first_tile;
            u = end;
        } else {
            tile = (u - first_stage) / stages;
            s0 = u - first_stage - tile * stages;
            s1 = end - u < stages - s0 ? s0 + (end - u) : stages;
            u += s1 - s0;
            tile += skip;
        }
        uint32_t tm, tn;
        if (j.symmetric)
            lower_tile(tile, &tm, &tn);
        else
            nt_tile(tile, (uint32_t)(j.M + BT - 1) / BT, (uint32_t)(j.N + BT - 1) / BT, &tm, &tn);
        const int32_t m0 = (int32_t)(tm * BT), n0 = (int32_t)(tn * BT);

        constexpr int STRIPS = FINISH ? 1 : TM;
        f32x16 acc[STRIPS][TN];
#pragma unroll
        for (int i = 0; i < STRIPS; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][t][v] = 0.0f;
        if constexpr (FINISH) {
            // the blocks of the tile's first and last stage
            const uint64_t first = (uint64_t)first_stage + (uint64_t)(tile - skip) * stages;
            const uint32_t b0 = (uint32_t)(((first + 1) * a.blocks + a.stages - 1) / a.stages) - 1;
            const uint32_t b1 = (uint32_t)(((first + stages) * a.blocks + a.stages - 1) / a.stages) - 1;
            if (b0 == b1) return;  // its product wrote it
#pragma unroll UNROLL
            for (uint32_t b = b0; b <= b1; ++b) {
                const f32x4* src = a.part + (((int64_t)(2 * b + (b == b0)) * QUADS + strip * TN * 4) * Loop::WAVES + wave) * 64 + lane;
#pragma unroll
                for (int t = 0; t < TN; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 v = src[(t * 4 + g) * Loop::WAVES * 64];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[0][t][4 * g + e] += v[e];
                    }
            }
        } else {
            typename Loop::RowsA ra;
            typename Loop::RowsB rb;
            ra.init(j.a, m0, j.M, j.pitch, wave, lane, Loop::copy_seg(wave, lane));
            rb.init(j.b, n0, j.N, j.pitch, wave, lane, Loop::copy_seg(wave, lane));
            Loop::run(ra, rb, smem, (int)s0, (int)s1, (int)(s1 - s0), j.pitch, wave, lane, acc);
            if (s1 - s0 < stages) {
                f32x4* dst = a.part + ((int64_t)(2 * block + (s0 == 0)) * QUADS * Loop::WAVES + wave) * 64 + lane;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int t = 0; t < TN; ++t)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            dst[((i * TN + t) * 4 + g) * Loop::WAVES * 64] =
                                f32x4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
                continue;
            }
        }

        // ---- v = p acc + q aux, 32 rows of the wave's tile at a time, through LDS: written along the rows, and turned ----
        float* stage = reinterpret_cast<float*>(smem) + wave * 32 * PITCH;
        const int wm = wave / WAVES_N, wn = wave % WAVES_N, half = lane >> 5, l32 = lane & 31;
        constexpr int CG = Loop::WN / 8, RPP = 64 / CG;
        const int32_t Np = (j.N + 31) / 32 * 32, Mp = (j.M + 31) / 32 * 32;
        const float lr = j.to_w ? (a.lr_dev ? *a.lr_dev : a.lr) : 0.0f;
        const float keep = 1.0f - lr * x->weight_decay, move = -lr * x->scale * (1.0f / kXScale);
        const bool even = j.N % 4 == 0 && (reinterpret_cast<uintptr_t>(x->w) & 15) == 0;
        const bool turn = j.turned && !(j.symmetric && tm == tn);
#pragma unroll
        for (int i = 0; i < STRIPS; ++i) {
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4*>(stage + l32 * PITCH + 32 * t + 8 * g + 4 * half) =
                        f32x4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
            __builtin_amdgcn_wave_barrier();
            const int32_t row0 = m0 + wm * Loop::WM + 32 * (FINISH ? strip : i), col = n0 + wn * Loop::WN + 8 * (lane % CG);
#pragma unroll
            for (int p = 0; p < 32 / RPP; ++p) {
                const int r = p * RPP + lane / CG;
                const int32_t row = row0 + r;
                f32x4* s = reinterpret_cast<f32x4*>(stage + r * PITCH + 8 * (lane % CG));
                const f32x4 lo = s[0], hi = s[1];
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                const bool in = row < j.M && col < Np;
                if (j.aux) {
                    float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (in) get8(j.aux + (int64_t)row * j.pitch_o + place(col), y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = j.p * v[e] + j.q * y[e] + (row == col + e && row < j.M ? j.diag : 0.0f);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= j.p;
                }
                if (j.direct && in) put8(j.direct + (int64_t)row * j.pitch_o + place(col), v);
                if (turn) {
                    s[0] = f32x4{v[0], v[1], v[2], v[3]};
                    s[1] = f32x4{v[4], v[5], v[6], v[7]};
                }
                if (j.to_w && even && row < j.M) {
                    float* w = x->w + (int64_t)row * j.N + col;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (col + 4 * h < j.N) {
                            f32x4 y = *reinterpret_cast<f32x4*>(w + 4 * h);
#pragma unroll
                            for (int e = 0; e < 4; ++e) y[e] = keep * y[e] + move * v[4 * h + e];
                            *reinterpret_cast<f32x4*>(w + 4 * h) = y;
                        }
                }
            }
            if (j.to_w && !even) {  // rows begin anywhere: a value a lane, side by side (p of it is still to come: no aux here)
                constexpr int ROWS = Loop::WN < 64 ? 64 / Loop::WN : 1, COLS = Loop::WN < 64 ? Loop::WN : 64;
#pragma unroll 4
                for (int k = 0; k < 32 / ROWS * (Loop::WN / COLS); ++k) {
                    const int r = k / (Loop::WN / COLS) * ROWS + lane / COLS, c = k % (Loop::WN / COLS) * COLS + lane % COLS;
                    const int32_t n = n0 + wn * Loop::WN + c;
                    if (row0 + r < j.M && n < j.N) {
                        float* const w = x->w + (int64_t)(row0 + r) * j.N + n;
                        *w = keep * *w + move * (j.p * stage[r * PITCH + c]);
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
            if (turn) {
                // eight lanes write the 128 bytes of 32 values: leading halves of 8 each, then trailing ones
#pragma unroll
                for (int k = 0; k < Loop::WN / 8; ++k) {
                    const int c = 8 * k + lane / 8, r = lane % 4 * 8;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = stage[(r + e) * PITCH + c];
                    const int32_t n = n0 + wn * Loop::WN + c;
                    if (n < j.N && row0 + r < Mp) put_half8(j.turned + (int64_t)n * j.pitch_t + place(row0 + r), v, lane & 4);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (!FINISH && u < end) __syncthreads();  // the next tile's copies land where this one was turned
    }
}

// What a product costs with a tile, in units of 10 ns: a stage of a block that is one of `side` on its CU, and of one alone; adding a
// part of a divided tile.  Measured on 4096 x 8192 x 4096 (2.46, 1.32 and 0.7 us a stage side by side) and on 512 x 3200 x 2048 (0.78
// and 0.44 us alone, 128 and 64).
struct TileCost {
    int tile, side, busy, alone, part;
};
constexpr TileCost kTiles[3] = {{256, 1, 246, 246, 400}, {128, 2, 132, 78, 100}, {64, 3, 70, 44, 30}};
constexpr int kCus = 256;

int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

uint64_t job_tiles(const Matrix& x, const Step& step, int tile) {
    const uint64_t m = tiles_of(x.m, tile);
    return step.kind == APPLY ? m * tiles_of(x.n, tile) : m * (m + 1) / 2;
}

// How a launch is run: a block a tile for `whole` of its tiles, `blocks` for the stages of the rest.
struct Plan {
    Step step;
    int tile;
    uint32_t tiles, whole, stages, blocks;
};

// The tile, and how many tiles have a block of their own: whatever ends first by the costs above.
Plan plan_of(const Matrix* x, int count, const Step& step) {
    Plan a = {step, 0, 0, 0, 0, 0};
    double least = 1e300;
    for (const TileCost& c : kTiles) {
        uint64_t tiles = 0, stages = 0, longest = 0;
        for (int i = 0; i < count; ++i) {
            const uint64_t s = (step.kind == GRAM ? x[i].np : x[i].mp) / 128, t = job_tiles(x[i], step, c.tile);
            tiles += t;
            stages += t * s;
            longest = longest > s ? longest : s;
        }
        if (stages >> 32) continue;
        const uint64_t slots = (uint64_t)kCus * c.side;
        const double mean = (double)stages / tiles;
        auto time = [&](uint64_t blocks, double each) { return blocks <= kCus ? c.alone * each : (double)((blocks + slots - 1) / slots) * c.busy * each; };
        const double all = std::max(time(tiles, mean), (double)c.alone * longest);
        if (all < least) {
            least = all;
            a.tile = c.tile;
            a.tiles = a.whole = (uint32_t)tiles;
            a.blocks = 0;
        }
        // the rest divided among up to `slots` blocks: a launch more, in which the sums of a tile are added one after the other, and
        // sums that are written and read at 4 TB/s
        const uint64_t whole = tiles / slots * slots, rest = tiles - whole;
        for (uint64_t blocks = slots; blocks > rest && rest; blocks /= 2) {
            const double each = rest * mean / blocks;
            if (each < 4) continue;
            const double even = time(whole, mean) * (whole != 0) + time(blocks, each) + 500 + (1 + (double)blocks / rest) * c.part +
                                (double)(blocks + rest) * c.tile * c.tile * 4 * 2 / 4e4;
            if (even < least) {
                least = even;
                a.tile = c.tile;
                a.tiles = (uint32_t)tiles;
                a.whole = (uint32_t)whole;
                a.blocks = (uint32_t)blocks;
            }
        }
    }
    uint64_t before = 0;
    for (int i = 0; i < count; ++i) {
        const uint64_t t = job_tiles(x[i], step, a.tile), skip = a.whole <= before ? 0 : std::min(a.whole - before, t);
        before += t;
        a.stages += (uint32_t)((t - skip) * ((step.kind == GRAM ? x[i].np : x[i].mp) / 128));
    }
    return a;
}

template <int BT, int WAVES_M, int WAVES_N, int STAGES>
hipError_t launch_tile(const Products& a, const Plan& p, hipStream_t s) {
    const dim3 threads(64 * WAVES_M * WAVES_N);
    hipLaunchKernelGGL((muon_product_kernel<BT, WAVES_M, WAVES_N, STAGES, false>), dim3(p.whole + p.blocks), threads, 0, s, a);
    if (p.blocks) hipLaunchKernelGGL((muon_product_kernel<BT, WAVES_M, WAVES_N, STAGES, true>), dim3((p.tiles - p.whole) * (BT / WAVES_M / 32)), threads, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_products(const Products& a, const Plan& p, hipStream_t s) {
    if (p.tile == 256) return launch_tile<256, 2, 2, 2>(a, p, s);
    return p.tile == 128 ? launch_tile<128, 2, 2, 2>(a, p, s) : launch_tile<64, 2, 2, 3>(a, p, s);
}

// Words on their way into the workspace, some 4000 bytes a launch.  A launch that fails is the last one, and what follows is dropped.
struct Writer {
    Words w;
    uint32_t* next;
    hipStream_t s;
    hipError_t e;
    Writer(void* to, hipStream_t stream) : next(static_cast<uint32_t*>(to)), s(stream), e(hipSuccess) { w.n = 0; }
    void put(const void* p, int n) {
        const uint32_t* v = static_cast<const uint32_t*>(p);
        for (int i = 0; i < n && e == hipSuccess; ++i) {
            if (w.n == 0) w.to = next;
            w.word[w.n++] = v[i];
            ++next;
            if (w.n == kWords) flush();
        }
    }
    void flush() {
        if (w.n == 0 || e != hipSuccess) return;
        hipLaunchKernelGGL(muon_table_kernel, dim3(1), dim3(256), 0, s, w);
        e = hipGetLastError();
        w.n = 0;
    }
};

// The launches of so many steps, in order.
template <typename F>
void each_step(int steps, F f) {
    for (int now = 0; steps > 0; now ^= 1) {
        const int two = steps > 1;
        steps -= two ? 2 : 1;
        f(Step{GRAM, 0, 0, now, 0});
        f(Step{POLY, 0, 0, now, 0});
        if (two) {
            f(Step{TIMES, 0, 0, now, 0});
            f(Step{BOTH, 0, 0, now, 0});
            f(Step{POLY, 1, 0, now, 0});
            f(Step{PAIR, 1, 0, now, 0});
        }
        f(Step{APPLY, 0, two, now, steps == 0});
    }
}
constexpr int kMostLaunches = kMuonSteps / 2 * 7;

// The workspace of a group: the matrices' arrays, the most sums of divided tiles (three steps have every kind of launch), the table.
struct Layout {
    Matrix x[kMuonMatrices];
    int64_t part, table, end;
};

void lay_out(const tbn_muon_tensor* t, int n, uint8_t* ws, Layout* l) {
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        uint8_t* const was = ws + at;
        at += round_up(bytes, 256);
        return was;
    };
    for (int i = 0; i < n; ++i) {
        Matrix& x = l->x[i];
        x.w = t[i].w;
        x.mom = t[i].m;
        x.g = t[i].g;
        x.tall = t[i].rows > t[i].cols;
        x.m = x.tall ? t[i].cols : t[i].rows;
        x.n = x.tall ? t[i].rows : t[i].cols;
        x.mp = (uint32_t)round_up(x.m, 32) * 4;
        x.np = (uint32_t)round_up(x.n, 32) * 4;
        x.weight_decay = t[i].weight_decay;
        x.scale = t[i].scale;
        const int64_t parts = ((int64_t)x.m * x.n + 4095) / 4096;
        x.parts = (uint32_t)(parts < 256 ? parts : 256);
        for (int k = 0; k < 2; ++k) x.x[k] = take((int64_t)x.m * x.np), x.xt[k] = take((int64_t)x.n * x.mp);
        x.a = take((int64_t)x.m * x.mp);
        x.t = take((int64_t)x.m * x.mp);
        for (uint8_t*& p : x.p) p = take((int64_t)x.m * x.mp);
        x.norm = reinterpret_cast<double*>(take(256 * 8));
    }
    l->part = at;
    int64_t most = 0;
    each_step(3, [&](const Step& step) {
        const Plan p = plan_of(l->x, n, step);
        most = std::max(most, (int64_t)p.blocks * 2 * p.tile * p.tile * 4);
    });
    l->table = l->part + round_up(most, 256);
    l->end = l->table + n * (int64_t)sizeof(Matrix) + (kMostLaunches + 1) * 2 * round_up(n, 8) * 4;
}

static_assert(sizeof(Matrix) % 8 == 0, "one behind the other");

}  // namespace

// Matrices that go together: up to kMuonMatrices of them, and no more than 2^25 values (one larger matrix goes alone).
int muon_group(const tbn_muon_tensor* t, int n) {
    int64_t sum = 0;
    for (int i = 0; i < n; ++i) {
        sum += t[i].rows * (int64_t)t[i].cols;
        if (i == kMuonMatrices || (i && sum > (1 << 25))) return i;
    }
    return n;
}

int64_t muon_group_bytes(const tbn_muon_tensor* t, int n) {
    Layout l;
    lay_out(t, n, nullptr, &l);
    return l.end;
}

hipError_t launch_muon_group(const tbn_muon_tensor* t, int n, const MuonHyper& h, uint8_t* ws, hipStream_t s) {
    Layout l;
    lay_out(t, n, ws, &l);
    hipError_t e;

    // the tables of all launches, then the launches
    const int64_t each = round_up(n, 8);
    Writer to(ws + l.table, s);
    to.put(l.x, n * (int)sizeof(Matrix) / 4);
    auto put_firsts = [&](auto of) {  // running sums over the matrices
        uint32_t sum = 0;
        for (int i = 0; i < each; ++i) {
            to.put(&sum, 1);
            if (i < n) sum += of(i);
        }
        return sum;
    };
    const uint32_t blocks = put_firsts([&](int i) { return l.x[i].parts; });
    const uint32_t tiles = put_firsts([&](int i) { return (uint32_t)(tiles_of(l.x[i].m, 64) * tiles_of(l.x[i].n, 64)); });
    Plan plans[kMostLaunches];
    int launches = 0;
    each_step(h.steps, [&](const Step& step) {
        const Plan p = plans[launches++] = plan_of(l.x, n, step);
        put_firsts([&](int i) { return (uint32_t)job_tiles(l.x[i], step, p.tile); });
        uint64_t before = 0;
        put_firsts([&](int i) {
            const uint64_t t = job_tiles(l.x[i], step, p.tile), skip = p.whole <= before ? 0 : std::min(p.whole - before, t);
            before += t;
            return (uint32_t)((t - skip) * ((step.kind == GRAM ? l.x[i].np : l.x[i].mp) / 128));
        });
    });
    to.flush();
    if ((e = to.e) != hipSuccess) return e;

    const uint32_t* first = reinterpret_cast<const uint32_t*>(ws + l.table + n * (int64_t)sizeof(Matrix));
    Table table = {first, first + each, reinterpret_cast<const Matrix*>(ws + l.table), n};
    const Start st = {table, h.nesterov, h.momentum, h.eps};
    if (h.g_f32)
        hipLaunchKernelGGL((muon_momentum_kernel<false>), dim3(blocks), dim3(256), 0, s, st);
    else
        hipLaunchKernelGGL((muon_momentum_kernel<true>), dim3(blocks), dim3(256), 0, s, st);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (h.g_f32)
        hipLaunchKernelGGL((muon_start_kernel<false>), dim3(tiles), dim3(256), 0, s, st);
    else
        hipLaunchKernelGGL((muon_start_kernel<true>), dim3(tiles), dim3(256), 0, s, st);
    if ((e = hipGetLastError()) != hipSuccess) return e;

    for (int i = 0; i < launches; ++i) {
        const Plan& p = plans[i];
        table.first += 2 * each;
        table.divided += 2 * each;
        Products a = {};
        a.table = table;
        a.step = p.step;
        a.part = reinterpret_cast<f32x4*>(ws + l.part);
        a.lr = h.lr;
        a.lr_dev = h.lr_dev;
        a.whole = p.whole;
        a.stages = p.stages;
        a.blocks = p.blocks;
        if ((e = launch_products(a, p, s)) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tbn
