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
// A launch's table: the first blocks (tiles) of its jobs, the first divided stages, and the jobs.
static_assert(kMuonMatrices <= 64, "a lane finds a job");

template <typename T>
struct Table {
    const uint32_t* first[2];  // round_up(n, 8) each, the largest value behind the last
    const T* job;
    int32_t n;
    // The job that `at` falls into.
    __device__ __forceinline__ const T& find(int which, uint32_t at) const {
        const int lane = threadIdx.x & 63;
        const uint32_t f = lane < n ? first[which][lane] : 0xFFFFFFFFu;
        return job[__popcll(__ballot(f <= at)) - 1];
    }
};

struct StartJob {
    float* m;
    const void* g;
    uint8_t* direct;  // X (or X^T) in the layout of m, and its transpose
    uint8_t* turned;
    double* norm;     // partial sums of squares
    int32_t rows, cols;
    uint32_t pitch_d, pitch_t;
    uint32_t first, first_tile, parts, unused;
};
struct Start {
    Table<StartJob> table;
    int32_t nesterov;
    float momentum, eps;
};
// v = p (a b^T) + q aux + diag on the diagonal
struct Job {
    const uint8_t* a;    // rows of M and of N, `pitch` bytes each
    const uint8_t* b;
    const uint8_t* aux;  // rows of pitch_o bytes, or null
    uint8_t* direct;     // v by rows, or null
    uint8_t* turned;     // v by columns, or null
    float* w;            // [M][N] moved along v, or null
    uint32_t pitch, pitch_o, pitch_t;
    int32_t M, N;
    uint32_t first, first_tile;  // divided stages, and tiles, of the jobs before it
    int32_t symmetric;
    float p, q, diag, weight_decay, scale;
    uint32_t unused;
};
struct Products {
    Table<Job> table;
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
// m = momentum m + g; the sum of the squares of u = g + momentum m (or of m), in 64 bits, a partial sum a block.
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
__device__ __forceinline__ bool wide(const StartJob& j) {
    return ((reinterpret_cast<uintptr_t>(j.m) | reinterpret_cast<uintptr_t>(j.g)) & 15) == 0;
}

template <bool BF16>
__global__ __launch_bounds__(256) void muon_momentum_kernel(const Start a) {
    __shared__ double sums[4];
    const StartJob& j = a.table.find(0, blockIdx.x);
    const uint32_t block = blockIdx.x - j.first_tile;
    const int64_t count = (int64_t)j.rows * j.cols;
    double sum = 0.0;
    const int64_t vecs = wide(j) ? count / 4 : 0, stride = (int64_t)j.parts * 256;
    constexpr int U = 4;  // pieces in flight a thread
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < vecs; i += U * stride) {
        f32x4 m[U], g[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t at = i + k * stride < vecs ? i + k * stride : i;
            m[k] = reinterpret_cast<const f32x4*>(j.m)[at];
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
            reinterpret_cast<f32x4*>(j.m)[i + k * stride] = m[k];
        }
    }
    for (int64_t i = vecs * 4 + (int64_t)block * 256 + threadIdx.x; i < count; i += stride) {
        const float g = grad_at<BF16>(j.g, i), m = a.momentum * j.m[i] + g;
        j.m[i] = m;
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
// A block takes 64 x 64 values of the update over its norm: rows of `direct` as they lie, rows of `turned` from LDS.
template <bool BF16>
__global__ __launch_bounds__(256) void muon_start_kernel(const Start a) {
    __shared__ float tile[64][65];
    __shared__ double sums[4];
    const StartJob& j = a.table.find(1, blockIdx.x);
    const uint32_t block = blockIdx.x - j.first;
    const int tid = threadIdx.x;
    double sum = tid < (int)j.parts ? j.norm[tid] : 0.0;
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d, 64);
    if ((tid & 63) == 0) sums[tid >> 6] = sum;
    __syncthreads();
    const float inv = (float)((double)kXScale / (sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + (double)a.eps));
    const uint32_t tiles = (uint32_t)(j.cols + 63) / 64;
    const int32_t r0 = (int32_t)(block / tiles) * 64, c0 = (int32_t)(block % tiles) * 64;
    const bool fours = j.cols % 4 == 0 && wide(j);
    // thread (r, 8 values): two passes of 32 rows
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int r = 32 * p + tid / 8, c = tid % 8 * 8;
        const int64_t i = (int64_t)(r0 + r) * j.cols + c0 + c;
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 m = {0.0f, 0.0f, 0.0f, 0.0f}, g = m;
            if (fours) {
                if (r0 + r < j.rows && c0 + c + 4 * h < j.cols) {
                    m = *reinterpret_cast<const f32x4*>(j.m + i + 4 * h);
                    if (a.nesterov) g = grad4<BF16>(j.g, i / 4 + h);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (r0 + r < j.rows && c0 + c + 4 * h + e < j.cols) {
                        m[e] = j.m[i + 4 * h + e];
                        if (a.nesterov) g[e] = grad_at<BF16>(j.g, i + 4 * h + e);
                    }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[4 * h + e] = (a.nesterov ? g[e] + a.momentum * m[e] : m[e]) * inv;
                tile[r][c + 4 * h + e] = v[4 * h + e];
            }
        }
        if (r0 + r < j.rows && c0 + c < (j.cols + 31) / 32 * 32) put8(j.direct + (r0 + r) * (int64_t)j.pitch_d + place(c0 + c), v);
    }
    __syncthreads();
    // eight lanes write the 128 bytes of 32 values: leading halves of 8 each, then trailing ones
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int c = 32 * (p & 1) + tid / 8, r = 32 * (p >> 1) + tid % 4 * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[r + e][c];
        if (c0 + c < j.cols && r0 + r < (j.rows + 31) / 32 * 32)
            put_half8(j.turned + (c0 + c) * (int64_t)j.pitch_t + place(r0 + r), v, tid & 4);
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
template <int BT, int WAVES_M, int WAVES_N, int STAGES, bool FINISH>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, BT >= 256 ? 1 : BT >= 128 ? 2 : 3) void muon_product_kernel(const Products a) {
    typedef NtLoop<BT, BT, WAVES_M, WAVES_N, STAGES, NtF16x2> Loop;
    constexpr int TM = Loop::TM, TN = Loop::TN, PITCH = Loop::WN + 4;
    static_assert(Loop::BYTES >= Loop::WAVES * 32 * PITCH * 4, "staging fits in the ring");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[Loop::BYTES];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int QUADS = TM * TN * 4, UNROLL = BT >= 256 ? 1 : BT >= 128 ? 2 : 4;
    // blocks below a.whole: a tile each; those behind them: an even part of the stages of the other tiles
    const bool whole = !FINISH && blockIdx.x < a.whole;
    uint32_t block, u = 0, end = 1;
    if (FINISH) {
        block = a.whole + blockIdx.x;
    } else if (whole) {
        block = (uint32_t)xcd_remap(blockIdx.x, a.whole);
    } else {
        block = (uint32_t)xcd_remap(blockIdx.x - a.whole, a.blocks);
        u = (uint32_t)((uint64_t)block * a.stages / a.blocks);
        end = (uint32_t)((uint64_t)(block + 1) * a.stages / a.blocks);
    }
    while (u < end) {
        const Job& j = FINISH || whole ? a.table.find(0, block) : a.table.find(1, u);
        const uint32_t stages = j.pitch / 128;
        const uint32_t skip = a.whole > j.first_tile ? a.whole - j.first_tile : 0;  // of its tiles, those with a block of their own
        uint32_t tile, s0 = 0, s1 = stages;
        if (FINISH || whole) {
            tile = block - j.first_tile;
            u = end;
        } else {
            tile = (u - j.first) / stages;
            s0 = u - j.first - tile * stages;
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

        f32x16 acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][t][v] = 0.0f;
        if constexpr (FINISH) {
            // the blocks of the tile's first and last stage
            const uint64_t first = (uint64_t)j.first + (uint64_t)(tile - skip) * stages;
            const uint32_t b0 = (uint32_t)(((first + 1) * a.blocks + a.stages - 1) / a.stages) - 1;
            const uint32_t b1 = (uint32_t)(((first + stages) * a.blocks + a.stages - 1) / a.stages) - 1;
            if (b0 == b1) return;  // its product wrote it
#pragma unroll UNROLL
            for (uint32_t b = b0; b <= b1; ++b) {
                const f32x4* src = a.part + ((int64_t)(2 * b + (b == b0)) * QUADS * Loop::WAVES + wave) * 64 + lane;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int t = 0; t < TN; ++t)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const f32x4 v = src[((i * TN + t) * 4 + g) * Loop::WAVES * 64];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][t][4 * g + e] += v[e];
                        }
            }
        } else {
            typename Loop::RowsA ra;
            typename Loop::RowsB rb;
            ra.init(j.a, m0, j.M, j.pitch, wave, lane, Loop::copy_seg(wave, lane));
            rb.init(j.b, n0, j.N, j.pitch, wave, lane, Loop::copy_seg(wave, lane));
            Loop::run(ra, rb, smem, (int)s0, (int)s1, j.pitch, wave, lane, acc);
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
        const float lr = j.w ? (a.lr_dev ? *a.lr_dev : a.lr) : 0.0f;
        const float keep = 1.0f - lr * j.weight_decay, move = -lr * j.scale * (1.0f / kXScale);
        const bool even = j.N % 4 == 0 && (reinterpret_cast<uintptr_t>(j.w) & 15) == 0;
        const bool turn = j.turned && !(j.symmetric && tm == tn);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4*>(stage + l32 * PITCH + 32 * t + 8 * g + 4 * half) =
                        f32x4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
            __builtin_amdgcn_wave_barrier();
            const int32_t row0 = m0 + wm * Loop::WM + 32 * i, col = n0 + wn * Loop::WN + 8 * (lane % CG);
#pragma unroll
            for (int p = 0; p < 32 / RPP; ++p) {
                const int r = p * RPP + lane / CG;
                const int32_t row = row0 + r;
                f32x4* s = reinterpret_cast<f32x4*>(stage + r * PITCH + 8 * (lane % CG));
                const f32x4 lo = s[0], hi = s[1];
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                const bool in = row < j.M && col < Np;
                if (j.aux) {
                    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (in) get8(j.aux + (int64_t)row * j.pitch_o + place(col), x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = j.p * v[e] + j.q * x[e] + (row == col + e && row < j.M ? j.diag : 0.0f);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= j.p;
                }
                if (j.direct && in) put8(j.direct + (int64_t)row * j.pitch_o + place(col), v);
                if (turn) {
                    s[0] = f32x4{v[0], v[1], v[2], v[3]};
                    s[1] = f32x4{v[4], v[5], v[6], v[7]};
                }
                if (j.w && row < j.M) {
                    float* w = j.w + (int64_t)row * j.N + col;
                    if (even) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if (col + 4 * h < j.N) {
                                f32x4 x = *reinterpret_cast<f32x4*>(w + 4 * h);
#pragma unroll
                                for (int e = 0; e < 4; ++e) x[e] = keep * x[e] + move * v[4 * h + e];
                                *reinterpret_cast<f32x4*>(w + 4 * h) = x;
                            }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (col + e < j.N) w[e] = keep * w[e] + move * v[e];
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

// What a product costs with a tile, in units of 10 ns: a stage of a block that is one of `side` on its CU, and of one alone; bytes
// of the sums of a block.  Measured on 4096 x 8192 x 4096 (2.46, 1.32 and 0.7 us a stage side by side) and on 512 x 3200 x 2048 (0.78
// and 0.44 us alone, 128 and 64).
struct TileCost {
    int tile, side, busy, alone, part;
};
constexpr TileCost kTiles[3] = {{256, 1, 246, 246, 400}, {128, 2, 132, 78, 100}, {64, 3, 70, 44, 30}};
constexpr int kCus = 256;

int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t part_bytes(const TileCost& c, int64_t blocks) { return blocks * 2 * c.tile * c.tile * 4; }


// The jobs of a launch, and how they are run.
struct Plan {
    int tile;
    uint32_t tiles, whole, stages, blocks;  // a block a tile for `whole` of them, `blocks` for the stages of the rest
};
struct Launch : Plan {
    Job job[kMuonMatrices];
    int n;
};

// The tile, and how many tiles have a block of their own: whatever ends first by the costs above.
void plan(Launch& a) {
    double least = 1e300;
    for (const TileCost& c : kTiles) {
        uint64_t tiles = 0, stages = 0, longest = 0;
        for (int i = 0; i < a.n; ++i) {
            const uint64_t m = tiles_of(a.job[i].M, c.tile), n = tiles_of(a.job[i].N, c.tile), s = a.job[i].pitch / 128;
            const uint64_t t = a.job[i].symmetric ? m * (m + 1) / 2 : m * n;
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
    uint32_t stage = 0, tile = 0;
    for (int i = 0; i < a.n; ++i) {
        Job& j = a.job[i];
        const uint32_t m = (uint32_t)tiles_of(j.M, a.tile), n = (uint32_t)tiles_of(j.N, a.tile);
        const uint32_t t = j.symmetric ? m * (m + 1) / 2 : m * n;
        j.first = stage;
        j.first_tile = tile;
        const uint32_t skip = a.whole <= tile ? 0 : std::min(a.whole - tile, t);
        tile += t;
        stage += (t - skip) * (j.pitch / 128);
    }
    a.stages = stage;
}

template <bool FINISH>
hipError_t launch_tiles(const Products& a, int tile, uint32_t blocks, hipStream_t s) {
    if (tile == 256)
        hipLaunchKernelGGL((muon_product_kernel<256, 2, 4, 2, FINISH>), dim3(blocks), dim3(512), 0, s, a);
    else if (tile == 128)
        hipLaunchKernelGGL((muon_product_kernel<128, 2, 2, 2, FINISH>), dim3(blocks), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((muon_product_kernel<64, 2, 2, 3, FINISH>), dim3(blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

// Words on their way into the workspace, some 4000 bytes a launch.
struct Writer {
    Words w;
    uint32_t* next;
    hipStream_t s;
    hipError_t e;
    Writer(void* to, hipStream_t stream) : next(static_cast<uint32_t*>(to)), s(stream), e(hipSuccess) { w.n = 0; }
    void put(const void* p, int n) {
        const uint32_t* v = static_cast<const uint32_t*>(p);
        for (int i = 0; i < n; ++i) {
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

// Words of the table of n jobs.
template <typename T>
int64_t table_words(int n) {
    static_assert(sizeof(T) % 8 == 0, "pointers lie at multiples of 8");
    return 2 * round_up(n, 8) + n * (int64_t)sizeof(T) / 4;
}

template <typename T>
Table<T> table_at(const void* p, int n) {
    const uint32_t* w = static_cast<const uint32_t*>(p);
    const int64_t each = round_up(n, 8);
    return {{w, w + each}, reinterpret_cast<const T*>(w + 2 * each), n};
}

template <typename T>
void write_table(Writer& to, const T* job, int n) {
    const uint32_t most = 0xFFFFFFFFu;
    for (int64_t i = 0; i < round_up(n, 8); ++i) to.put(i < n ? &job[i].first_tile : &most, 1);
    for (int64_t i = 0; i < round_up(n, 8); ++i) to.put(i < n ? &job[i].first : &most, 1);
    to.put(job, n * (int)sizeof(T) / 4);
}

// A matrix in the workspace: its sides, m <= n, and where its arrays begin (bytes).
struct Place {
    int64_t m, n, mp, np;  // mp, np: bytes of a row of m (n) values
    int64_t x[2], xt[2], a, t, p[3], norm, end;
    bool tall;
};

Place place_of(const tbn_muon_tensor& t, int64_t at) {
    Place p;
    p.tall = t.rows > t.cols;
    p.m = p.tall ? t.cols : t.rows;
    p.n = p.tall ? t.rows : t.cols;
    p.mp = round_up(p.m, 32) * 4;
    p.np = round_up(p.n, 32) * 4;
    auto take = [&](int64_t bytes) {
        const int64_t was = at;
        at += round_up(bytes, 256);
        return was;
    };
    for (int i = 0; i < 2; ++i) p.x[i] = take(p.m * p.np), p.xt[i] = take(p.n * p.mp);
    p.a = take(p.m * p.mp);
    p.t = take(p.m * p.mp);
    for (int64_t& b : p.p) b = take(p.m * p.mp);
    p.norm = take(256 * 8);
    p.end = at;
    return p;
}

// C = A B^T of rows of k values in `bytes`, for symmetric C (m x m) or any (m x n).
Job product(const uint8_t* a, const uint8_t* b, int64_t bytes, int64_t m, int64_t n, bool symmetric, float p) {
    Job j = {};
    j.a = a;
    j.b = b;
    j.pitch = (uint32_t)bytes;
    j.M = (int32_t)m;
    j.N = (int32_t)n;
    j.symmetric = symmetric;
    j.p = p;
    return j;
}

// ... a symmetric one of symmetric factors of this matrix, into `to`.
Job square(const Place& at, uint8_t* ws, int64_t a, int64_t b, int64_t to, float p) {
    Job j = product(ws + a, ws + b, at.mp, at.m, at.m, true, p);
    j.direct = j.turned = ws + to;
    j.pitch_o = j.pitch_t = (uint32_t)at.mp;
    return j;
}

// The launches of a group's steps, in order, each given to `run`.
template <typename F>
hipError_t muon_launches(const tbn_muon_tensor* t, int n, const Place* at, uint8_t* ws, int steps, F run) {
    Launch l;
    hipError_t e;
    auto begin = [&] { l.n = 0; };
    auto end = [&] {
        plan(l);
        return run(l);
    };
    for (int now = 0; steps > 0; now ^= 1) {
        const bool two = steps > 1;
        steps -= two ? 2 : 1;
        begin();
        for (int i = 0; i < n; ++i) {
            const Place& p = at[i];
            Job& j = l.job[l.n++] = product(ws + p.x[now], ws + p.x[now], p.np, p.m, p.m, true, 0x1p-10f);  // 2^24 to 2^14
            j.direct = j.turned = ws + p.a;
            j.pitch_o = j.pitch_t = (uint32_t)p.mp;
        }
        if ((e = end()) != hipSuccess) return e;
        for (int k = 0; k < (two ? 2 : 1); ++k) {
            begin();
            for (int i = 0; i < n; ++i) {
                const Place& p = at[i];
                Job& j = l.job[l.n++] = square(p, ws, p.a, p.a, p.p[k], kC * 0x1p-15f);  // 2^28 and 2^14 to 2^13
                j.aux = ws + p.a;
                j.q = kB * 0.5f;
                j.diag = kA * 0x1p13f;
            }
            if ((e = end()) != hipSuccess) return e;
            if (!two) break;
            begin();
            for (int i = 0; i < n; ++i) {
                const Place& p = at[i];
                // P A; after the second step the product of both P
                l.job[l.n++] = k == 0 ? square(p, ws, p.p[0], p.a, p.t, 0x1p-14f) : square(p, ws, p.p[1], p.p[0], p.p[2], 0x1p-14f);
            }
            if ((e = end()) != hipSuccess) return e;
            if (k) break;
            begin();
            for (int i = 0; i < n; ++i) l.job[l.n++] = square(at[i], ws, at[i].p[0], at[i].t, at[i].a, 0x1p-12f);  // P A P
            if ((e = end()) != hipSuccess) return e;
        }
        begin();
        for (int i = 0; i < n; ++i) {
            const Place& p = at[i];
            const uint8_t *by = ws + p.p[two ? 2 : 0], *xt = ws + p.xt[now];
            const float down = two ? 0x1p-12f : 0x1p-13f;
            const bool last = steps == 0, turn = last && p.tall;  // the last one along the rows of w
            Job& j = l.job[l.n++] = turn ? product(xt, by, p.mp, p.n, p.m, false, down) : product(by, xt, p.mp, p.m, p.n, false, down);
            if (last) {
                j.w = t[i].w;
                j.weight_decay = t[i].weight_decay;
                j.scale = t[i].scale;
            } else {
                j.direct = ws + p.x[now ^ 1];
                j.turned = ws + p.xt[now ^ 1];
                j.pitch_o = (uint32_t)p.np;
                j.pitch_t = (uint32_t)p.mp;
            }
        }
        if ((e = end()) != hipSuccess) return e;
    }
    return hipSuccess;
}

// The most bytes of sums of divided tiles: three steps have every kind of launch.
int64_t part_bytes(const tbn_muon_tensor* t, int n, const Place* at) {
    int64_t most = 0;
    (void)muon_launches(t, n, at, nullptr, 3, [&](const Launch& l) {
        most = std::max(most, (int64_t)l.blocks * 2 * l.tile * l.tile * 4);
        return hipSuccess;
    });
    return round_up(most, 256);
}

constexpr int kMostLaunches = kMuonSteps / 2 * 7;

int64_t place_all(const tbn_muon_tensor* t, int n, Place* at) {
    int64_t end = 0;
    for (int i = 0; i < n; ++i) {
        at[i] = place_of(t[i], end);
        end = at[i].end;
    }
    return end;
}

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
    Place at[kMuonMatrices];
    const int64_t end = place_all(t, n, at);
    return end + part_bytes(t, n, at) + (table_words<StartJob>(n) + kMostLaunches * table_words<Job>(n)) * 4;
}

hipError_t launch_muon_group(const tbn_muon_tensor* t, int n, const MuonHyper& h, uint8_t* ws, hipStream_t s) {
    Place at[kMuonMatrices];
    const int64_t end = place_all(t, n, at);
    f32x4* const part = reinterpret_cast<f32x4*>(ws + end);
    uint32_t* table = reinterpret_cast<uint32_t*>(ws + end + part_bytes(t, n, at));
    hipError_t e;

    // the tables of all launches, then the launches
    StartJob start[kMuonMatrices] = {};
    uint32_t blocks = 0, tiles = 0;
    for (int i = 0; i < n; ++i) {
        StartJob& j = start[i];
        const Place& p = at[i];
        j.m = t[i].m;
        j.g = t[i].g;
        j.rows = t[i].rows;
        j.cols = t[i].cols;
        j.direct = ws + (p.tall ? p.xt[0] : p.x[0]);
        j.turned = ws + (p.tall ? p.x[0] : p.xt[0]);
        j.pitch_d = (uint32_t)(p.tall ? p.mp : p.np);
        j.pitch_t = (uint32_t)(p.tall ? p.np : p.mp);
        j.norm = reinterpret_cast<double*>(ws + p.norm);
        const int64_t parts = ((int64_t)j.rows * j.cols + 4095) / 4096;
        j.parts = (uint32_t)(parts < 256 ? parts : 256);
        j.first_tile = blocks;  // of the first kernel
        j.first = tiles;        // of the second
        blocks += j.parts;
        tiles += (uint32_t)(tiles_of(j.rows, 64) * tiles_of(j.cols, 64));
    }
    Writer to(table, s);
    write_table(to, start, n);
    Plan plans[kMostLaunches];
    int launches = 0;
    e = muon_launches(t, n, at, ws, h.steps, [&](const Launch& l) {
        write_table(to, l.job, l.n);
        plans[launches++] = l;
        return to.e;
    });
    to.flush();
    if (e != hipSuccess || (e = to.e) != hipSuccess) return e;

    Start st = {};
    st.table = table_at<StartJob>(table, n);
    st.momentum = h.momentum;
    st.eps = h.eps;
    st.nesterov = h.nesterov;
    table += table_words<StartJob>(n);
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
        Products a = {};
        a.table = table_at<Job>(table, n);
        a.part = part;
        a.lr = h.lr;
        a.lr_dev = h.lr_dev;
        a.whole = p.whole;
        a.stages = p.stages;
        a.blocks = p.blocks;
        table += table_words<Job>(n);
        if ((e = launch_tiles<false>(a, p.tile, p.whole + p.blocks, s)) != hipSuccess) return e;
        if (p.blocks && (e = launch_tiles<true>(a, p.tile, p.tiles - p.whole, s)) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tbn
