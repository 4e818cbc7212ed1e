// tbn_muon.hip -- Muon's step on the real weights: momentum, the update made orthogonal by Newton-Schulz products, and the
// weights moved along it, for many matrices in the launches of one.
//
// With X the update over its Frobenius norm, m x n, m <= n (a taller matrix is taken transposed), each step is
//   A = X X^T,  B = b A + c A A,  X = a X + B X,   (a, b, c) = (3.4445, -4.7750, 2.0315),
// which moves every singular value s to a s + b s^3 + c s^5 and, five times, into the neighbourhood of 1.
//
//   * Every factor is held as two fp16 halves (22 bits) and multiplied on the matrix cores with three products (tbn_nt.h), at a
//     third of the matrix rate; sums are fp32.  One fp16 or bf16 product in place of the three would leave 2^-9 to 2^-12 of X,
//     which small singular values carry through five steps that each multiply them by 3.4.  The halves are scaled by powers of
//     two (X by 2^12, A by 2^14, B by 2^13) so that both keep their bits: |X| <= 1.21, |A| <= 1.47, |B| <= 2.81.
//   * Rows are groups of 32 values, 64 bytes of leading and 64 of trailing halves, zeros behind the last: the 128 bytes of
//     a stage.
//   * A and B are symmetric: tiles on and below the diagonal are computed and written to both places.
//   * B X needs the rows of X^T: every X is written in both layouts, by the epilogue that has the tile in LDS anyway.
#include "tbn_kernels.h"
#include "tbn_nt.h"

namespace tbn {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kXScale = 4096.0f;

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
__device__ __forceinline__ void get8(const uint8_t* p, float (&v)[8]) {
    const f16x8 hi = *reinterpret_cast<const f16x8*>(p), lo = *reinterpret_cast<const f16x8*>(p + 64);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)hi[e] + (float)lo[e];
}
// Byte of value c (a multiple of 8) in a row.
__device__ __forceinline__ int64_t place(int64_t c) { return c / 32 * 128 + c % 32 * 2; }

template <typename T>
__device__ __forceinline__ const T& job_of(const T* jobs, int n, uint32_t block) {
    int i = 0;
    while (i + 1 < n && block >= jobs[i + 1].first) ++i;
    return jobs[i];
}

// ---- momentum and the update's norm ------------------------------------------------------
// m = momentum m + g; the sum of the squares of u = g + momentum m (or of m), in 64 bits, a partial sum a block.
template <bool BF16>
__device__ __forceinline__ float grad_at(const void* g, int64_t i) {
    return BF16 ? bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(g)[i]) : reinterpret_cast<const float*>(g)[i];
}

template <bool BF16>
__global__ __launch_bounds__(256) void muon_momentum_kernel(const MuonStart a) {
    __shared__ double sums[4];
    const MuonStartJob& j = job_of(a.job, a.n, blockIdx.x);
    const uint32_t block = blockIdx.x - j.first;
    const int64_t count = (int64_t)j.rows * j.cols;
    double sum = 0.0;
    const bool wide = ((reinterpret_cast<uintptr_t>(j.m) | reinterpret_cast<uintptr_t>(j.g)) & 15) == 0;
    const int64_t vecs = wide ? count / 4 : 0, stride = (int64_t)j.blocks * 256;
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < vecs; i += stride) {
        f32x4 m = reinterpret_cast<const f32x4*>(j.m)[i], g;
        if constexpr (BF16) {
            const u32x2 r = reinterpret_cast<const u32x2*>(j.g)[i];
            g = f32x4{bf16_bits_to_f32(r.x & 0xFFFFu), __uint_as_float(r.x & 0xFFFF0000u), bf16_bits_to_f32(r.y & 0xFFFFu),
                      __uint_as_float(r.y & 0xFFFF0000u)};
        } else {
            g = reinterpret_cast<const f32x4*>(j.g)[i];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = a.momentum * m[e] + g[e];
            const double u = a.nesterov ? g[e] + a.momentum * m[e] : m[e];
            sum += u * u;
        }
        reinterpret_cast<f32x4*>(j.m)[i] = m;
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
__global__ __launch_bounds__(256) void muon_start_kernel(const MuonStart a) {
    __shared__ float tile[64][65];
    __shared__ double sums[4];
    const MuonStartJob& j = job_of(a.job, a.n, blockIdx.x);
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
    // thread (r, 8 values): two passes of 32 rows
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int r = 32 * p + tid / 8, c = tid % 8 * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = 0.0f;
            if (r0 + r < j.rows && c0 + c + e < j.cols) {
                const int64_t i = (int64_t)(r0 + r) * j.cols + c0 + c + e;
                const float m = j.m[i];
                v[e] = (a.nesterov ? grad_at<BF16>(j.g, i) + a.momentum * m : m) * inv;
            }
            tile[r][c + e] = v[e];
        }
        if (r0 + r < j.rows && c0 + c < (j.cols + 31) / 32 * 32) put8(j.direct + (r0 + r) * (int64_t)j.pitch_d + place(c0 + c), v);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int c = tid % 64, r = 32 * p + tid / 64 * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[r + e][c];
        if (c0 + c < j.cols && r0 + r < (j.rows + 31) / 32 * 32) put8(j.turned + (c0 + c) * (int64_t)j.pitch_t + place(r0 + r), v);
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

// FINISH: the sums of a tile's parts are added in place of its product (the block that computed a part left it as it held it).
template <int BT, int WAVES_M, int WAVES_N, int STAGES, bool FINISH>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N, BT >= 256 ? 1 : 2) void muon_product_kernel(const MuonProducts a) {
    typedef NtLoop<BT, BT, WAVES_M, WAVES_N, STAGES, NtF16x2> Loop;
    constexpr int TM = Loop::TM, TN = Loop::TN, PITCH = Loop::WN + 4;
    static_assert(Loop::BYTES >= Loop::WAVES * 32 * PITCH * 4, "staging fits in the ring");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[Loop::BYTES];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t block = FINISH ? blockIdx.x : (uint32_t)xcd_remap(blockIdx.x, gridDim.x);
    const MuonJob& j = job_of(a.job, a.n, block);
    const uint32_t work = block - j.first;
    const uint32_t tile = FINISH ? work : work / j.splits, split = work - tile * (FINISH ? 1 : j.splits);
    if (FINISH && j.splits == 1) return;  // its product wrote it
    const uint32_t tiles_m = (uint32_t)(j.M + BT - 1) / BT, tiles_n = (uint32_t)(j.N + BT - 1) / BT;
    uint32_t tm, tn;
    if (j.symmetric)
        lower_tile(tile, &tm, &tn);
    else
        nt_tile(tile, tiles_m, tiles_n, &tm, &tn);
    const int32_t m0 = (int32_t)(tm * BT), n0 = (int32_t)(tn * BT);

    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][t][v] = 0.0f;
    constexpr int QUADS = TM * TN * 4;
    if constexpr (FINISH) {
        for (uint32_t s = 0; s < j.splits; ++s) {
            const f32x4* src = j.part + ((int64_t)(tile * j.splits + s) * QUADS * Loop::WAVES + wave) * 64 + lane;
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
        const int stages = (int)(j.pitch / 128);
        Loop::run(ra, rb, smem, (int)(stages * split / j.splits), (int)(stages * (split + 1) / j.splits), j.pitch, wave, lane, acc);
        if (j.splits > 1) {
            f32x4* dst = j.part + ((int64_t)(tile * j.splits + split) * QUADS * Loop::WAVES + wave) * 64 + lane;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int t = 0; t < TN; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        dst[((i * TN + t) * 4 + g) * Loop::WAVES * 64] =
                            f32x4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
            return;
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
                for (int e = 0; e < 8; ++e) v[e] = j.p * v[e] + j.q * x[e];
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
            constexpr int ITEMS = Loop::WN * 4 / 64;
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const int item = 64 * k + lane, c = item % Loop::WN, r = item / Loop::WN * 8;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = stage[(r + e) * PITCH + c];
                const int32_t n = n0 + wn * Loop::WN + c;
                if (n < j.N && row0 + r < Mp) put8(j.turned + (int64_t)n * j.pitch_t + place(row0 + r), v);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <bool FINISH>
hipError_t launch_products(const MuonProducts& a, int tile, uint32_t blocks, hipStream_t s) {
    if (tile == 256)
        hipLaunchKernelGGL((muon_product_kernel<256, 2, 2, 2, FINISH>), dim3(blocks), dim3(256), 0, s, a);
    else if (tile == 128)
        hipLaunchKernelGGL((muon_product_kernel<128, 2, 2, 2, FINISH>), dim3(blocks), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((muon_product_kernel<64, 2, 2, 4, FINISH>), dim3(blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// A matrix in the workspace: its sides, m <= n, and where its arrays begin.
struct Place {
    int64_t m, n, mp, np;  // mp, np: bytes of a row of m (n) values
    int64_t x[2], xt[2], a, b, part, norm, end;
    uint32_t splits;
};

// The tile: large ones move fewer bytes through LDS for a product, small ones fill the GPU.
int tile_for(const tbn_muon_tensor* t, int n) {
    int64_t tiles[2] = {0, 0};
    for (int i = 0; i < n; ++i)
        for (int k = 0; k < 2; ++k) tiles[k] += tiles_of(t[i].rows, k ? 128 : 256) * tiles_of(t[i].cols, k ? 128 : 256);
    return tiles[0] >= 192 ? 256 : tiles[1] >= 256 ? 128 : 64;
}

Place place_of(const tbn_muon_tensor& t, int64_t at, int tile, int64_t lower_tiles) {
    Place p;
    p.m = t.rows < t.cols ? t.rows : t.cols;
    p.n = t.rows < t.cols ? t.cols : t.rows;
    p.mp = round_up(p.m, 32) * 4;
    p.np = round_up(p.n, 32) * 4;
    auto take = [&](int64_t bytes) {
        const int64_t was = at;
        at += round_up(bytes, 256);
        return was;
    };
    for (int i = 0; i < 2; ++i) p.x[i] = take(p.m * p.np), p.xt[i] = take(p.n * p.mp);
    p.a = take(p.m * p.mp);
    p.b = take(p.m * p.mp);
    // the Gram products reduce over the long side: split where their tiles are few
    const int64_t stages = p.np / 128, lower = tiles_of(p.m, tile) * (tiles_of(p.m, tile) + 1) / 2;
    int64_t splits = lower_tiles >= 256 ? 1 : 512 / lower_tiles;
    if (splits > stages / 8) splits = stages / 8;
    p.splits = (uint32_t)(splits < 1 ? 1 : splits);
    p.part = p.splits > 1 ? take(lower * p.splits * tile * tile * 4) : 0;
    p.norm = take(256 * 8);
    p.end = at;
    return p;
}

int64_t lower_of(const tbn_muon_tensor* t, int n, int tile) {
    int64_t sum = 0;
    for (int i = 0; i < n; ++i) {
        const int64_t k = tiles_of(t[i].rows < t[i].cols ? t[i].rows : t[i].cols, tile);
        sum += k * (k + 1) / 2;
    }
    return sum;
}

}  // namespace

// Matrices that go together: up to kMuonJobs of them, and no more than 2^25 values (one larger matrix goes alone).
int muon_group(const tbn_muon_tensor* t, int n) {
    int64_t sum = 0;
    for (int i = 0; i < n; ++i) {
        sum += t[i].rows * (int64_t)t[i].cols;
        if (i == kMuonJobs || (i && sum > (1 << 25))) return i;
    }
    return n;
}

int64_t muon_group_bytes(const tbn_muon_tensor* t, int n) {
    const int tile = tile_for(t, n);
    const int64_t lower = lower_of(t, n, tile);
    int64_t at = 0;
    for (int i = 0; i < n; ++i) at = place_of(t[i], at, tile, lower).end;
    return at;
}

hipError_t launch_muon_group(const tbn_muon_tensor* t, int n, const MuonHyper& h, uint8_t* ws, hipStream_t s) {
    const int tile = tile_for(t, n);
    const int64_t lower = lower_of(t, n, tile);
    Place at[kMuonJobs];
    int64_t end = 0;
    for (int i = 0; i < n; ++i) {
        at[i] = place_of(t[i], end, tile, lower);
        end = at[i].end;
    }
    hipError_t e;

    MuonStart st = {};
    st.n = n;
    st.momentum = h.momentum;
    st.eps = h.eps;
    st.nesterov = h.nesterov;
    uint32_t first = 0;
    for (int i = 0; i < n; ++i) {
        MuonStartJob& j = st.job[i];
        const bool tall = t[i].rows > t[i].cols;
        j.m = t[i].m;
        j.g = t[i].g;
        j.rows = t[i].rows;
        j.cols = t[i].cols;
        j.direct = ws + (tall ? at[i].xt[0] : at[i].x[0]);
        j.turned = ws + (tall ? at[i].x[0] : at[i].xt[0]);
        j.pitch_d = (uint32_t)(tall ? at[i].mp : at[i].np);
        j.pitch_t = (uint32_t)(tall ? at[i].np : at[i].mp);
        j.norm = reinterpret_cast<double*>(ws + at[i].norm);
        const int64_t count = (int64_t)j.rows * j.cols, blocks = (count + 4095) / 4096;
        j.blocks = j.parts = (uint32_t)(blocks < 256 ? blocks : 256);
        j.first = first;
        first += j.blocks;
    }
    if (h.g_f32)
        hipLaunchKernelGGL((muon_momentum_kernel<false>), dim3(first), dim3(256), 0, s, st);
    else
        hipLaunchKernelGGL((muon_momentum_kernel<true>), dim3(first), dim3(256), 0, s, st);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    first = 0;
    for (int i = 0; i < n; ++i) {
        st.job[i].first = first;
        first += (uint32_t)(tiles_of(t[i].rows, 64) * tiles_of(t[i].cols, 64));
    }
    if (h.g_f32)
        hipLaunchKernelGGL((muon_start_kernel<false>), dim3(first), dim3(256), 0, s, st);
    else
        hipLaunchKernelGGL((muon_start_kernel<true>), dim3(first), dim3(256), 0, s, st);
    if ((e = hipGetLastError()) != hipSuccess) return e;

    for (int step = 0; step < h.steps; ++step) {
        const int now = step & 1, next = now ^ 1;
        MuonProducts gram = {}, poly = {}, apply = {};
        gram.n = poly.n = apply.n = n;
        apply.lr = h.lr;
        apply.lr_dev = h.lr_dev;
        uint32_t first_g = 0, first_p = 0, first_a = 0;
        bool split = false;
        for (int i = 0; i < n; ++i) {
            const Place& p = at[i];
            const uint32_t low = (uint32_t)(tiles_of(p.m, tile) * (tiles_of(p.m, tile) + 1) / 2);
            MuonJob& g = gram.job[i];
            g.a = g.b = ws + p.x[now];
            g.pitch = (uint32_t)p.np;
            g.M = g.N = (int32_t)p.m;
            g.direct = g.turned = ws + p.a;
            g.pitch_o = g.pitch_t = (uint32_t)p.mp;
            g.p = 0x1p-10f;  // 2^24 of the halves to 2^14
            g.symmetric = 1;
            g.splits = p.splits;
            g.part = reinterpret_cast<f32x4_t*>(ws + p.part);
            g.first = first_g;
            first_g += low * p.splits;
            split |= p.splits > 1;
            MuonJob& q = poly.job[i];
            q.a = q.b = q.aux = ws + p.a;
            q.pitch = q.pitch_o = q.pitch_t = (uint32_t)p.mp;
            q.M = q.N = (int32_t)p.m;
            q.direct = q.turned = ws + p.b;
            q.p = kC * 0x1p-15f;  // 2^28 and 2^14 to 2^13
            q.q = kB * 0.5f;
            q.symmetric = 1;
            q.splits = 1;
            q.first = first_p;
            first_p += low;
            MuonJob& x = apply.job[i];
            x.pitch = (uint32_t)p.mp;
            x.p = 0x1p-13f;  // 2^25 to 2^12
            x.q = kA;
            x.splits = 1;
            const bool tall = t[i].rows > t[i].cols, last = step + 1 == h.steps;
            if (last && tall) {  // the product transposed, along the rows of w
                x.a = ws + p.xt[now];
                x.b = ws + p.b;
                x.aux = ws + p.xt[now];
                x.pitch_o = (uint32_t)p.mp;
                x.M = (int32_t)p.n;
                x.N = (int32_t)p.m;
            } else {
                x.a = ws + p.b;
                x.b = ws + p.xt[now];
                x.aux = ws + p.x[now];
                x.pitch_o = (uint32_t)p.np;
                x.M = (int32_t)p.m;
                x.N = (int32_t)p.n;
            }
            if (last) {
                x.w = t[i].w;
                x.weight_decay = t[i].weight_decay;
                x.scale = t[i].scale;
            } else {
                x.direct = ws + p.x[next];
                x.turned = ws + p.xt[next];
                x.pitch_t = (uint32_t)p.mp;
            }
            x.first = first_a;
            first_a += (uint32_t)(tiles_of(x.M, tile) * tiles_of(x.N, tile));
        }
        if ((e = launch_products<false>(gram, tile, first_g, s)) != hipSuccess) return e;
        if (split) {
            uint32_t f = 0;
            for (int i = 0; i < n; ++i) {
                gram.job[i].first = f;
                f += (uint32_t)(tiles_of(at[i].m, tile) * (tiles_of(at[i].m, tile) + 1) / 2);
            }
            if ((e = launch_products<true>(gram, tile, f, s)) != hipSuccess) return e;
        }
        if ((e = launch_products<false>(poly, tile, first_p, s)) != hipSuccess) return e;
        if ((e = launch_products<false>(apply, tile, first_a, s)) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tbn
