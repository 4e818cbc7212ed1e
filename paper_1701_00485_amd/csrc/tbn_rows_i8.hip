// tbn_rows_i8.hip -- products in 8-bit integers with a scale for each row of both operands (each token, each channel):
// the rows made 8-bit, and y[m][n] = act(scale_m scale_n sum over k of q[m][k] w[n][k] + bias_n + residual), the sum exact.
#include <algorithm>
#include <type_traits>

#include "tbn_kernels.h"
#include "tbn_nt.h"

namespace tbn {

namespace {

// ---- rows to 8 bits ----------------------------------------------------------------------
// scale = t fp32(1/127) with t the row's largest finite magnitude, q = x (127 / t) rounded to the nearest, ties to even, and
// held within +-127; NaN gives 0.  A row whose t is below 2^-100 has scale 0 and zeros (127 / t would leave fp32's range).
// One pass over x where a thread can hold its part of the row (VECS pieces of 8 values), else two, the second from
// the caches.  Bound by memory (8192 x 4096 bf16 in 18.6 us, 5.4 TB/s), in short rows by the sums' and the scale's latency.
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

template <bool F32>
__device__ __forceinline__ void load8(const void* x, int64_t at, int n, bool wide, float (&v)[8]) {
    if (n >= 8 && wide) {
        if constexpr (F32) {
            const f32x4* p = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(x) + at);
            const f32x4 a = p[0], b = p[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
        } else {
            const u32x4 r = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(x) + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[2 * e] = bf16_bits_to_f32(r[e] & 0xFFFFu), v[2 * e + 1] = __uint_as_float(r[e] & 0xFFFF0000u);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    if (n <= 0) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e < n) v[e] = F32 ? reinterpret_cast<const float*>(x)[at + e] : bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(x)[at + e]);
    }
}

__device__ __forceinline__ float top8(const float (&v)[8], float t) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float m = fabsf(v[e]);
        t = m <= 3.402823466e38f ? fmaxf(t, m) : t;  // neither infinities nor NaN
    }
    return t;
}

// Added to a value within 2^22, 1.5 2^23 rounds it to the nearest, ties to even, into the low bits.
__device__ __forceinline__ u32x2_t codes8(const float (&v)[8], float inv) {
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float q = v[e] * inv;
        q = q == q ? q : 0.0f;  // of NaN, and of an infinity where inv is 0
        b[e] = __float_as_uint(fminf(fmaxf(q, -127.0f), 127.0f) + 12582912.0f);
    }
    u32x2_t r;
#pragma unroll
    for (int h = 0; h < 2; ++h)
        r[h] = __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400u) | __builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x04000c0cu);
    return r;
}

// THREADS of a row, 256 / THREADS rows a block.
template <bool F32, int THREADS, int VECS>
__global__ __launch_bounds__(256) void rows_i8_kernel(const void* __restrict__ x, int64_t rows, int32_t c, int32_t pitch, bool wide,
                                                      int8_t* __restrict__ q, float* __restrict__ scale) {
    __shared__ float tops[4];
    const int tid = threadIdx.x % THREADS;
    const int64_t row = (int64_t)blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS;
    if (THREADS < 256 && row >= rows) return;  // (a wave a row: no barrier follows)
    const int64_t x0 = row * c, q0 = row * pitch;
    const int vecs = pitch / 8;
    float v[VECS ? VECS : 1][8];
    float t = 0.0f;
    if constexpr (VECS > 0) {
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            const int e = (tid + THREADS * j) * 8;
            load8<F32>(x, x0 + e, c - e, wide, v[j]);
        }
#pragma unroll
        for (int j = 0; j < VECS; ++j) t = top8(v[j], t);
    } else {
        for (int i = tid; i < vecs; i += THREADS) {
            load8<F32>(x, x0 + 8 * i, c - 8 * i, wide, v[0]);
            t = top8(v[0], t);
        }
    }
#pragma unroll
    for (int d = 32; d; d /= 2) t = fmaxf(t, __shfl_xor(t, d, 64));
    if constexpr (THREADS == 256) {
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = t;
        __syncthreads();
        t = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    }
    const float inv = t >= 0x1p-100f ? 127.0f / t : 0.0f;
    if (tid == 0) scale[row] = inv > 0.0f ? t * (1.0f / 127.0f) : 0.0f;
    if constexpr (VECS > 0) {
#pragma unroll
        for (int j = 0; j < VECS; ++j)
            if (tid + THREADS * j < vecs) *reinterpret_cast<u32x2_t*>(q + q0 + (tid + THREADS * j) * 8) = codes8(v[j], inv);
    } else {
        for (int i = tid; i < vecs; i += THREADS) {
            load8<F32>(x, x0 + 8 * i, c - 8 * i, wide, v[0]);
            *reinterpret_cast<u32x2_t*>(q + q0 + 8 * i) = codes8(v[0], inv);
        }
    }
}

// ---- what follows the sums ---------------------------------------------------------------
// y of channel n of row m from its sum, the row's and the channel's scale and its bias.
__device__ __forceinline__ void finish1(const RowsI8Args& a, int64_t m, int32_t n, float s, float sx, float sw, float bias) {
    const int64_t o = m * a.n + n;
    float v = s * (sx * sw) + bias;
    if (a.residual) v += a.y_f32 ? reinterpret_cast<const float*>(a.residual)[o] : bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(a.residual)[o]);
    if (a.relu) v = v > 0.0f || v != v ? v : 0.0f;
    if (a.y_f32)
        reinterpret_cast<float*>(a.y)[o] = v;
    else
        reinterpret_cast<uint16_t*>(a.y)[o] = (uint16_t)f32_to_bf16_bits(v);
}

// ... of 8 consecutive channels, `EVEN`: 16-byte aligned (n % 8 == 0).
template <bool EVEN>
__device__ __forceinline__ void finish8(const RowsI8Args& a, int64_t m, int32_t n0, const float (&s)[8], float sx, const float (&sw)[8],
                                        const float (&bias)[8]) {
    typedef typename std::conditional<EVEN, f32x4, f32x4_at4>::type V32;
    typedef typename std::conditional<EVEN, u32x4, u32x4_at2>::type V16;
    const int64_t o = m * a.n + n0;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[e] * (sx * sw[e]) + bias[e];
    if (a.residual && a.y_f32) {
        const V32* r = reinterpret_cast<const V32*>(reinterpret_cast<const float*>(a.residual) + o);
        const f32x4 lo = r[0], hi = r[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += lo[e], v[4 + e] += hi[e];
    } else if (a.residual) {
        const u32x4 r = *reinterpret_cast<const V16*>(reinterpret_cast<const uint16_t*>(a.residual) + o);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[2 * e] += bf16_bits_to_f32(r[e] & 0xFFFFu), v[2 * e + 1] += __uint_as_float(r[e] & 0xFFFF0000u);
    }
    if (a.relu) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] > 0.0f || v[e] != v[e] ? v[e] : 0.0f;
    }
    if (a.y_f32) {
        V32* p = reinterpret_cast<V32*>(reinterpret_cast<float*>(a.y) + o);
        p[0] = f32x4{v[0], v[1], v[2], v[3]};
        p[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        *reinterpret_cast<V16*>(reinterpret_cast<uint16_t*>(a.y) + o) =
            u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
}

// ---- many rows ---------------------------------------------------------------------------
// A tile of BM x BN outputs a block, 128 values a stage (tbn_nt.h); the matrix instructions bound it: 8192 x 4096 x 8192 in 241 us,
// 2.28 PFLOP/s, 256 sums a lane of four waves (by eight waves, twice the operand reads from LDS: 286).  GROUPS groups of such waves, each
// with a part of the stages and a ring of its own, serve tiles that are too few to fill the GPU.
template <int BM, int BN, int WAVES_M, int WAVES_N, int STAGES, int GROUPS>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N * GROUPS, BM * BN >= 65536 || GROUPS > 1 ? 1 : BM * BN >= 8192 ? 2 : 3) void matmul_i8_kernel(const RowsI8Args a) {
    typedef NtLoop<BM, BN, WAVES_M, WAVES_N, STAGES, NtI8> Loop;
    constexpr int PITCH = Loop::WN + 4;  // of a staged row, in floats
    static_assert(Loop::BYTES >= Loop::WAVES * 32 * PITCH * 4 + (BM + 2 * BN) * 4, "staging fits in the ring");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[GROUPS * Loop::BYTES];
    const int lane = threadIdx.x & 63;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * Loop::WAVES));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - group * Loop::WAVES;
    const uint32_t tiles_n = (uint32_t)((a.n + BN - 1) / BN), tiles_m = (uint32_t)((a.rows + BM - 1) / BM);
    uint32_t tm, tn;
    nt_tile((uint32_t)xcd_remap(blockIdx.x, gridDim.x), tiles_m, tiles_n, &tm, &tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int32_t n0 = (int32_t)(tn * BN);

    typename Loop::RowsA ra;
    typename Loop::RowsB rb;
    ra.init(a.x, m0, a.rows, (uint32_t)a.c, wave, lane, Loop::copy_seg(wave, lane));
    rb.init(a.w, n0, a.n, (uint32_t)a.c, wave, lane, Loop::copy_seg(wave, lane));
    i32x16 acc[Loop::TM][Loop::TN];
#pragma unroll
    for (int i = 0; i < Loop::TM; ++i)
#pragma unroll
        for (int t = 0; t < Loop::TN; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][t][v] = 0;
    const int stages = (a.c + 127) / 128, each = (stages + GROUPS - 1) / GROUPS;
    Loop::run(ra, rb, smem + group * Loop::BYTES, min(group * each, stages), min((group + 1) * each, stages), each, (uint32_t)a.c, wave, lane, acc);
    nt_join<GROUPS, Loop>(smem, group, wave, lane, acc);

    // the tile's scales and biases, behind the waves' staging
    float* const row_scale = reinterpret_cast<float*>(smem) + Loop::WAVES * 32 * PITCH;
    float* const col_scale = row_scale + BM;
    float* const col_bias = col_scale + BN;
    for (int i = threadIdx.x; i < BM + BN; i += 64 * Loop::WAVES * GROUPS) {
        if (i < BM) {
            row_scale[i] = m0 + i < a.rows ? a.x_scale[m0 + i] : 0.0f;
        } else {
            const int32_t n = n0 + (i - BM);
            const bool in = n < a.n;
            row_scale[i] = in ? (a.scale ? a.w_scale[n] * a.scale[n] : a.w_scale[n]) : 0.0f;
            row_scale[i + BN] = in && a.bias ? a.bias[n] : 0.0f;
        }
    }
    __syncthreads();
    if (group) return;
    // a wave turns each 32 rows of its tile in LDS and writes them with 16-byte stores
    float* stage = reinterpret_cast<float*>(smem) + wave * 32 * PITCH;
    const int wm = wave / WAVES_N, wn = wave % WAVES_N, half = lane >> 5, l32 = lane & 31;
    constexpr int CG = Loop::WN / 8, RPP = 64 / CG;
    const bool even = a.n % 8 == 0;  // y and the residual begin 16-byte aligned
    float sw[8], bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sw[e] = col_scale[wn * Loop::WN + 8 * (lane % CG) + e], bias[e] = col_bias[wn * Loop::WN + 8 * (lane % CG) + e];
#pragma unroll
    for (int i = 0; i < Loop::TM; ++i) {
#pragma unroll
        for (int t = 0; t < Loop::TN; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(stage + l32 * PITCH + 32 * t + 8 * g + 4 * half) =
                    f32x4{(float)acc[i][t][4 * g], (float)acc[i][t][4 * g + 1], (float)acc[i][t][4 * g + 2], (float)acc[i][t][4 * g + 3]};
        __builtin_amdgcn_wave_barrier();
        const int col = n0 + wn * Loop::WN + 8 * (lane % CG);
        auto row8 = [&](int p, auto then) {
            const int r = p * RPP + lane / CG;
            const int64_t m = m0 + wm * Loop::WM + 32 * i + r;
            const f32x4* s = reinterpret_cast<const f32x4*>(stage + r * PITCH + 8 * (lane % CG));
            const f32x4 lo = s[0], hi = s[1];
            const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (m < a.rows && col < a.n) then(m, v, row_scale[wm * Loop::WM + 32 * i + r]);
        };
        if (even) {
#pragma unroll
            for (int p = 0; p < 32 / RPP; ++p) row8(p, [&](int64_t m, const float(&v)[8], float sx) { finish8<true>(a, m, col, v, sx, sw, bias); });
        } else {
#pragma unroll 1
            for (int p = 0; p < 32 / RPP; ++p)
                row8(p, [&](int64_t m, const float(&v)[8], float sx) {
                    if (col + 8 <= a.n) {
                        finish8<false>(a, m, col, v, sx, sw, bias);
                    } else {
#pragma unroll
                        for (int e = 0; e < 7; ++e)
                            if (col + e < a.n) finish1(a, m, col + e, v[e], sx, sw[e], bias[e]);
                    }
                });
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- up to 16 rows -----------------------------------------------------------------------
// The weights are read once and bound it: 8192 -> 28672 for 1 row in 42.2 us, 5.6 TB/s, for 16 in 43.9.  A step is 128 bytes of each of
// 16 channels: lane (f = l % 16, q = l / 16) reads bytes 32 q .. 32 q + 31 of channel f's as two 16-byte pieces, a matrix instruction
// each, and of row f of x the same bytes (the order of the values in a sum of integers is free).

// Of up to 2048 SL values: a block, one a compute unit, owns a range of the groups of 16 channels.  Wave (i, j) of its KS x GS keeps x's
// steps i, i + KS, .. of 128 bytes in registers and streams the weights of groups j, j + GS, .., two ahead; the KS sums of an
// output meet in LDS, four groups a wave at a time.  Without x in registers (matvec_i8_kernel): 44.9 us and, for 16 rows, 67.7.
template <int SL>
__global__ __launch_bounds__(1024) void stream_i8_kernel(const RowsI8Args a, int KS, int GS) {
    constexpr int BATCH = 4, AHEAD = 2;
    __shared__ __attribute__((aligned(16))) int32_t part[BATCH * 16 * 256];  // [BATCH GS groups][KS][16 rows][16 channels]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = wave / KS, i = wave - j * KS;
    const int f = lane & 15, q = lane >> 4;
    const int groups = (a.n + 15) / 16;
    const int g0 = (int)((int64_t)groups * blockIdx.x / gridDim.x), g1 = (int)((int64_t)groups * (blockIdx.x + 1) / gridDim.x);
    const int rounds = (g1 - g0 + GS - 1) / GS;
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(a.x), 0, (int)(a.rows * a.c), 0x00020000);
    i32x4 w[AHEAD][SL][2], x[SL][2];
    auto at = [&](int s, int u) { return (i + KS * s) * 128 + 32 * q + 16 * u; };
    auto load = [&](int d, int r) {
        const int8_t* const p = a.w + (int64_t)min((g0 + j + GS * r) * 16 + f, a.n - 1) * a.c;
#pragma unroll
        for (int s = 0; s < SL; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) w[d][s][u] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p + (at(s, u) < a.c ? at(s, u) : 0)));
    };
#pragma unroll
    for (int s = 0; s < SL; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u) {  // zeros past the row's end and past the last row
            const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rx, at(s, u) < a.c ? f * a.c + at(s, u) : (int)0x80000000, 0, 0);
            x[s][u] = __builtin_bit_cast(i32x4, v);
        }
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
        if (d < rounds) load(d, d);
    for (int r0 = 0; r0 < rounds; r0 += BATCH) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (r0 + b >= rounds) break;
            i32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < SL; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[b % AHEAD][s][u], x[s][u], acc, 0, 0, 0);
            if (r0 + b + AHEAD < rounds) load(b % AHEAD, r0 + b + AHEAD);
            // lane (f, q) holds row f, channels 4 q .. 4 q + 3
            *reinterpret_cast<i32x4*>(part + ((b * GS + j) * KS + i) * 256 + f * 16 + 4 * q) = acc;
        }
        __syncthreads();
        const int outputs = min(BATCH, rounds - r0) * GS * 256;
        for (int o = threadIdx.x; o < outputs; o += 64 * KS * GS) {
            const int row = o / 16 % 16, n = (g0 + GS * r0 + o / 256) * 16 + o % 16;
            if (row >= a.rows || n >= min(g1 * 16, a.n)) continue;
            const int32_t* const v = part + o / 256 * KS * 256 + o % 256;
            int32_t t = v[0];
#pragma unroll 4
            for (int k = 1; k < KS; ++k) t += v[256 * k];
            finish1(a, row, n, (float)t, a.x_scale[row], a.scale ? a.w_scale[n] * a.scale[n] : a.w_scale[n], a.bias ? a.bias[n] : 0.0f);
        }
        if (r0 + BATCH < rounds) __syncthreads();
    }
}

template <int SL>
hipError_t launch_stream(const RowsI8Args& a, hipStream_t s) {
    const int steps = (a.c + 127) / 128, groups = (a.n + 15) / 16;
    const int KS = (steps + SL - 1) / SL, GS = std::max(1, std::min((groups + 255) / 256, 16 / KS));
    hipLaunchKernelGGL((stream_i8_kernel<SL>), dim3((unsigned)std::min(groups, 256)), dim3(64 * KS * GS), 0, s, a, KS, GS);
    return hipGetLastError();
}

// Of more values: a block owns 16 channels, each of its WAVES waves a range of the values of which x is read with the weights.
template <int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void matvec_i8_kernel(const RowsI8Args a) {
    __shared__ i32x4 sums[WAVES][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int f = lane & 15, q = lane >> 4;
    const int32_t n0 = (int32_t)blockIdx.x * 16;
    const int steps = (a.c + 127) / 128;
    const int s0 = (int)((int64_t)steps * wave / WAVES), s1 = (int)((int64_t)steps * (wave + 1) / WAVES);
    const int8_t* const wp = a.w + (int64_t)min(n0 + f, a.n - 1) * a.c;
    const bool have = f < a.rows;
    const int8_t* const xp = a.x + (int64_t)(have ? f : 0) * a.c;
    i32x4 acc = {0, 0, 0, 0};
    i32x4 wv[DEPTH][2], xv[DEPTH][2];
    auto load = [&](int d, int s) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = s * 128 + 32 * q + 16 * u;
            const bool in = k < a.c;
            const int kk = in ? k : 0;
            wv[d][u] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(wp + kk));
            xv[d][u] = i32x4{0, 0, 0, 0};
            if (have && in) xv[d][u] = *reinterpret_cast<const i32x4*>(xp + kk);
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (s0 + d < s1) load(d, s0 + d);
    for (int s = s0; s < s1; s += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (s + d >= s1) break;
#pragma unroll
            for (int u = 0; u < 2; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[d][u], xv[d][u], acc, 0, 0, 0);
            if (s + d + DEPTH < s1) load(d, s + d + DEPTH);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    // lane (f, q) holds row f, channels 4 q .. 4 q + 3
    if (wave || !have) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) acc += sums[w][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t n = n0 + 4 * q + e;
        if (n >= a.n) break;
        finish1(a, f, n, (float)acc[e], a.x_scale[f], a.scale ? a.w_scale[n] * a.scale[n] : a.w_scale[n], a.bias ? a.bias[n] : 0.0f);
    }
}

template <int BM, int BN, int WM, int WN, int STAGES, int GROUPS>
hipError_t launch_tiles(const RowsI8Args& a, hipStream_t s) {
    const int64_t blocks = (a.rows + BM - 1) / BM * ((a.n + BN - 1) / BN);
    hipLaunchKernelGGL((matmul_i8_kernel<BM, BN, WM, WN, STAGES, GROUPS>), dim3((unsigned)blocks), dim3(64 * WM * WN * GROUPS), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rows_i8(const void* x, int x_f32, int64_t rows, int32_t c, int8_t* q, float* scale, hipStream_t s) {
    const int32_t pitch = (c + 15) / 16 * 16;
    const bool wide = c % (x_f32 ? 4 : 8) == 0;
    // A wave a row, a block that holds the row, or one that reads it twice, in us: 8192 x 1024 6.5, 12.4, 10.4; 8192 x 4096 -, 18.6, 20.5;
    // 4096 x 8192 -, 22.6, 23.5; 1 x 8192 -, 3.5, 4.3.
#define TBN_ROWS(f32, threads, vecs)                                                                                           \
    hipLaunchKernelGGL((rows_i8_kernel<f32, threads, vecs>), dim3((unsigned)((rows + 256 / threads - 1) / (256 / threads))), dim3(256), \
                       0, s, x, rows, c, pitch, wide, q, scale)
#define TBN_ROWS_BY_SIZE(f32)            \
    if (c <= 64 * 8 * 2)                 \
        TBN_ROWS(f32, 64, 2);            \
    else if (c <= 256 * 8 * 2)           \
        TBN_ROWS(f32, 256, 2);           \
    else if (c <= 256 * 8 * 4)           \
        TBN_ROWS(f32, 256, 4);           \
    else                                 \
        TBN_ROWS(f32, 256, 0)
    if (x_f32) {
        TBN_ROWS_BY_SIZE(true);
    } else {
        TBN_ROWS_BY_SIZE(false);
    }
#undef TBN_ROWS_BY_SIZE
#undef TBN_ROWS
    return hipGetLastError();
}

hipError_t launch_matmul_i8(const RowsI8Args& a, hipStream_t s) {
    if (a.rows <= 16) {
        if (a.c <= 2048 * 2) return launch_stream<2>(a, s);
        if (a.c <= 2048 * 4) return launch_stream<4>(a, s);
        hipLaunchKernelGGL((matvec_i8_kernel<4, 4>), dim3((unsigned)((a.n + 15) / 16)), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    // The largest tile of which there are enough for the 256 compute units: 128 x 128 by four waves, two blocks a unit, from 257 on (or 256 x 256,
    // whichever takes less time in rounds), by eight, one a unit, from 160 on (up to three units in eight are idle); 128 x 64 from 256 on; else 64 x 64,
    // up to 256 of them in four groups of waves that divide the stages where these are many.  Times in us, c 4096:
    //   rows x n        256x256  128x128/4  128x128/8  128x64  64x64  64x64 x 4
    //   8192 x 8192      241       256        334        343    401     657
    //   4000 x 4097      118        90                                126        272 tiles of 256 x 256
    //   3200 x 4096       57.2      61.7       79.0       75.5   87.8   140.5    208
    //   2560 x 4096       56.1      56.6       59.5       57.1   69.7   108.8    160
    //   2048 x 4096       54.5      36.1       42.3       47.5   57.9    88.4    512 tiles of 128 x 128
    //   1024 x 4096       51.0      27.4       22.1       24.3   31.5    45.5    256
    //    768 x 4096       50.7      26.0       20.5       20.9   23.9    35.8    192
    //    640 x 4096       51.9      25.5       19.9       20.0   21.6    34.7    160
    //    512 x 4096       49.0      23.3       19.4       15.7   16.7    24.3    256 tiles of 128 x 64
    //    256 x 4352                                       14.9   15.3    20.5    272 tiles of 64 x 64
    //    256 x 4096                                       14.9   12.8    11.3    256; c 2048: 8.3, 8.1; c 1024: 6.0, 6.5
    auto tiles = [&](int64_t m, int64_t n) { return (a.rows + m - 1) / m * ((a.n + n - 1) / n); };
    // (256 x 256 go in rounds of 256, 56 us here, 128 x 128 in rounds of 512, 36.)
    if (tiles(128, 128) > 256) {
        const int64_t large = (tiles(256, 256) + 255) / 256 * 14, small = (tiles(128, 128) + 511) / 512 * 9;
        return large <= small ? launch_tiles<256, 256, 2, 2, 2, 1>(a, s) : launch_tiles<128, 128, 2, 2, 2, 1>(a, s);
    }
    if (tiles(128, 128) >= 160) return launch_tiles<128, 128, 2, 4, 4, 1>(a, s);
    if (tiles(128, 64) >= 256) return launch_tiles<128, 64, 2, 2, 3, 1>(a, s);
    if (tiles(64, 64) <= 256 && a.c >= 2048) return launch_tiles<64, 64, 2, 2, 2, 4>(a, s);
    return launch_tiles<64, 64, 2, 2, 2, 1>(a, s);
}

}  // namespace tbn
