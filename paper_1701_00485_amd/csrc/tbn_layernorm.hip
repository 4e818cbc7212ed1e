// tbn_layernorm.hip -- layer normalisation of rows of C features, forward and backward.
//
//   forward   mu = mean_c x, s = 1 / sqrt(mean_c (x - mu)^2 + eps), y = (x - mu) s gamma + beta
//   backward  xh = (x - mu) s, h = dy gamma,  dx = s (h - mean_c h - xh mean_c(h xh)),
//             dgamma = sum_rows dy xh,  dbeta = sum_rows dy
//
// Bound by HBM: each tensor is read or written once (rows beyond 16384 values are read twice backward).  Measured: forward 8192
// rows of 8192 bf16 values 51 us (5.2 TB/s), one row of 512 2.3 us of kernel; backward 16384 rows of 4096 82 us (4.9 TB/s), of
// which the last sums are 6; 777 rows of 1000 6 + 4 us: launch and one row's latency, then 195 rows of partial sums, 7 loads in turn.
// A team of T threads (8 to 64 lanes of a wave, or a whole block) keeps a row in registers, NV pieces of 8 neighbouring
// values per thread, so that the centred sum of squares is a second pass over registers.  Teams walk the rows with the
// stride of the grid and keep what belongs to their columns in registers over all of them: gamma and beta, and in the
// backward pass the sums of dgamma and dbeta, which are added over the teams of a block and written as one row of partial
// sums per block; a second kernel adds those in a fixed order (no atomics: the same bits every time).
// Rows longer than the registers hold are read again, forward in ln_fwd_long_kernel (2048 rows of 65536 bf16 values 190 us, 2.8 TB/s
// of x and y; of 20001 72 us, 2.3), backward in two kernels.
//
// All sums and statistics are fp32; a value is rounded once, where a bf16 output is stored.  Pieces are
// loaded as 16-byte words at the alignment of an element, so odd C needs no other path than its last piece.
#include "tbn_device.h"
#include "tbn_kernels.h"

namespace tbn {

namespace {

struct Piece {
    float v[8];
};

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

// 8 values as they lie in memory: what is in flight.
template <typename T>
struct Raw;
template <>
struct Raw<uint16_t> {
    u32x4 w = {0u, 0u, 0u, 0u};
    // from here on the compiler does not know what was formed from it before
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w)); }
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4_a2*>(p); }
    // the first `left` (1 to 7); the last one again where there are no more, so that the loads go out together
    __device__ __forceinline__ void load_some(const uint16_t* p, int left) {
        uint32_t h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = p[j < left ? j : left - 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (2 * j < left ? h[2 * j] : 0u) | (2 * j + 1 < left ? h[2 * j + 1] << 16 : 0u);
    }
    __device__ __forceinline__ Piece piece() const {
        Piece r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            r.v[2 * j] = __uint_as_float(w[j] << 16);
            r.v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
        return r;
    }
};
template <>
struct Raw<float> {
    f32x4 w[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w[0]), "+v"(w[1])); }
    __device__ __forceinline__ void load(const float* p) {
        w[0] = *reinterpret_cast<const f32x4_a4*>(p);
        w[1] = *reinterpret_cast<const f32x4_a4*>(p + 4);
    }
    __device__ __forceinline__ void load_some(const float* p, int left) {
        float h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = p[j < left ? j : left - 1];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j >> 2][j & 3] = j < left ? h[j] : 0.0f;
    }
    __device__ __forceinline__ Piece piece() const {
        Piece r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r.v[j] = w[j >> 2][j & 3];
        return r;
    }
};

// A thread's NV pieces of a row of C values (WHOLE: a multiple of 8), thread t of T; zeros beyond C.  The whole pieces first, without a branch that
// writes (it would wait for the loads of the others), then the last, shorter one.
template <bool WHOLE, int T, int NV, typename E>
__device__ __forceinline__ void load_row(Raw<E> (&r)[NV], const E* row, int t, int C) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = (i * T + t) * 8;
        r[i] = Raw<E>();
        if (e + 8 <= C) r[i].load(row + e);
    }
    if constexpr (!WHOLE) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * T + t) * 8;
            if (e < C && e + 8 > C) r[i].load_some(row + e, C - e);
        }
    }
}

// 8 values from p, or the first `left` (>= 1) of them, the rest 0.
template <typename E>
__device__ __forceinline__ Piece load_piece(const E* p, int left) {
    Raw<E> r;
    if (left >= 8) r.load(p);
    else r.load_some(p, left);
    return r.piece();
}

__device__ __forceinline__ void store_piece(uint16_t* p, const Piece& r, int left) {
    if (left >= 8) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(r.v[2 * j], r.v[2 * j + 1]);
        *reinterpret_cast<u32x4_a2*>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) p[j] = (uint16_t)f32_to_bf16_bits(r.v[j]);
    }
}

__device__ __forceinline__ void store_piece(float* p, const Piece& r, int left) {
    if (left >= 8) {
        *reinterpret_cast<f32x4_a4*>(p) = f32x4{r.v[0], r.v[1], r.v[2], r.v[3]};
        *reinterpret_cast<f32x4_a4*>(p + 4) = f32x4{r.v[4], r.v[5], r.v[6], r.v[7]};
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) p[j] = r.v[j];
    }
}

// The sum of v (and of w) over the T threads of a team, in every one of them.  T > 64: the team is the block,
// and `sh` holds two buffers of 2 T / 64 floats, used in turn (`turn`), so that one barrier a sum is enough.
template <int T>
__device__ __forceinline__ void team_sum2(float& v, float& w, float* sh, int& turn) {
#pragma unroll
    for (int off = (T < 64 ? T : 64) / 2; off >= 1; off >>= 1) {
        v += __shfl_xor(v, off, kWave);
        w += __shfl_xor(w, off, kWave);
    }
    if constexpr (T > 64) {
        constexpr int W = T / 64;
        float* b = sh + (turn & 1) * 2 * W;
        ++turn;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            b[wave] = v;
            b[W + wave] = w;
        }
        __syncthreads();
        v = 0.0f;
        w = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v += b[i];
            w += b[W + i];
        }
    }
}

template <int T>
__device__ __forceinline__ float team_sum(float v, float* sh, int& turn) {
    if constexpr (T <= 64) {
#pragma unroll
        for (int off = T / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
        return v;
    } else {
        float unused = 0.0f;
        team_sum2<T>(v, unused, sh, turn);
        return v;
    }
}

template <typename XT, typename YT, int T, int NV, int BLOCK, bool WHOLE>
__global__ __launch_bounds__(BLOCK) void ln_fwd_kernel(const XT* __restrict__ x, int64_t rows, int32_t C,
                                                       const float* __restrict__ gamma,
                                                       const float* __restrict__ beta, float eps,
                                                       YT* __restrict__ y, float* __restrict__ mean,
                                                       float* __restrict__ inv_std) {
    __shared__ float sh[T > 64 ? T / 16 : 1];
    constexpr int RPB = BLOCK / T;
    const int t = threadIdx.x % T;
    int turn = 0;
    constexpr bool HOLD = NV <= 4;  // gamma and beta in registers; otherwise from the L2 for every row
    Piece g[HOLD ? NV : 1], b[HOLD ? NV : 1];
    auto parameters = [&](int e, Piece& gp, Piece& bp) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            gp.v[j] = 1.0f;
            bp.v[j] = 0.0f;
        }
        if (e < C && gamma) gp = load_piece(gamma + e, WHOLE ? 8 : C - e);
        if (e < C && beta) bp = load_piece(beta + e, WHOLE ? 8 : C - e);
    };
    if constexpr (HOLD) {
#pragma unroll
        for (int i = 0; i < NV; ++i) parameters((i * T + t) * 8, g[i], b[i]);
    }
    const float inv_c = 1.0f / (float)C;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / T;
    Raw<XT> raw[NV];
    if (row < rows) load_row<WHOLE, T, NV>(raw, x + row * C, t, C);
    for (; row < rows; row += stride) {
        Piece v[NV];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            v[i] = raw[i].piece();
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[i].v[j];
        }
        if (row + stride < rows) load_row<WHOLE, T, NV>(raw, x + (row + stride) * C, t, C);  // the next row, in flight
        __builtin_amdgcn_sched_barrier(0);
        const float mu = team_sum<T>(sum, sh, turn) * inv_c;
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * T + t) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = v[i].v[j] - mu;
                v[i].v[j] = e + (WHOLE ? 0 : j) < C ? d : 0.0f;
                sq += v[i].v[j] * v[i].v[j];
            }
        }
        const float s = 1.0f / sqrtf(team_sum<T>(sq, sh, turn) * inv_c + eps);
        YT* yr = y + row * C;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * T + t) * 8;
            if (e >= C) break;
            constexpr int kHeld = HOLD ? 1 : 0;
            if constexpr (!HOLD) parameters(e, g[0], b[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i].v[j] = v[i].v[j] * s * g[kHeld * i].v[j] + b[kHeld * i].v[j];
            store_piece(yr + e, v[i], WHOLE ? 8 : C - e);
        }
        if (t == 0) {
            if (mean) mean[row] = mu;
            if (inv_std) inv_std[row] = s;
        }
    }
}

// Rows that no team holds in registers: a block per row, three passes over it.
template <typename XT, typename YT>
__global__ __launch_bounds__(1024) void ln_fwd_long_kernel(const XT* __restrict__ x, int64_t rows, int32_t C,
                                                           const float* __restrict__ gamma,
                                                           const float* __restrict__ beta, float eps,
                                                           YT* __restrict__ y, float* __restrict__ mean,
                                                           float* __restrict__ inv_std) {
    __shared__ float sh[64];
    int turn = 0;
    const float inv_c = 1.0f / (float)C;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const XT* xr = x + row * C;
        float sum = 0.0f;
        for (int e = threadIdx.x * 8; e < C; e += 8192) {
            const Piece v = load_piece(xr + e, C - e);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v.v[j];
        }
        const float mu = team_sum<1024>(sum, sh, turn) * inv_c;
        float sq = 0.0f;
        for (int e = threadIdx.x * 8; e < C; e += 8192) {
            const Piece v = load_piece(xr + e, C - e);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e + j < C) sq += (v.v[j] - mu) * (v.v[j] - mu);
        }
        const float s = 1.0f / sqrtf(team_sum<1024>(sq, sh, turn) * inv_c + eps);
        YT* yr = y + row * C;
        for (int e = threadIdx.x * 8; e < C; e += 8192) {
            Piece v = load_piece(xr + e, C - e), g, b;
            if (gamma) g = load_piece(gamma + e, C - e);
            if (beta) b = load_piece(beta + e, C - e);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v.v[j] = (v.v[j] - mu) * s * (gamma ? g.v[j] : 1.0f) + (beta ? b.v[j] : 0.0f);
            store_piece(yr + e, v, C - e);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (inv_std) inv_std[row] = s;
        }
    }
}

// partial: [2][gridDim.x][C] (dgamma, then dbeta).
template <typename XT, typename YT, int T, int NV, int BLOCK, bool WHOLE>
__global__ __launch_bounds__(BLOCK) void ln_bwd_kernel(const XT* __restrict__ x, const YT* __restrict__ dy,
                                                       int64_t rows, int32_t C, const float* __restrict__ mean,
                                                       const float* __restrict__ inv_std,
                                                       const float* __restrict__ gamma, XT* __restrict__ dx,
                                                       float* __restrict__ partial) {
    constexpr int RPB = BLOCK / T;
    __shared__ float sh[T > 64 ? T / 16 : 1];
    __shared__ float acc[RPB > 1 ? RPB * T * 8 : 1];
    const int t = threadIdx.x % T, team = threadIdx.x / T;
    int turn = 0;
    Piece g[NV], dg[NV], db[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = (i * T + t) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            g[i].v[j] = 1.0f;
            dg[i].v[j] = 0.0f;
            db[i].v[j] = 0.0f;
        }
        if (e < C && gamma) g[i] = load_piece(gamma + e, WHOLE ? 8 : C - e);
    }
    const float inv_c = 1.0f / (float)C;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + team;
    Raw<XT> xnext[NV];
    Raw<YT> dnext[NV];
    float mu_next = 0.0f, s_next = 0.0f;
    auto load = [&](int64_t r) {
        load_row<WHOLE, T, NV>(xnext, x + r * C, t, C);
        load_row<WHOLE, T, NV>(dnext, dy + r * C, t, C);
        mu_next = mean[r];
        s_next = inv_std[r];
    };
    constexpr bool AHEAD = T < 512;  // the widest team has no registers for the next row
    if (AHEAD && row < rows) load(row);
    for (; row < rows; row += stride) {
        if constexpr (!AHEAD) load(row);
        const float mu = mu_next, s = s_next;
        Raw<XT> xr[NV];  // a row stays as it lies in memory; the second pass over it forms xh and h again
        Raw<YT> dr[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            xr[i] = xnext[i];
            dr[i] = dnext[i];
        }
        if (AHEAD && row + stride < rows) load(row + stride);  // the next row, in flight
        __builtin_amdgcn_sched_barrier(0);
        // xh and h of a piece; beyond C the gradient is 0 and xh is made so, whatever mu and s are
        auto form = [&](int i, Piece& xh, Piece& d, Piece& h) {
            const int e = (i * T + t) * 8;
            xh = xr[i].piece();
            d = dr[i].piece();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x0 = (xh.v[j] - mu) * s;
                xh.v[j] = e + (WHOLE ? 0 : j) < C ? x0 : 0.0f;
                h.v[j] = d.v[j] * g[i].v[j];
            }
        };
        float sh1 = 0.0f, sh2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Piece xh, d, h;
            form(i, xh, d, h);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dg[i].v[j] += d.v[j] * xh.v[j];
                db[i].v[j] += d.v[j];
                sh1 += h.v[j];
                sh2 += h.v[j] * xh.v[j];
            }
        }
        team_sum2<T>(sh1, sh2, sh, turn);
        sh1 *= inv_c;
        sh2 *= inv_c;
        if constexpr (NV >= 4) {  // where registers are short
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                xr[i].forget();
                dr[i].forget();
            }
        }
        XT* dxr = dx + row * C;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = (i * T + t) * 8;
            if (e >= C) break;
            Piece xh, d, h;
            form(i, xh, d, h);
#pragma unroll
            for (int j = 0; j < 8; ++j) d.v[j] = s * (h.v[j] - sh1 - xh.v[j] * sh2);
            store_piece(dxr + e, d, WHOLE ? 8 : C - e);
        }
    }
    float* pg = partial + (int64_t)blockIdx.x * C;
    float* pb = partial + (int64_t)(gridDim.x + blockIdx.x) * C;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = (i * T + t) * 8;
        if constexpr (RPB == 1) {
            if (e < C) {
                store_piece(pg + e, dg[i], WHOLE ? 8 : C - e);
                store_piece(pb + e, db[i], WHOLE ? 8 : C - e);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {  // teams added in order
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[(team * 8 + j) * T + t] = q ? db[i].v[j] : dg[i].v[j];
                __syncthreads();
                for (int o = threadIdx.x; o < 8 * T; o += BLOCK) {
                    float sum = 0.0f;
#pragma unroll
                    for (int m = 0; m < RPB; ++m) sum += acc[m * 8 * T + o];
                    const int c = (i * T + o % T) * 8 + o / T;
                    if (c < C) (q ? pb : pg)[c] = sum;
                }
            }
        }
    }
}

// Rows that no team holds in registers, in two kernels.  The first, a block a row, leaves mean(h) and mean(h xhat) of
// each row; in the second a thread has 8 columns and walks down a share of the rows, kDown at a time, with the sums of
// dgamma and dbeta in registers.  x and dy are read twice, so 4096 rows of 16384, which a team does hold, stay with
// it; 2048 rows of 32768 bf16 values take 72 + 74 us and 13 for the last sums (those in registers 92 + 15).  One kernel, a
// block a row, would read and write its sums of dgamma and dbeta in memory for every row: 283 + 39 us.
constexpr int kDown = 4;

template <typename XT, typename YT>
__global__ __launch_bounds__(1024) void ln_bwd_means_kernel(const XT* __restrict__ x, const YT* __restrict__ dy, int64_t rows,
                                                            int32_t C, const float* __restrict__ mean,
                                                            const float* __restrict__ inv_std,
                                                            const float* __restrict__ gamma, float2* __restrict__ means) {
    __shared__ float sh[64];
    int turn = 0;
    const int pieces = C / 8;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const XT* xr = x + row * C;
        const YT* dr = dy + row * C;
        const float mu = mean[row], s = inv_std[row];
        float sh1 = 0.0f, sh2 = 0.0f;
        for (int first = threadIdx.x; first < pieces; first += 1024 * 2) {
            Raw<XT> xv[2];
            Raw<YT> dv[2];
            Raw<float> gv[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {  // the last piece again behind the end
                const int e = 8 * (first + 1024 * k < pieces ? first + 1024 * k : pieces - 1);
                xv[k].load(xr + e);
                dv[k].load(dr + e);
                if (gamma) gv[k].load(gamma + e);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Piece xp = xv[k].piece(), d = dv[k].piece(), g = gv[k].piece();
                const bool is = first + 1024 * k < pieces;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float h = gamma ? d.v[j] * g.v[j] : d.v[j], hx = h * ((xp.v[j] - mu) * s);
                    sh1 += is ? h : 0.0f;
                    sh2 += is ? hx : 0.0f;
                }
            }
        }
        if (threadIdx.x == 0 && C % 8) {
            const Piece xp = load_piece(xr + 8 * pieces, C % 8), d = load_piece(dr + 8 * pieces, C % 8);
            Piece g;
            if (gamma) g = load_piece(gamma + 8 * pieces, C % 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = gamma ? d.v[j] * g.v[j] : d.v[j], hx = h * ((xp.v[j] - mu) * s);
                sh1 += j < C % 8 ? h : 0.0f;
                sh2 += j < C % 8 ? hx : 0.0f;
            }
        }
        team_sum2<1024>(sh1, sh2, sh, turn);
        const float inv_c = 1.0f / (float)C;
        if (threadIdx.x == 0) means[row] = float2{sh1 * inv_c, sh2 * inv_c};
    }
}

// partial: [2][gridDim.y][C]; block (i, j): columns 2048 i + 0..2047 of rows j, j + gridDim.y, ...
template <typename XT, typename YT>
__global__ __launch_bounds__(256) void ln_bwd_down_kernel(const XT* __restrict__ x, const YT* __restrict__ dy, int64_t rows,
                                                          int32_t C, const float* __restrict__ mean,
                                                          const float* __restrict__ inv_std,
                                                          const float* __restrict__ gamma,
                                                          const float2* __restrict__ means, XT* __restrict__ dx,
                                                          float* __restrict__ partial) {
    const int e = 2048 * (int)blockIdx.x + 8 * (int)threadIdx.x;
    if (e >= C) return;
    const int left = C - e;
    Piece g, dg = {}, db = {};
    if (gamma) g = load_piece(gamma + e, left);
    auto one = [&](int64_t row, const Piece& xp, const Piece& d, int count) {
        const float mu = mean[row], s = inv_std[row];
        const float2 m = means[row];
        Piece out;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float xh = (xp.v[j] - mu) * s, h = gamma ? d.v[j] * g.v[j] : d.v[j];
            dg.v[j] += d.v[j] * xh;
            db.v[j] += d.v[j];
            out.v[j] = s * (h - m.x - xh * m.y);
        }
        store_piece(dx + row * C + e, out, count);
    };
    const int64_t stride = gridDim.y;
    int64_t row = blockIdx.y;
    if (2048 * ((int)blockIdx.x + 1) <= C)  // all of the block's columns: no load has a branch
        for (; row + (kDown - 1) * stride < rows; row += kDown * stride) {
            Raw<XT> xv[kDown];
            Raw<YT> dv[kDown];
#pragma unroll
            for (int k = 0; k < kDown; ++k) {
                xv[k].load(x + (row + k * stride) * C + e);
                dv[k].load(dy + (row + k * stride) * C + e);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < kDown; ++k) one(row + k * stride, xv[k].piece(), dv[k].piece(), 8);
        }
    for (; row < rows; row += stride) one(row, load_piece(x + row * C + e, left), load_piece(dy + row * C + e, left), left);
    store_piece(partial + (int64_t)blockIdx.y * C + e, dg, left);
    store_piece(partial + (int64_t)(gridDim.y + blockIdx.y) * C + e, db, left);
}

// dgamma, dbeta = the sums of the blocks' partial rows: 32 columns a block, whose 32 groups of threads take every
// 32nd row and are added in order.
__global__ __launch_bounds__(1024) void ln_reduce_kernel(const float* __restrict__ partial, int32_t blocks, int32_t C,
                                                         float* __restrict__ dgamma, float* __restrict__ dbeta) {
    __shared__ float sh[32][33];
    const int col = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + col;
    const float* p = partial + (int64_t)blockIdx.y * blocks * C;
    float s = 0.0f;
    if (c < C)
        for (int b = grp; b < blocks; b += 32) s += p[(int64_t)b * C + c];
    sh[grp][col] = s;
    __syncthreads();
    if (grp == 0 && c < C) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sh[i][col];
        (blockIdx.y ? dbeta : dgamma)[c] = t;
    }
}

// The team that holds rows of C values: the smallest of these whose 8 T NV values suffice (an index of the
// switches below; -1: the long kernels).
constexpr int kTeams[][3] = {{8, 1, 256},  {16, 1, 256}, {32, 1, 256}, {64, 1, 256},  {64, 2, 256},
                             {64, 4, 256}, {256, 2, 256}, {256, 4, 256}, {512, 4, 512}, {512, 8, 512}};
constexpr int kNumTeams = sizeof(kTeams) / sizeof(kTeams[0]);

int team_of(int32_t C) {
    for (int i = 0; i < kNumTeams; ++i)
        if (C <= 8 * kTeams[i][0] * kTeams[i][1]) return i;
    return -1;
}

// The widest team only where its registers suffice: forward, rows of whole pieces (2048 rows of 32768 65 us, the long
// kernel, which reads them again from the caches, for the others).  Backward the next one, of 512 threads and rows of 8193 to
// 16384 values, spills where they are no whole pieces, 344 to 472 bytes a lane (whole fp32 rows and gradients 68).  It and the two
// kernels for longer rows: 2048 rows of 16383 bf16 values 97 and 105 us, of 12001 83 and 88, 8192 of those 252 and 302; with few
// rows or fp32 on both sides the two kernels: 300 of 12001 37 and 23, 2048 of 8201 fp32 values 116 and 90.
int fwd_team(int32_t C) {
    const int team = team_of(C);
    return team == kNumTeams - 1 && C % 8 ? -1 : team;
}
int bwd_team(int32_t C) {
    const int team = team_of(C);
    return team == kNumTeams - 1 ? -1 : team;
}

template <typename XT, typename YT>
void fwd(const LnArgs& a, hipStream_t stream) {
    const int team = fwd_team(a.C);
    const XT* x = reinterpret_cast<const XT*>(a.x);
    YT* y = reinterpret_cast<YT*>(a.y);
    const int rpb = team < 0 ? 1 : kTeams[team][2] / kTeams[team][0];
    int64_t blocks = (a.rows + rpb - 1) / rpb;
    const int64_t most = team < 0 ? 512 : 256 * 2048 / kTeams[team][2];
    if (blocks > most) blocks = most;
#define TBN_LN_CALL(T, NV, B, WHOLE)                                                                                   \
    hipLaunchKernelGGL((ln_fwd_kernel<XT, YT, T, NV, B, WHOLE>), dim3((unsigned)blocks), dim3(B), 0, stream, x, a.rows, \
                       a.C, a.gamma, a.beta, a.eps, y, a.mean, a.inv_std)
#define TBN_LN_WHOLE(i, T, NV, B)       \
    case i:                             \
        TBN_LN_CALL(T, NV, B, true);    \
        break
#define TBN_LN(i, T, NV, B)                              \
    case i:                                              \
        if (a.C % 8 == 0) TBN_LN_CALL(T, NV, B, true);   \
        else TBN_LN_CALL(T, NV, B, false);               \
        break
    switch (team) {
        TBN_LN(0, 8, 1, 256);
        TBN_LN(1, 16, 1, 256);
        TBN_LN(2, 32, 1, 256);
        TBN_LN(3, 64, 1, 256);
        TBN_LN(4, 64, 2, 256);
        TBN_LN(5, 64, 4, 256);
        TBN_LN(6, 256, 2, 256);
        TBN_LN(7, 256, 4, 256);
        TBN_LN(8, 512, 4, 512);
        TBN_LN_WHOLE(9, 512, 8, 512);
        default:
            hipLaunchKernelGGL((ln_fwd_long_kernel<XT, YT>), dim3((unsigned)blocks), dim3(1024), 0, stream, x, a.rows, a.C,
                               a.gamma, a.beta, a.eps, y, a.mean, a.inv_std);
    }
#undef TBN_LN
#undef TBN_LN_WHOLE
#undef TBN_LN_CALL
}

template <typename XT, typename YT>
void bwd(const LnArgs& a, int64_t blocks, hipStream_t stream) {
    const XT* x = reinterpret_cast<const XT*>(a.x);
    const YT* dy = reinterpret_cast<const YT*>(a.dy);
    XT* dx = reinterpret_cast<XT*>(a.dx);
#define TBN_LN_CALL(T, NV, B, WHOLE)                                                                                   \
    hipLaunchKernelGGL((ln_bwd_kernel<XT, YT, T, NV, B, WHOLE>), dim3((unsigned)blocks), dim3(B), 0, stream, x, dy, a.rows, \
                       a.C, a.mean, a.inv_std, a.gamma, dx, a.partial)
#define TBN_LN(i, T, NV, B)                              \
    case i:                                              \
        if (a.C % 8 == 0) TBN_LN_CALL(T, NV, B, true);   \
        else TBN_LN_CALL(T, NV, B, false);               \
        break
    switch (bwd_team(a.C)) {
        TBN_LN(0, 8, 1, 256);
        TBN_LN(1, 16, 1, 256);
        TBN_LN(2, 32, 1, 256);
        TBN_LN(3, 64, 1, 256);
        TBN_LN(4, 64, 2, 256);
        TBN_LN(5, 64, 4, 256);
        TBN_LN(6, 256, 2, 256);
        TBN_LN(7, 256, 4, 256);
        TBN_LN(8, 512, 4, 512);
        default:
            float2* means = reinterpret_cast<float2*>(a.partial + 2 * blocks * a.C);
            hipLaunchKernelGGL((ln_bwd_means_kernel<XT, YT>), dim3((unsigned)(a.rows < 4096 ? a.rows : 4096)), dim3(1024), 0,
                               stream, x, dy, a.rows, a.C, a.mean, a.inv_std, a.gamma, means);
            hipLaunchKernelGGL((ln_bwd_down_kernel<XT, YT>), dim3((unsigned)((a.C + 2047) / 2048), (unsigned)blocks), dim3(256),
                               0, stream, x, dy, a.rows, a.C, a.mean, a.inv_std, a.gamma, means, dx, a.partial);
    }
#undef TBN_LN
#undef TBN_LN_CALL
}

}  // namespace

int64_t layernorm_bwd_blocks(int64_t rows, int32_t C) {
    const int team = bwd_team(C);
    if (team < 0) {  // shares of the rows: 2048 blocks, at least kDown rows each
        const int64_t most = (rows + kDown - 1) / kDown, fill = 2048 / ((C + 2047) / 2048);
        const int64_t shares = fill < most ? fill : most;
        return shares > 1 ? shares : 1;
    }
    const int rpb = kTeams[team][2] / kTeams[team][0];
    const int64_t blocks = (rows + rpb - 1) / rpb;
    const int64_t most = kTeams[team][2] > 256 ? 256 : 512;  // the widest have a CU for themselves
    return blocks < most ? blocks : most;
}

size_t layernorm_bwd_bytes(int64_t rows, int32_t C) {
    return (size_t)layernorm_bwd_blocks(rows, C) * (size_t)C * 8 + (bwd_team(C) < 0 ? (size_t)rows * sizeof(float2) : 0);
}

hipError_t launch_layernorm_fwd(const LnArgs& a, hipStream_t stream) {
    if (a.x_f32)
        a.y_f32 ? fwd<float, float>(a, stream) : fwd<float, uint16_t>(a, stream);
    else
        a.y_f32 ? fwd<uint16_t, float>(a, stream) : fwd<uint16_t, uint16_t>(a, stream);
    return hipGetLastError();
}

hipError_t launch_layernorm_bwd(const LnArgs& a, hipStream_t stream) {
    const int64_t blocks = layernorm_bwd_blocks(a.rows, a.C);
    if (a.x_f32)
        a.y_f32 ? bwd<float, float>(a, blocks, stream) : bwd<float, uint16_t>(a, blocks, stream);
    else
        a.y_f32 ? bwd<uint16_t, float>(a, blocks, stream) : bwd<uint16_t, uint16_t>(a, blocks, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(ln_reduce_kernel, dim3((unsigned)((a.C + 31) / 32), 2), dim3(1024), 0, stream, a.partial,
                       (int32_t)blocks, a.C, a.dgamma, a.dbeta);
    return hipGetLastError();
}

}  // namespace tbn
