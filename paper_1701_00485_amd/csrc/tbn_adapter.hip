// tbn_adapter.hip -- low-rank adapters beside a shared projection: row i of a batch has the adapter index[i], a
// pair A [R][C], B [K][R] of a bank of S, or none.
//
//   forward   t_i = A x_i,  y_i = residual_i + scale B t_i
//   backward  dt_i = scale B^T dy_i,  dx_i = residual_i + A^T dt_i,  dA = sum_i dt_i x_i^T,  dB = scale sum_i dy_i t_i^T
//
// Three kernels, each for both directions:
//   shrink  rows of C values -> R values: bound by reading the rows (long batches) or the adapters (one token each)
//   expand  rows of R values -> K values, added to the residual: bound by the residual and the output
//   outer   the gradients: for each adapter the products of its rows' R values with their C values, summed
// Measured: 48 tokens of 48 requests, 8192 -> 32768, rank 16, 8 + 16 us (70 MB of adapters, 3.2 TB/s in one pass of 22 us);
// 5000 rows of 11 prompts, 4096 -> 4096, rank 32, 21 + 5 + 25 us (floor 26; fp32 rows 34 + 5 + 24, fp32 factors 27 + 5 + 28, rank 64
// 35 + 5 + 30, rank 128 48 + 5 + 54); backward of 8192 rows, 4096 -> 8192, four fp32 adapters of rank 16, 43 + 5 (dt) + 44 + 6
// (gradients) + 43 us (dx), floor 71, 28 us more for reading dy twice.
// All run on v_mfma_f32_16x16x32_bf16.  What has 32 bits (t, dt, fp32 weights or rows) enters exactly, as the sum of three
// bf16 numbers (8 bits each), and a product of two such factors leaves out only the parts below 2^-23 of it: every result is
// one of fp32 sums, a bf16 one rounded once.  Two parts, 16 bits, would save a third of these MFMAs, which do not
// bound any of the kernels, and cost gradients that are off by 4e-6.
//
// Rows may lie in any order: a tile of rows is run once for each adapter that it holds, and each row takes the
// result of its own (nothing of another row or adapter enters it, NaN included); tiles of one request's rows run once.
// The gradients gather the rows of their adapter into a list first.  An index outside [0, S) is no adapter.
// Every sum is in a fixed order.
#include <type_traits>

#include "tbn_device.h"
#include "tbn_kernels.h"

namespace tbn {

namespace {

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// 8 factors of an MFMA operand: bf16 as they are, fp32 as hi + mid + lo.
template <typename T>
struct Frag {
    bf16x8 hi;
};
template <>
struct Frag<float> {
    bf16x8 hi, mid, lo;
};

__device__ __forceinline__ Frag<float> split8(const float (&v)[8]) {
    Frag<float> f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f.hi[j] = (__bf16)v[j];
        const float r = v[j] - (float)f.hi[j];
        f.mid[j] = (__bf16)r;
        f.lo[j] = (__bf16)(r - (float)f.mid[j]);
    }
    return f;
}

// 8 values as they lie in memory: what is in flight while the ones before are multiplied.
template <typename T>
struct Raw {
    u32x4 v;
};
template <>
struct Raw<float> {
    float v[8];
};
__device__ __forceinline__ Frag<uint16_t> frag(const Raw<uint16_t>& r) { return Frag<uint16_t>{as_bf16x8(r.v)}; }
__device__ __forceinline__ Frag<float> frag(const Raw<float>& r) { return split8(r.v); }

// 8 neighbouring values of a row that has `left` more from p on (or none: left <= 0), zeros behind its end; there the
// row's last value is read instead, so that all loads are issued at once.
__device__ __forceinline__ Raw<uint16_t> load_raw(const uint16_t* p, int64_t left) {
    Raw<uint16_t> r;
    if (left >= 8) {
        r.v = *reinterpret_cast<const u32x4_a2*>(p);
    } else {
        uint32_t h[8] = {};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (left > 0) h[j] = p[j < left ? j : left - 1];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r.v[j] = (2 * j < left ? h[2 * j] : 0u) | (2 * j + 1 < left ? h[2 * j + 1] << 16 : 0u);
    }
    return r;
}
__device__ __forceinline__ Raw<float> load_raw(const float* p, int64_t left) {
    Raw<float> r;
    if (left >= 8) {
        const f32x4 a = *reinterpret_cast<const f32x4_a4*>(p), b = *reinterpret_cast<const f32x4_a4*>(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            r.v[j] = a[j];
            r.v[4 + j] = b[j];
        }
    } else {
        float h[8] = {};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (left > 0) h[j] = p[j < left ? j : left - 1];
#pragma unroll
        for (int j = 0; j < 8; ++j) r.v[j] = j < left ? h[j] : 0.0f;
    }
    return r;
}
// 8 values `stride` apart, of `left` >= 1 more, zeros behind them (and all of them zeros without `any`, loaded all the same).
__device__ __forceinline__ Raw<uint16_t> gather_raw(const uint16_t* p, int64_t stride, int64_t left, bool any = true) {
    Raw<uint16_t> r;
    uint32_t h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = p[(j < left ? j : left - 1) * stride];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        r.v[j] = (any && 2 * j < left ? h[2 * j] : 0u) | (any && 2 * j + 1 < left ? h[2 * j + 1] << 16 : 0u);
    return r;
}
__device__ __forceinline__ Raw<float> gather_raw(const float* p, int64_t stride, int64_t left, bool any = true) {
    Raw<float> r;
    float h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = p[(j < left ? j : left - 1) * stride];
#pragma unroll
    for (int j = 0; j < 8; ++j) r.v[j] = any && j < left ? h[j] : 0.0f;
    return r;
}

__device__ __forceinline__ f32x4 product(const Frag<uint16_t>& a, const Frag<uint16_t>& b, f32x4 c) {
    return mfma16(a.hi, b.hi, c);
}
__device__ __forceinline__ f32x4 product(const Frag<float>& a, const Frag<uint16_t>& b, f32x4 c) {
    return mfma16(a.hi, b.hi, mfma16(a.mid, b.hi, mfma16(a.lo, b.hi, c)));
}
__device__ __forceinline__ f32x4 product(const Frag<uint16_t>& a, const Frag<float>& b, f32x4 c) {
    return mfma16(a.hi, b.hi, mfma16(a.hi, b.mid, mfma16(a.hi, b.lo, c)));
}
__device__ __forceinline__ f32x4 product(const Frag<float>& a, const Frag<float>& b, f32x4 c) {
    c = mfma16(a.mid, b.mid, mfma16(a.lo, b.hi, mfma16(a.hi, b.lo, c)));
    return mfma16(a.hi, b.hi, mfma16(a.mid, b.hi, mfma16(a.hi, b.mid, c)));
}

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

// 8 rows of 16 columns of an LDS tile, a column a lane.  Of 16 lanes each names the 8 bytes of 4 neighbouring columns of one of
// 4 rows (lane i those of columns 4 (i % 4) .. + 3 of row i / 4) and gets the 4 rows of column i; the 4 rows behind likewise.
__device__ __forceinline__ bf16x8 read_columns(const uint16_t* p, int pitch) {
    const v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)p);
    const v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(p + 4 * pitch));
    typedef short v8i16 __attribute__((ext_vector_type(8)));
    const v8i16 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, v);
}

// Nothing moves across: left alone, the compiler turns a loop that multiplies what the round before has loaded back
// into one that loads and waits.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// Row r of the kernels' order in the batch.
template <bool SORTED>
__device__ __forceinline__ int64_t batch_row(const AdapterArgs& a, int64_t r) {
    return SORTED ? (int64_t)a.sorted[r] : r;
}

// The adapter of a row, -1 for none.
__device__ __forceinline__ int adapter_of(const int32_t* index, int64_t row, int32_t S) {
    const int32_t a = index[row];
    return (uint32_t)a < (uint32_t)S ? a : -1;
}

// ---- the rows of each adapter ------------------------------------------------------------
// order[]: the rows that have an adapter, by adapter and ascending, with a block S the rest behind them; span[s] = where adapter
// s begins and how many rows it has.  One block an adapter: the rows of lower adapters counted, its own listed behind them, 16 rows a thread
// at a time, each wave behind the rows of the waves before it.
template <int WV, bool REST>
__device__ void order_rows(const int32_t* __restrict__ index, int64_t rows, int32_t S, int32_t aid,
                           int32_t* __restrict__ order, int2* __restrict__ span, int* sh) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int lower = 0;
#pragma unroll 8
    for (int64_t r = threadIdx.x; r < rows; r += 64 * WV) lower += (uint32_t)index[r] < (uint32_t)aid;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) lower += __shfl_xor(lower, off, kWave);
    if (lane == 0) sh[wave] = lower;
    __syncthreads();
    int begin = 0, total = 0;
#pragma unroll
    for (int k = 0; k < WV; ++k) begin += sh[k];
    for (int64_t base = 0; base < rows; base += 1024 * WV) {
        const int64_t first = base + wave * 1024 + lane;
        uint32_t found = 0;
        int count = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int64_t row = first + 64 * k;
            const int32_t of = index[row < rows ? row : 0];
            const bool is = row < rows && (!REST || aid < S ? of == aid : (uint32_t)of >= (uint32_t)S);
            found |= (uint32_t)is << k;
            count += __popcll(__ballot(is));
        }
        __syncthreads();  // the counts of the round before have been read
        if (lane == 0) sh[wave] = count;
        __syncthreads();
        int at = begin + total;
#pragma unroll
        for (int k = 0; k < WV; ++k) {
            at += k < wave ? sh[k] : 0;
            total += sh[k];
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const bool is = found >> k & 1;
            const uint64_t m = __ballot(is);
            if (is) order[at + __popcll(m & ((1ull << lane) - 1))] = (int32_t)(first + 64 * k);
            at += __popcll(m);
        }
    }
    if (threadIdx.x == 0 && (!REST || aid < S)) span[aid] = int2{begin, total};
}

__global__ __launch_bounds__(1024) void order_kernel(const AdapterArgs a) {
    __shared__ int sh[16];
    order_rows<16, true>(a.index, a.rows, a.S, (int32_t)blockIdx.x, a.order, a.span, sh);
}

// ---- shrink ------------------------------------------------------------------------------
// out[split][row][r] = scale sum over the split's c of x[row][c] W[r][c], W = the row's adapter: [R][C], or with ACROSS
// [C][R].  A block has a tile of 16 RT rows and one split; its WV waves take 64 values of c each (whole 128-byte lines of
// bf16 rows), then the same again behind those of all splits, the next ones in flight, and add through LDS.  Blocks next to
// each other are the splits of one tile: what runs at the same time reads long runs of a row (with the tiles next to
// each other, all at the same columns of rows that are a power of two apart, a 134 MB batch took 50 us instead of 37).
// 8192 rows of 8192 bf16 values: 42 us, 3.2 TB/s (a tile's every further adapter adds about 5); with 4 splits
// 49, with 2 56.  What bounds it is the chain index, adapter, product at the few rounds a block has.  fp32 rows 74 us, rank 64 81,
// rank 128, in two slices that both read the rows, 128.
// With gridDim.y > 1 the tile's adapters are dealt over y.  In the backward pass S more blocks order the rows for the
// gradients beside it.
constexpr int kShrinkWaves = 4;

template <bool ACROSS, typename WT>
__device__ __forceinline__ Raw<WT> across_or_along(const WT* w, int c, int R, int left) {
    if constexpr (ACROSS) {
        const int back = left > 0 ? 0 : 1 - left;  // beyond the end: from the last value on
        return gather_raw(w + (int64_t)(c - back) * R, R, left + back, left > 0);
    } else {
        return load_raw(w + c, left);
    }
}

template <typename XT, typename WT, bool ACROSS, bool SORTED, int RN, int RT, int WV>
__global__ __launch_bounds__(64 * WV) void shrink_kernel(const AdapterArgs a) {
    __shared__ f32x4 red[WV][RN * RT * 64];
    if (blockIdx.x >= a.row_blocks) {
        if (blockIdx.y == 0)
            order_rows<WV, false>(a.index, a.rows, a.S, (int32_t)(blockIdx.x - a.row_blocks), a.order, a.span,
                           reinterpret_cast<int*>(red));
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const XT* x = reinterpret_cast<const XT*>(a.x);
    const WT* w = reinterpret_cast<const WT*>(a.w);
    const uint32_t slices = (uint32_t)(a.R + 63) / 64, all = (uint32_t)a.splits * slices;
    const uint32_t tile = blockIdx.x / all, split = (blockIdx.x - tile * all) / slices;
    const int r0 = 64 * (int)(blockIdx.x % slices);  // of ranks above 64 a block has 64
    const int64_t row0 = (int64_t)tile * (16 * RT);
    const int rows = a.rows - row0 < 16 * RT ? (int)(a.rows - row0) : 16 * RT;
    const int32_t C = a.C, R = a.R;
    const int step = 64 * WV * a.splits;
    const int c0 = 64 * (WV * (int)split + wave);
    float* out = a.part + ((int64_t)split * a.rows + (SORTED ? 0 : row0)) * R;

    const XT* xr[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = 16 * t + i < rows ? 16 * t + i : rows - 1;
        xr[t] = x + batch_row<SORTED>(a, row0 + r) * C + 8 * g;
    }
    Raw<XT> xv[2][RT];
    Raw<WT> wv[2][RN];
    auto load_x = [&](int h, int c, int left) {
#pragma unroll
        for (int t = 0; t < RT; ++t) xv[h][t] = load_raw(xr[t] + c, left);
    };
    const bool ahead = c0 + 64 <= C;  // the first rows' values need no adapter
    if (ahead) {
        load_x(0, c0, 8);
        load_x(1, c0 + 32, 8);
    }
    const int mine = lane < rows ? adapter_of(a.index, batch_row<SORTED>(a, row0 + lane), a.S) : -1;
    uint64_t todo = __ballot(mine >= 0);
    bool first = true;
    for (uint32_t slot = 0; todo; ++slot) {
        const int aid = __builtin_amdgcn_readfirstlane(__shfl(mine, __ffsll((unsigned long long)todo) - 1, kWave));
        const uint64_t same = __ballot(mine == aid);
        todo &= ~same;
        if (slot % gridDim.y != blockIdx.y) continue;
        const WT* wr[RN];
#pragma unroll
        for (int n = 0; n < RN; ++n) {
            const int r = r0 + 16 * n + i < R ? r0 + 16 * n + i : R - 1;
            wr[n] = w + (int64_t)aid * R * C + (ACROSS ? (int64_t)8 * g * R + r : (int64_t)r * C + 8 * g);
        }
        f32x4 acc[RN][RT];
#pragma unroll
        for (int n = 0; n < RN; ++n)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[n][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        auto load_w = [&](int h, int c, int left) {
#pragma unroll
            for (int n = 0; n < RN; ++n) wv[h][n] = across_or_along<ACROSS>(wr[n], c, R, left);
        };
        auto multiply = [&](int h) {
            Frag<WT> wf[RN];
#pragma unroll
            for (int n = 0; n < RN; ++n) wf[n] = frag(wv[h][n]);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const Frag<XT> xf = frag(xv[h][t]);
#pragma unroll
                for (int n = 0; n < RN; ++n) acc[n][t] = product(wf[n], xf, acc[n][t]);
            }
        };
        int c = c0;
        if (ahead) {
            load_w(0, c, 8);
            load_w(1, c + 32, 8);
            if (!first) {
                load_x(0, c, 8);
                load_x(1, c + 32, 8);
            }
            for (; c + step + 64 <= C; c += step) {
                multiply(0);
                load_w(0, c + step, 8);
                load_x(0, c + step, 8);
                in_order();
                multiply(1);
                load_w(1, c + step + 32, 8);
                load_x(1, c + step + 32, 8);
                in_order();
            }
            multiply(0);
            multiply(1);
            c += step;
        }
        if (c < C) {  // the last, shorter 64 values
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                load_w(h, c + 32 * h, C - c - 32 * h - 8 * g);
                load_x(h, c + 32 * h, C - c - 32 * h - 8 * g);
            }
            multiply(0);
            multiply(1);
        }
        first = false;
#pragma unroll
        for (int n = 0; n < RN; ++n)
#pragma unroll
            for (int t = 0; t < RT; ++t) red[wave][(n * RT + t) * 64 + lane] = acc[n][t];
        __syncthreads();
        const float sc = a.scale ? a.scale[aid] : 1.0f;
        for (int o = threadIdx.x; o < RN * RT * 64; o += 64 * WV) {
            f32x4 s = red[0][o];
#pragma unroll
            for (int k = 1; k < WV; ++k) s += red[k][o];
            const int l = o & 63, n = (o >> 6) / RT, row = 16 * ((o >> 6) % RT) + (l & 15);
            if (!(same >> row & 1)) continue;
            float* to = out + (SORTED ? (int64_t)a.sorted[row0 + row] : row) * R;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = r0 + 16 * n + 4 * (l >> 4) + j;
                if (r < R) to[r] = sc * s[j];
            }
        }
        __syncthreads();
    }
    if (blockIdx.y == 0 && wave == 0) {  // rows without an adapter
        uint64_t none = __ballot(lane < rows && mine < 0);
        while (none) {
            const int row = __ffsll((unsigned long long)none) - 1;
            none &= none - 1;
            const int64_t at = SORTED ? (int64_t)a.sorted[row0 + row] : row;
            if (r0 + lane < R) out[at * R + r0 + lane] = 0.0f;
        }
    }
}

// t[i] = the sum over the splits, in order.
__global__ __launch_bounds__(256) void finish_kernel(const float* __restrict__ part, int64_t count, int32_t splits,
                                                     float* __restrict__ t) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        float s = part[i];
        for (int k = 1; k < splits; ++k) s += part[k * count + i];
        t[i] = s;
    }
}

// ---- expand ------------------------------------------------------------------------------
// y[row][k] = residual[row][k] + scale sum_r t[row][r] W[k][r], W = the row's adapter: [K][R], or with ACROSS [R][K];
// for few rows t is the sum of `splits` partial ones.  Rows of the MFMA's result are dealt to columns so that the four
// lanes of a row read and store 64 neighbouring bytes at a time.
// The 16 outputs of lane group g: for bf16 columns 32 p + 8 g + 0..7 (p = 0, 1), for fp32 16 q + 4 g + 0..3 (q = 0..3);
// result q of the MFMAs, row 4 g + j, is the lane's output 4 q + j.
template <typename T>
struct Outputs;
template <>
struct Outputs<uint16_t> {
    u32x4 v[2];
    static __device__ __forceinline__ int column(int q, int m) { return 32 * (q >> 1) + 8 * (m >> 2) + 4 * (q & 1) + (m & 3); }
    // p: the row's column col0 + 8 g, of which `left` = K - col0 - 8 g are inside the row; full: all 64 columns are
    __device__ __forceinline__ void load(const uint16_t* p, bool full, int left) {
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = full ? *reinterpret_cast<const u32x4_a2*>(p + 32 * h) : load_raw(p + 32 * h, left - 32 * h).v;
    }
    __device__ __forceinline__ float get(int o) const {
        const uint32_t w = v[o >> 3][(o & 7) >> 1];
        return __uint_as_float(o & 1 ? w & 0xFFFF0000u : w << 16);
    }
    static __device__ __forceinline__ void store(uint16_t* p, bool full, int left, const f32x4 (&y)[4]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(y[2 * h + (j >> 1)][2 * (j & 1)], y[2 * h + (j >> 1)][2 * (j & 1) + 1]);
            if (full) {
                *reinterpret_cast<u32x4_a2*>(p + 32 * h) = w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (32 * h + j < left) p[32 * h + j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
            }
        }
    }
    static constexpr int kLane = 8;  // a lane group's first column is kLane g
};
template <>
struct Outputs<float> {
    f32x4 v[4];
    static __device__ __forceinline__ int column(int q, int m) { return 16 * q + m; }
    __device__ __forceinline__ void load(const float* p, bool full, int left) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (full) {
                v[q] = *reinterpret_cast<const f32x4_a4*>(p + 16 * q);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[q][j] = p[16 * q + j < left ? 16 * q + j : left - 1];
            }
        }
    }
    __device__ __forceinline__ float get(int o) const { return v[o >> 2][o & 3]; }
    static __device__ __forceinline__ void store(float* p, bool full, int left, const f32x4 (&y)[4]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (full) {
                *reinterpret_cast<f32x4_a4*>(p + 16 * q) = y[q];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (16 * q + j < left) p[16 * q + j] = y[q][j];
            }
        }
    }
    static constexpr int kLane = 4;
};

// Values r..r + 7 of a row of R, zeros behind its end.  Every lane loads (from the row's end where it has nothing to): a
// branch that writes the zeros would wait for the loads of the others.  WHOLE: R is a multiple of 8.
template <bool WHOLE, typename T>
__device__ __forceinline__ Raw<T> rank_raw(const T* row, int r, int R) {
    if constexpr (WHOLE) {
        Raw<T> v = load_raw(row + (r < R ? r : R - 8), 8);
        const uint32_t keep = r < R ? 0xFFFFFFFFu : 0u;
        u32x4* w = reinterpret_cast<u32x4*>(&v);
#pragma unroll
        for (int j = 0; j < (int)sizeof v / 16; ++j) w[j] &= keep;
        return v;
    } else {
        return gather_raw(row + (r < R ? r : R - 1), 1, r < R ? R - r : 1, r < R);
    }
}
// Factors r..r + 7 of a column (of the last one beyond K: not stored).
template <bool ACROSS, bool WHOLE, typename WT>
__device__ __forceinline__ Raw<WT> factors(const WT* w, int aid, int col, int r, int K, int R) {
    col = col < K ? col : K - 1;
    if constexpr (ACROSS)
        return gather_raw(w + ((int64_t)aid * R + (r < R ? r : R - 1)) * K + col, K, r < R ? R - r : 1, r < R);
    else return rank_raw<WHOLE>(w + ((int64_t)aid * K + col) * R, r, R);
}
// Values r..r + 7 of a row's t: the partial sums in order, four loads in flight.
template <bool WHOLE>
__device__ __forceinline__ Raw<float> sum_t(const float* row, int64_t stride, int splits, int r, int R) {
    Raw<float> t = rank_raw<WHOLE>(row, r, R);
    int s = 1;
    for (; s + 4 <= splits; s += 4) {
        Raw<float> u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = rank_raw<WHOLE>(row + (s + k) * stride, r, R);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) t.v[j] += u[k].v[j];
    }
    for (; s < splits; ++s) {
        const Raw<float> u = rank_raw<WHOLE>(row + s * stride, r, R);
#pragma unroll
        for (int j = 0; j < 8; ++j) t.v[j] += u.v[j];
    }
    return t;
}
__device__ __forceinline__ void store_t(float* row, const Raw<float>& t, int r, int R) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (r + j < R) row[r + j] = t.v[j];
}
__device__ __forceinline__ Frag<float> scaled(const Raw<float>& t, float scale) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = t.v[j] * scale;
    return split8(v);
}

// WHOLE: every wave's columns are inside and R is a multiple of 8, so that no load has a branch (whose other side would wait
// for the loads of this one).

// Long batches: a block has 64 NC columns of 128 rows, 16 a wave.  Residual (128 NC bytes a row) and t are in flight while
// the block puts an adapter's factors into LDS, as bf16 parts (so that fp32 ones are split once for 128 rows; [R][K] ones are
// turned by the transposing LDS read); then every wave that has rows of this adapter multiplies and stores them.
// Usually all of a block's rows have one adapter.  The chain index, factors, LDS, product, store is long, so what counts is
// how much each wave has in flight, and two blocks a CU.  8192 rows of 4096 bf16 values: 34 us with bf16 adapters of rank
// 16 (4.0 TB/s), 43 with fp32 ones (50 with 128 columns a block instead of 256, 46 with one block a CU).  Two blocks a CU are
// 128 registers a lane: the forms that turn [R][K] factors spill there, 256 columns a block 20 bytes a lane with bf16 factors and 52
// with fp32 ones, ranks above 64 52 and 68.
constexpr int kExpandWaves = 8;

// The parts of fp32 factors lie `part` values apart.
__device__ __forceinline__ void put_factors(uint16_t* to, int, const Frag<uint16_t>& f) { *reinterpret_cast<bf16x8*>(to) = f.hi; }
__device__ __forceinline__ void put_factors(uint16_t* to, int part, const Frag<float>& f) {
    *reinterpret_cast<bf16x8*>(to) = f.hi;
    *reinterpret_cast<bf16x8*>(to + part) = f.mid;
    *reinterpret_cast<bf16x8*>(to + 2 * part) = f.lo;
}
__device__ __forceinline__ void get_factors(const uint16_t* from, int, Frag<uint16_t>& f) {
    f.hi = *reinterpret_cast<const bf16x8*>(from);
}
__device__ __forceinline__ void get_factors(const uint16_t* from, int part, Frag<float>& f) {
    f.hi = *reinterpret_cast<const bf16x8*>(from);
    f.mid = *reinterpret_cast<const bf16x8*>(from + part);
    f.lo = *reinterpret_cast<const bf16x8*>(from + 2 * part);
}

__device__ __forceinline__ void get_across(const uint16_t* from, int pitch, int, Frag<uint16_t>& f) {
    f.hi = read_columns(from, pitch);
}
__device__ __forceinline__ void get_across(const uint16_t* from, int pitch, int part, Frag<float>& f) {
    f.hi = read_columns(from, pitch);
    f.mid = read_columns(from + part, pitch);
    f.lo = read_columns(from + 2 * part, pitch);
}

template <typename WT, typename OT, bool ACROSS, int RK, int NC>
__global__ __launch_bounds__(64 * kExpandWaves, 4) void expand_kernel(const AdapterArgs a) {
    // in LDS as they lie in memory: [columns][R], or with ACROSS [R][columns]
    constexpr int COLS = 64 * NC, PITCH = (ACROSS ? COLS : 32 * RK) + 8, PART = (ACROSS ? 32 * RK : COLS) * PITCH;
    __shared__ __attribute__((aligned(16))) uint16_t wt[(sizeof(WT) == 4 ? 3 : 1) * PART];
    __shared__ int next[kExpandWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int32_t K = a.C, R = a.R;
    const uint32_t blocks = (uint32_t)(K + COLS - 1) / COLS, row_block = blockIdx.x / blocks;
    const int col0 = (int)(blockIdx.x - row_block * blocks) * COLS;
    const int lc = Outputs<OT>::kLane * g;
    const bool whole = col0 + COLS <= K, whole_r = R % 8 == 0;
    const WT* w = reinterpret_cast<const WT*>(a.w);
    int64_t row = (int64_t)row_block * (16 * kExpandWaves) + 16 * wave + i;
    const bool in = row < a.rows;
    if (!in) row = a.rows - 1;  // loaded for nothing, not stored
    if (a.sorted) row = a.sorted[row];

    const int mine = in ? adapter_of(a.index, row, a.S) : -1;
    Outputs<OT> res[NC] = {};
    if (a.residual) {
        const OT* p = reinterpret_cast<const OT*>(a.residual) + row * K + col0 + lc;
        if (whole) {
#pragma unroll
            for (int c = 0; c < NC; ++c) res[c].load(p + 64 * c, true, 64);
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (col0 + 64 * c + lc < K) res[c].load(p + 64 * c, false, K - col0 - 64 * c - lc);
        }
    }
    Raw<float> t[RK];
#pragma unroll
    for (int k = 0; k < RK; ++k) {
        if (whole_r) t[k] = rank_raw<true>(a.part + row * R, 32 * k + 8 * g, R);
        else t[k] = rank_raw<false>(a.part + row * R, 32 * k + 8 * g, R);
    }
    OT* y = reinterpret_cast<OT*>(a.y) + row * K + col0 + lc;
    auto store = [&](int c, const f32x4 (&out)[4]) {
        if (whole) Outputs<OT>::store(y + 64 * c, true, 64, out);
        else Outputs<OT>::store(y + 64 * c, false, K - col0 - 64 * c - lc, out);
    };

    uint32_t todo = (uint32_t)__ballot(mine >= 0) & 0xFFFFu;
    while (true) {
        // the next adapter that a wave has rows of left
        if (lane == 0) next[wave] = todo ? __builtin_amdgcn_readlane(mine, __ffs(todo) - 1) : -1;
        __syncthreads();
        int aid = -1;
#pragma unroll
        for (int k = kExpandWaves - 1; k >= 0; --k) aid = next[k] >= 0 ? next[k] : aid;
        aid = __builtin_amdgcn_readfirstlane(aid);
        if (aid < 0) break;
        for (int p = threadIdx.x; p < COLS * 4 * RK; p += 64 * kExpandWaves) {
            if constexpr (ACROSS) {
                const int r = p / (8 * NC), c = 8 * (p % (8 * NC));
                Raw<WT> v = {};
                if (r < R) {
                    const WT* from = w + ((int64_t)aid * R + r) * K + col0 + c;
                    v = whole ? load_raw(from, 8) : load_raw(from, K - col0 - c);
                }
                put_factors(wt + r * PITCH + c, PART, frag(v));
            } else {
                const int c = p / (4 * RK), r = 8 * (p % (4 * RK));
                const WT* from = w + ((int64_t)aid * K + (col0 + c < K ? col0 + c : K - 1)) * R;
                put_factors(wt + c * PITCH + r, PART, frag(whole_r ? rank_raw<true>(from, r, R) : rank_raw<false>(from, r, R)));
            }
        }
        __syncthreads();
        const uint32_t same = (uint32_t)__ballot(mine == aid) & 0xFFFFu;
        if (same) {
            todo &= ~same;
            const float scale = a.scale ? a.scale[aid] : 1.0f;
            Frag<float> tf[RK];
#pragma unroll
            for (int k = 0; k < RK; ++k) tf[k] = scaled(t[k], scale);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                f32x4 out[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) out[q][j] = res[c].get(4 * q + j);
#pragma unroll
                    for (int k = 0; k < RK; ++k) {
                        Frag<WT> wf;
                        if constexpr (ACROSS)
                            get_across(wt + (32 * k + 8 * g + (i >> 2)) * PITCH + 64 * c + Outputs<OT>::column(q, 4 * (i & 3)),
                                       PITCH, PART, wf);
                        else get_factors(wt + (64 * c + Outputs<OT>::column(q, i)) * PITCH + 32 * k + 8 * g, PART, wf);
                        out[q] = product(wf, tf[k], out[q]);
                    }
                }
                if (mine == aid) store(c, out);
            }
        }
        __syncthreads();  // before the next adapter's factors
    }
    if (in && mine < 0) {  // rows without an adapter
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            f32x4 out[4];
#pragma unroll
            for (int j = 0; j < 16; ++j) out[j >> 2][j & 3] = res[c].get(j);
            store(c, out);
        }
    }
}

// Few rows, each likely with an adapter of its own: the adapters of a tile of 16 rows are dealt over z (never more of
// them than gridDim.z), so that a block streams the factors of one adapter, kGroups groups of 64 columns a wave, the
// next ones in flight (48 adapters 8192 -> 32768 of rank 16 16 us, 3.1 TB/s, of rank 64 46, 4.4), and touches that adapter's
// rows alone (z = 0 also those without one).
constexpr int kGroups = 4;

template <typename WT, typename OT, bool ACROSS, bool WHOLE, int RK>
__global__ __launch_bounds__(256) void expand_few_kernel(const AdapterArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int32_t K = a.C, R = a.R;
    const int col_lo = (blockIdx.x * 4 + wave) * (64 * kGroups);
    if (col_lo >= K) return;
    const int lc = Outputs<OT>::kLane * g;
    const WT* w = reinterpret_cast<const WT*>(a.w);
    const int64_t row = (int64_t)blockIdx.y * 16 + i;
    const bool in = row < a.rows;
    const int mine = in ? adapter_of(a.index, row, a.S) : -1;
    uint32_t todo = (uint32_t)__ballot(mine >= 0) & 0xFFFFu;
    int aid = -1;
    for (uint32_t slot = 0; todo; ++slot) {
        aid = __builtin_amdgcn_readfirstlane(__shfl(mine, __ffs(todo) - 1, kWave));
        if (slot == blockIdx.z) break;
        todo &= ~(uint32_t)__ballot(mine == aid);
        aid = -1;
    }
    const bool touch = in && ((aid >= 0 && mine == aid) || (mine < 0 && blockIdx.z == 0));
    if (!__ballot(touch)) return;
    if (aid < 0) aid = 0;  // only rows without an adapter: they take no product
    const OT* res = a.residual && touch ? reinterpret_cast<const OT*>(a.residual) + row * K + lc : nullptr;
    OT* y = reinterpret_cast<OT*>(a.y) + row * K + lc;

    // step 4 n + q: quarter q of group n, whose factors were loaded AHEAD steps before, its residual with its first quarter's.
    // For ranks above 32 one step ahead: a step has as many loads there as four have below.
    constexpr int STEPS = 4 * kGroups, AHEAD = RK == 1 ? 4 : 1;
    Raw<WT> wv[AHEAD + 1][RK];
    Outputs<OT> out[2] = {};
    auto load = [&](int step) {
        const int n = step / 4, q = step % 4, col0 = col_lo + 64 * n;
        if (!WHOLE && col0 >= K) return;
#pragma unroll
        for (int k = 0; k < RK; ++k)
            wv[step % (AHEAD + 1)][k] = factors<ACROSS, WHOLE>(w, aid, col0 + Outputs<OT>::column(q, i), 32 * k + 8 * g, K, R);
        if (q == 0 && res && (WHOLE || col0 + lc < K)) out[n % 2].load(res + col0, WHOLE, K - col0 - lc);
    };
#pragma unroll
    for (int step = 0; step < AHEAD; ++step) load(step);
    Frag<float> tf[RK];
    const float scale = a.scale ? a.scale[aid] : 1.0f;
    const float* part = a.part + (in ? row : a.rows - 1) * R;
#pragma unroll
    for (int k = 0; k < RK; ++k) {
        Raw<float> t = {};
        if (touch) {
            t = sum_t<WHOLE>(part, a.rows * R, a.splits, 32 * k + 8 * g, R);
            if (a.t && col_lo == 0) store_t(a.t + row * R, t, 32 * k + 8 * g, R);
        }
        tf[k] = scaled(t, scale);
    }
    f32x4 y4[4];
#pragma unroll
    for (int step = 0; step < STEPS; ++step) {
        const int n = step / 4, q = step % 4, col0 = col_lo + 64 * n;
        if (!WHOLE && col0 >= K) break;
        if (step + AHEAD < STEPS) load(step + AHEAD);
        in_order();
        f32x4 acc;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = y4[q][j] = out[n % 2].get(4 * q + j);
#pragma unroll
        for (int k = 0; k < RK; ++k) acc = product(frag(wv[step % (AHEAD + 1)][k]), tf[k], acc);
#pragma unroll
        for (int j = 0; j < 4; ++j) y4[q][j] = mine >= 0 ? acc[j] : y4[q][j];
        if (q == 3 && touch) Outputs<OT>::store(y + col0, WHOLE, K - col0 - lc, y4);
    }
}

// ---- outer -------------------------------------------------------------------------------
// The gradients: out[adapter] = sum over its rows of u[row][r] v[row][c], as [R][C] (da), or with COLS [C][R] (db), u times
// the adapter's scale.  A block has 64 columns of one adapter and a share of its rows (in the order of order[]), which
// its eight waves take in tiles of 32.  A wave copies a tile's rows (whole 128-byte pieces of bf16 ones) into LDS and
// reads the MFMA's operand, 8 rows of a column, by the transposing LDS read, the next tile's rows in flight and the rows of the
// one after that known.  The waves add through LDS at the end.  Both gradients are one launch.  Bound by reading the rows: 8192
// of 4096 and 8192 bf16 values 44 us (4.5 TB/s, part of them still in the caches), of fp32 ones 94; rank 64 100, rank 128 180 (the
// splits into bf16 parts and the gathers of u grow with the rank).
constexpr int kPitch = 72;  // elements of a tile's row in LDS: 64 and a shift of the banks
constexpr int kOuterWaves = 8;

__device__ __forceinline__ void put_tile(uint16_t* to, const Raw<uint16_t>& r) { *reinterpret_cast<u32x4*>(to) = r.v; }
__device__ __forceinline__ void put_tile(float* to, const Raw<float>& r) {
    reinterpret_cast<f32x4*>(to)[0] = f32x4{r.v[0], r.v[1], r.v[2], r.v[3]};
    reinterpret_cast<f32x4*>(to)[1] = f32x4{r.v[4], r.v[5], r.v[6], r.v[7]};
}
// Rows 8 g .. 8 g + 7 of column col0 + i.
__device__ __forceinline__ Frag<uint16_t> get_tile(const uint16_t* tile, int g, int i, int col0) {
    return Frag<uint16_t>{read_columns(tile + (8 * g + (i >> 2)) * kPitch + col0 + 4 * (i & 3), kPitch)};
}
__device__ __forceinline__ Frag<float> get_tile(const float* tile, int g, int i, int col0) {
    return frag(gather_raw(tile + 8 * g * kPitch + col0 + i, kPitch, 8));
}

template <typename VT, int RN>
__global__ __launch_bounds__(64 * kOuterWaves) void outer_kernel(const AdapterOuter o) {
    constexpr int WV = sizeof(VT) == 4 ? 6 : kOuterWaves;  // with a tile: what 64 KB of LDS hold
    constexpr int kTile = 32 * kPitch * (int)sizeof(VT), kRed = 4 * 64 * 16;
    __shared__ __attribute__((aligned(16))) char lds[WV * kTile > kOuterWaves * kRed ? WV * kTile : kOuterWaves * kRed];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const uint32_t slices = (uint32_t)(o.R + 63) / 64, block = blockIdx.x / slices;
    const int r0 = 64 * (int)(blockIdx.x % slices);  // of ranks above 64 a block has 64
    const bool second = block >= o.blocks0;
    const AdapterOuterJob& job = o.job[second ? 1 : 0];
    const VT* v = reinterpret_cast<const VT*>(job.v);
    const float* u = job.u;
    const int32_t C = job.C, R = o.R;
    const int col0 = (int)(block - (second ? o.blocks0 : 0)) * 64;
    const int aid = blockIdx.z;
    const float sc = job.scale ? job.scale[aid] : 1.0f;
    const int2 span = o.span[aid];
    const int share = ((span.y + (int)gridDim.y - 1) / (int)gridDim.y + 31) / 32 * 32;
    const int lo = share * (int)blockIdx.y < span.y ? share * (int)blockIdx.y : span.y;
    const int n = span.y - lo < share ? span.y - lo : share;  // rows of this block
    const int32_t* list = o.order + span.x + lo;

    f32x4 acc[RN][4];
#pragma unroll
    for (int m = 0; m < RN; ++m)
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[m][f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto body = [&](auto inside) {
        constexpr bool WHOLE = decltype(inside)::value;  // all 64 columns: no load has a branch
        VT* tile = reinterpret_cast<VT*>(lds + wave * kTile);
        const int e = 8 * (lane & 7);  // a row's 64 columns: 8 lanes
        Raw<VT> raw[4];
        Raw<float> ur[RN];
        // lane l: the batch's row of row l % 32 of a tile (of its last one behind the end: that one's values again, times 0)
        auto rows_of = [&](int t) { return list[t + (lane & 31) < n ? t + (lane & 31) : n - 1]; };
        auto load = [&](int t, int rows) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int lr = 8 * k + (lane >> 3);
                const int64_t row = __shfl(rows, lr, kWave);
                raw[k] = load_raw(v + row * C + col0 + e, WHOLE ? 8 : C - col0 - e);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float* ux = u + (int64_t)__shfl(rows, 8 * g + j, kWave) * R;
#pragma unroll
                for (int m = 0; m < RN; ++m) ur[m].v[j] = ux[r0 + 16 * m + i < R ? r0 + 16 * m + i : R - 1];
            }
        };
        constexpr int STEP = 32 * WV;
        int t = wave * 32, rows = 0;
        if (t < n) {
            rows = rows_of(t);
            load(t, rows);
            if (t + STEP < n) rows = rows_of(t + STEP);
        }
        for (; t < n; t += STEP) {
#pragma unroll
            for (int k = 0; k < 4; ++k) put_tile(tile + (8 * k + (lane >> 3)) * kPitch + e, raw[k]);
            Frag<float> uf[RN];
#pragma unroll
            for (int m = 0; m < RN; ++m) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    ur[m].v[j] = t + 8 * g + j < n && r0 + 16 * m + i < R ? ur[m].v[j] * sc : 0.0f;
                uf[m] = frag(ur[m]);
            }
            if (t + STEP < n) {
                load(t + STEP, rows);
                if (t + 2 * STEP < n) rows = rows_of(t + 2 * STEP);
            }
            in_order();
            // the tile is the wave's own: its stores before these reads, in program order
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const Frag<VT> vf = get_tile(tile, g, i, 16 * f);
#pragma unroll
                for (int m = 0; m < RN; ++m) acc[m][f] = product(uf[m], vf, acc[m][f]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (wave < WV) {
        if (col0 + 64 <= C) body(std::true_type());
        else body(std::false_type());
    }
    float* out = job.out + ((int64_t)blockIdx.y * o.split_stride + (int64_t)aid * R * C);
    f32x4* red = reinterpret_cast<f32x4*>(lds);  // [waves][4 * 64]
#pragma unroll
    for (int m = 0; m < RN; ++m) {
        __syncthreads();
#pragma unroll
        for (int f = 0; f < 4; ++f) red[wave * 256 + f * 64 + lane] = acc[m][f];
        __syncthreads();
        if (threadIdx.x >= 256) continue;
        f32x4 s = red[threadIdx.x];
#pragma unroll
        for (int k = 1; k < kOuterWaves; ++k) s += red[k * 256 + threadIdx.x];
        const int c = col0 + 16 * wave + i;  // thread = (column tile wave, lane)
        if (c < C) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = r0 + 16 * m + 4 * g + j;
                if (r < R) out[job.cols ? (int64_t)c * R + r : (int64_t)r * C + c] = s[j];
            }
        }
    }
}

// da[i], db[i] = the sum over the splits, in order; part: [splits][na + nb].
__global__ __launch_bounds__(256) void outer_sum_kernel(const float* __restrict__ part, int32_t splits, int64_t na,
                                                        int64_t nb, float* __restrict__ da, float* __restrict__ db) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < na + nb; i += (int64_t)gridDim.x * 256) {
        float s = part[i];
        for (int k = 1; k < splits; ++k) s += part[k * (na + nb) + i];
        if (i < na) da[i] = s;
        else db[i - na] = s;
    }
}

// ---- launches ----------------------------------------------------------------------------
int tiles16(int32_t R) { return R <= 16 ? 1 : R <= 32 ? 2 : 4; }

template <typename XT, typename WT, bool ACROSS>
void shrink(const AdapterArgs& args, const AdapterPlan& p, hipStream_t s) {
    AdapterArgs a = args;
    a.splits = p.splits;
    a.row_blocks = (uint32_t)((a.rows + 16 * p.row_tiles - 1) / (16 * p.row_tiles) * p.splits * ((a.R + 63) / 64));
    const dim3 grid(a.row_blocks + (a.order && !a.sorted ? (uint32_t)a.S : 0u), (unsigned)p.slots);
#define TBN_SHRINK(rn, rt, sorted) \
    hipLaunchKernelGGL((shrink_kernel<XT, WT, ACROSS, sorted, rn, rt, kShrinkWaves>), grid, dim3(64 * kShrinkWaves), 0, s, a)
    switch (tiles16(a.R) * 8 + p.row_tiles + (a.sorted ? 64 : 0)) {
        case 9: TBN_SHRINK(1, 1, false); break;
        case 12: TBN_SHRINK(1, 4, false); break;
        case 17: TBN_SHRINK(2, 1, false); break;
        case 20: TBN_SHRINK(2, 4, false); break;
        case 33: TBN_SHRINK(4, 1, false); break;
        case 34: TBN_SHRINK(4, 2, false); break;
        case 64 + 12: TBN_SHRINK(1, 4, true); break;
        case 64 + 20: TBN_SHRINK(2, 4, true); break;
        default: TBN_SHRINK(4, 2, true);
    }
#undef TBN_SHRINK
}

template <typename WT, typename OT, bool ACROSS>
void expand(const AdapterArgs& a, hipStream_t s) {
    if (adapter_few_rows(a.rows, a.S)) {
        const int64_t tiles = (a.rows + 15) / 16, slots = a.S < 16 ? a.S : 16;  // no tile holds more adapters
        const dim3 grid((unsigned)((a.C + 256 * kGroups - 1) / (256 * kGroups)), (unsigned)tiles,
                        (unsigned)(slots < a.rows ? slots : a.rows));
#define TBN_EXPAND(rk)                                                                                                 \
    if (a.R % 8 == 0 && a.C % (64 * kGroups) == 0)                                                                     \
        hipLaunchKernelGGL((expand_few_kernel<WT, OT, ACROSS, true, rk>), grid, dim3(256), 0, s, a);                   \
    else hipLaunchKernelGGL((expand_few_kernel<WT, OT, ACROSS, false, rk>), grid, dim3(256), 0, s, a)
        if (a.R <= 32) {
            TBN_EXPAND(1);
        } else if (a.R <= 64) {
            TBN_EXPAND(2);
        } else {
            TBN_EXPAND(4);
        }
#undef TBN_EXPAND
        return;
    }
    // Groups of 64 columns a wave: what 64 KB of LDS and 128 registers (two blocks a CU) hold.  With 64 columns up to rank 64
    // 8192 rows of 4096 and fp32 adapters of rank 64 took 68 us instead of 57; with 128 for higher ranks, which spills more,
    // 5000 rows of 8192 took 67 instead of 54.  Small batches take 64 columns, for more blocks: 100 rows of 512, 4.7 us
    // instead of 7.8.
    constexpr int kNarrow = 1, kMiddle = 2, kWide = 4;
    const int64_t tiles = (a.rows + 16 * kExpandWaves - 1) / (16 * kExpandWaves);
    const bool wide = tiles * ((a.C + 63) / 64) >= 1024;
#define TBN_EXPAND(rk, n)                                                                                             \
    hipLaunchKernelGGL((expand_kernel<WT, OT, ACROSS, rk, n>), dim3((unsigned)((a.C + 64 * n - 1) / (64 * n) * tiles)), \
                       dim3(64 * kExpandWaves), 0, s, a)
    if (a.R <= 32) {
        if (wide) TBN_EXPAND(1, kWide);
        else TBN_EXPAND(1, kNarrow);
    } else if (a.R <= 64) {
        if (wide) TBN_EXPAND(2, kMiddle);
        else TBN_EXPAND(2, kNarrow);
    } else {
        TBN_EXPAND(4, kNarrow);
    }
#undef TBN_EXPAND
}

template <typename VT>
void outer(const AdapterOuter& o, int32_t S, int32_t splits, hipStream_t s) {
    const unsigned slices = (unsigned)(o.R + 63) / 64;
    const dim3 grid((o.blocks0 + (unsigned)(o.job[1].out ? (o.job[1].C + 63) / 64 : 0)) * slices, (unsigned)splits, (unsigned)S);
#define TBN_OUTER(rn) hipLaunchKernelGGL((outer_kernel<VT, rn>), grid, dim3(64 * kOuterWaves), 0, s, o)
    switch (tiles16(o.R)) {
        case 1: TBN_OUTER(1); break;
        case 2: TBN_OUTER(2); break;
        default: TBN_OUTER(4);
    }
#undef TBN_OUTER
}

}  // namespace

AdapterPlan plan_adapter_shrink(int64_t rows, int32_t C, int32_t R, int32_t S) {
    AdapterPlan p;
    // Tiles of 16 rows also where a small bank's rows are expanded 128 at a time: 100 rows of 1000 values, rank 8, 5.7 us instead
    // of 7.1; 128 of 8192, rank 64, 6.1 instead of 7.3 (512 of 8192, one adapter of rank 16, 9 instead of 7).
    const bool few = rows <= 128 || adapter_few_rows(rows, S);
    p.row_tiles = few ? 1 : R <= 32 ? 4 : 2;
    p.slots = few ? (S < 16 ? S : 16) : 1;
    if (p.slots > rows) p.slots = (int32_t)rows;
    const int64_t tiles = (rows + 16 * p.row_tiles - 1) / (16 * p.row_tiles);
    // Enough blocks to fill the chip, two steps of the waves each at least.  With few rows also where each tile has one
    // adapter: 512 rows of 8192 values of one adapter take 9 us with 4 splits, 17 with one (of 512 adapters 31 either way).
    // For long batches (see the kernel's note) eight splits, four where their partial sums are a larger share of the traffic.
    const int64_t one = (128 + tiles - 1) / tiles;
    const int64_t least = few ? (one < 8 ? one : 8) : R <= 32 ? 8 : 4, most = C / (2 * 64 * kShrinkWaves);
    int64_t splits = few ? 512 / (tiles * p.slots) : 640 / tiles;
    if (splits < least) splits = least;
    if (splits > most) splits = most;
    p.splits = (int32_t)(splits < 1 ? 1 : splits);
    return p;
}

int32_t adapter_outer_splits(int64_t rows, int32_t C, int32_t K, int32_t S) {
    const int64_t blocks = (int64_t)((C + 63) / 64 + (K + 63) / 64) * S;
    int64_t splits = 2048 / blocks;
    const int64_t most = (rows + 255) / 256;  // two tiles a wave at least
    if (splits > most) splits = most;
    return (int32_t)(splits < 1 ? 1 : splits);
}

hipError_t launch_adapter_order(const AdapterArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(order_kernel, dim3((unsigned)a.S + 1u), dim3(1024), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_adapter_shrink(const AdapterArgs& a, const AdapterPlan& p, int across, hipStream_t s) {
    if (across) {
        if (a.x_f32) a.w_f32 ? shrink<float, float, true>(a, p, s) : shrink<float, uint16_t, true>(a, p, s);
        else a.w_f32 ? shrink<uint16_t, float, true>(a, p, s) : shrink<uint16_t, uint16_t, true>(a, p, s);
    } else {
        if (a.x_f32) a.w_f32 ? shrink<float, float, false>(a, p, s) : shrink<float, uint16_t, false>(a, p, s);
        else a.w_f32 ? shrink<uint16_t, float, false>(a, p, s) : shrink<uint16_t, uint16_t, false>(a, p, s);
    }
    return hipGetLastError();
}

hipError_t launch_adapter_finish(const float* part, int64_t count, int32_t splits, float* t, hipStream_t s) {
    int64_t blocks = (count + 255) / 256;
    if (blocks > 2048) blocks = 2048;
    hipLaunchKernelGGL(finish_kernel, dim3((unsigned)blocks), dim3(256), 0, s, part, count, splits, t);
    return hipGetLastError();
}

hipError_t launch_adapter_expand(const AdapterArgs& a, int across, hipStream_t s) {
    if (across) {
        if (a.w_f32) a.y_f32 ? expand<float, float, true>(a, s) : expand<float, uint16_t, true>(a, s);
        else a.y_f32 ? expand<uint16_t, float, true>(a, s) : expand<uint16_t, uint16_t, true>(a, s);
    } else {
        if (a.w_f32) a.y_f32 ? expand<float, float, false>(a, s) : expand<float, uint16_t, false>(a, s);
        else a.y_f32 ? expand<uint16_t, float, false>(a, s) : expand<uint16_t, uint16_t, false>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_adapter_outer(const AdapterOuter& o, int32_t S, int32_t splits, int v_f32, hipStream_t s) {
    v_f32 ? outer<float>(o, S, splits, s) : outer<uint16_t>(o, S, splits, s);
    return hipGetLastError();
}

hipError_t launch_adapter_outer_sum(const float* part, int32_t splits, int64_t na, int64_t nb, float* da, float* db,
                                    hipStream_t s) {
    int64_t blocks = (na + nb + 255) / 256;
    if (blocks > 8192) blocks = 8192;
    hipLaunchKernelGGL(outer_sum_kernel, dim3((unsigned)blocks), dim3(256), 0, s, part, splits, na, nb, da, db);
    return hipGetLastError();
}

}  // namespace tbn
