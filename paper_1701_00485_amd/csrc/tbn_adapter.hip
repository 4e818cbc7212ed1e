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
// All run on v_mfma_f32_16x16x32_bf16.  What has 32 bits (t, dt, fp32 weights or rows) enters exactly, as the sum of three
// bf16 numbers (8 bits each), and a product of two such factors leaves out only the parts below 2^-23 of it: every result is
// one of fp32 sums, a bf16 one rounded once.  Two parts, 16 bits, would save a third of these MFMAs, which do not
// bound any of the kernels, and cost gradients that are off by 4e-6.
//
// Rows may lie in any order: a tile of rows is run once for each adapter that it holds, and each row takes the
// result of its own (nothing of another row or adapter enters it, NaN included); tiles of one request's rows run once.
// The gradients gather the rows of their adapter into a list first.  An index outside [0, S) is no adapter.
// Every sum is in a fixed order.
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

// 8 neighbouring values, or the first `left` of them and zeros.
__device__ __forceinline__ Frag<uint16_t> load_frag(const uint16_t* p, int64_t left) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (left >= 8) {
        w = *reinterpret_cast<const u32x4_a2*>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) w[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
    }
    return Frag<uint16_t>{as_bf16x8(w)};
}
__device__ __forceinline__ void load_f32(const float* p, int64_t left, float (&v)[8]) {
    if (left >= 8) {
        const f32x4 a = *reinterpret_cast<const f32x4_a4*>(p), b = *reinterpret_cast<const f32x4_a4*>(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = a[j];
            v[4 + j] = b[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < left ? p[j] : 0.0f;
    }
}
__device__ __forceinline__ Frag<float> load_frag(const float* p, int64_t left) {
    float v[8];
    load_f32(p, left, v);
    return split8(v);
}
// 8 values `stride` apart.
__device__ __forceinline__ Frag<uint16_t> gather_frag(const uint16_t* p, int64_t stride, int64_t left) {
    u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) w[j / 2] |= (uint32_t)p[j * stride] << (16 * (j & 1));
    return Frag<uint16_t>{as_bf16x8(w)};
}
__device__ __forceinline__ Frag<float> gather_frag(const float* p, int64_t stride, int64_t left) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? p[j * stride] : 0.0f;
    return split8(v);
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

// The adapter of a row, -1 for none.
__device__ __forceinline__ int adapter_of(const int32_t* index, int64_t row, int32_t S) {
    const int32_t a = index[row];
    return (uint32_t)a < (uint32_t)S ? a : -1;
}

// ---- shrink ------------------------------------------------------------------------------
// out[split][row][r] = scale sum over the split's c of x[row][c] W[r][c], W = the row's adapter: [R][C], or with ACROSS
// [C][R].  A block has a tile of 16 RT rows and one split; its four waves take every fourth 32 values of c and
// add through LDS.  With gridDim.z > 1 (few rows, each with its own adapter) the tile's adapters are dealt over z.
template <typename XT, typename WT, bool ACROSS, int RN, int RT>
__global__ __launch_bounds__(256) void shrink_kernel(const AdapterArgs a) {
    __shared__ f32x4 red[4][RN * RT * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i = lane & 15, g = lane >> 4;
    const XT* x = reinterpret_cast<const XT*>(a.x);
    const WT* w = reinterpret_cast<const WT*>(a.w);
    const int64_t row0 = (int64_t)blockIdx.x * (16 * RT);
    const int rows = a.rows - row0 < 16 * RT ? (int)(a.rows - row0) : 16 * RT;
    const int32_t C = a.C, R = a.R;
    const int c_lo = blockIdx.y * a.per_split;
    const int c_hi = C - c_lo < a.per_split ? C : c_lo + a.per_split;
    float* out = a.part + ((int64_t)blockIdx.y * a.rows + row0) * R;

    const int mine = lane < rows ? adapter_of(a.index, row0 + lane, a.S) : -1;
    uint64_t todo = __ballot(mine >= 0);
    const XT* xr[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int r = 16 * t + i < rows ? 16 * t + i : rows - 1;
        xr[t] = x + (row0 + r) * C + 8 * g;
    }
    for (uint32_t slot = 0; todo; ++slot) {
        const int aid = __builtin_amdgcn_readfirstlane(__shfl(mine, __ffsll((unsigned long long)todo) - 1, kWave));
        const uint64_t same = __ballot(mine == aid);
        todo &= ~same;
        if (slot % gridDim.z != blockIdx.z) continue;
        const WT* wr[RN];
#pragma unroll
        for (int n = 0; n < RN; ++n) {
            const int r = 16 * n + i < R ? 16 * n + i : R - 1;
            wr[n] = w + (int64_t)aid * R * C + (ACROSS ? (int64_t)8 * g * R + r : (int64_t)r * C + 8 * g);
        }
        f32x4 acc[RN][RT];
#pragma unroll
        for (int n = 0; n < RN; ++n)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[n][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        auto step = [&](int c, int left) {
            Frag<WT> wf[RN];
            Frag<XT> xf[RT];
#pragma unroll
            for (int n = 0; n < RN; ++n)
                wf[n] = ACROSS ? gather_frag(wr[n] + (int64_t)c * R, R, left) : load_frag(wr[n] + c, left);
#pragma unroll
            for (int t = 0; t < RT; ++t) xf[t] = load_frag(xr[t] + c, left);
#pragma unroll
            for (int n = 0; n < RN; ++n)
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[n][t] = product(wf[n], xf[t], acc[n][t]);
        };
        int c = c_lo + 32 * wave;
        for (; c + 32 <= c_hi; c += 128) step(c, 8);
        if (c < c_hi) step(c, C - c - 8 * g);  // the last, shorter 32 values
#pragma unroll
        for (int n = 0; n < RN; ++n)
#pragma unroll
            for (int t = 0; t < RT; ++t) red[wave][(n * RT + t) * 64 + lane] = acc[n][t];
        __syncthreads();
        const float sc = a.scale ? a.scale[aid] : 1.0f;
        for (int o = threadIdx.x; o < RN * RT * 64; o += 256) {
            const f32x4 s = (red[0][o] + red[1][o]) + (red[2][o] + red[3][o]);
            const int l = o & 63, n = (o >> 6) / RT, row = 16 * ((o >> 6) % RT) + (l & 15);
            if (!(same >> row & 1)) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 16 * n + 4 * (l >> 4) + j;
                if (r < R) out[(int64_t)row * R + r] = sc * s[j];
            }
        }
        __syncthreads();
    }
    if (blockIdx.z == 0 && wave == 0) {  // rows without an adapter
        uint64_t none = __ballot(lane < rows && mine < 0);
        while (none) {
            const int row = __ffsll((unsigned long long)none) - 1;
            none &= none - 1;
            for (int r = lane; r < R; r += 64) out[(int64_t)row * R + r] = 0.0f;
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
// t = the sum of `splits` partial ones.  A wave has 64 columns, whose factors stay in registers from one tile of 16
// rows to the next while the adapter does.  Rows of the MFMA's result are dealt to columns so that a lane holds 16
// neighbouring ones of one row: 16-byte residual reads and stores.
template <typename T>
__device__ __forceinline__ void load_out(const T* p, int left, float (&y)[16]);
template <>
__device__ __forceinline__ void load_out(const float* p, int left, float (&y)[16]) {
    if (left >= 16) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = reinterpret_cast<const f32x4_a4*>(p)[q];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[4 * q + j] = v[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = j < left ? p[j] : 0.0f;
    }
}
template <>
__device__ __forceinline__ void load_out(const uint16_t* p, int left, float (&y)[16]) {
    if (left >= 16) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const u32x4 v = reinterpret_cast<const u32x4_a2*>(p)[q];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[8 * q + 2 * j] = __uint_as_float(v[j] << 16);
                y[8 * q + 2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = j < left ? bf16_bits_to_f32(p[j]) : 0.0f;
    }
}
__device__ __forceinline__ void store_out(float* p, int left, const float (&y)[16]) {
    if (left >= 16) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            reinterpret_cast<f32x4_a4*>(p)[q] = f32x4{y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]};
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < left) p[j] = y[j];
    }
}
__device__ __forceinline__ void store_out(uint16_t* p, int left, const float (&y)[16]) {
    if (left >= 16) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = pack_bf16x2(y[8 * q + 2 * j], y[8 * q + 2 * j + 1]);
            reinterpret_cast<u32x4_a2*>(p)[q] = v;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < left) p[j] = (uint16_t)f32_to_bf16_bits(y[j]);
    }
}

template <typename WT, typename OT, bool ACROSS, int RK>
__global__ __launch_bounds__(256) void expand_kernel(const AdapterArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i = lane & 15, g = lane >> 4;
    const int32_t K = a.C, R = a.R;
    const int col0 = (blockIdx.x * 4 + wave) * 64;
    if (col0 >= K) return;
    const WT* w = reinterpret_cast<const WT*>(a.w);
    const OT* res = reinterpret_cast<const OT*>(a.residual);
    OT* y = reinterpret_cast<OT*>(a.y);
    const int64_t tiles = (a.rows + 15) / 16;
    const bool writes_t = a.t && col0 == 0;
    const int out_col = col0 + 16 * g, out_left = K - out_col;
    Frag<WT> wf[4][RK];
    int held = -1;
    for (int64_t tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
        const int64_t row = tile * 16 + i;
        const bool in = row < a.rows;
        const int mine = in ? adapter_of(a.index, row, a.S) : -1;
        float out[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) out[j] = 0.0f;
        if (in && res && out_left > 0) load_out(res + row * K + out_col, out_left, out);
        Frag<float> tf[RK];
        const float sc = mine >= 0 && a.scale ? a.scale[mine] : 1.0f;
#pragma unroll
        for (int k = 0; k < RK; ++k) {
            const int r = 32 * k + 8 * g, left = in ? R - r : 0;
            float v[8];
            load_f32(a.part + row * R + r, left, v);
            for (int s = 1; s < a.splits; ++s) {
                float u[8];
                load_f32(a.part + ((int64_t)s * a.rows + row) * R + r, left, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += u[j];
            }
            if (writes_t) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) a.t[row * R + r + j] = v[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= sc;
            tf[k] = split8(v);
        }
        uint32_t todo = (uint32_t)__ballot(mine >= 0) & 0xFFFFu;
        while (todo) {
            const int aid = __builtin_amdgcn_readfirstlane(__shfl(mine, __ffs(todo) - 1, kWave));
            todo &= ~(uint32_t)__ballot(mine == aid);
            if (aid != held) {
                held = aid;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    int col = col0 + 16 * (i >> 2) + 4 * q + (i & 3);
                    col = col < K ? col : K - 1;
#pragma unroll
                    for (int k = 0; k < RK; ++k) {
                        const int r = 32 * k + 8 * g;
                        wf[q][k] = ACROSS ? gather_frag(w + ((int64_t)aid * R + r) * K + col, K, R - r)
                                          : load_frag(w + ((int64_t)aid * K + col) * R + r, R - r);
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < RK; ++k) acc = product(wf[q][k], tf[k], acc);
                if (mine == aid) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) out[4 * q + j] += acc[j];
                }
            }
        }
        if (in && out_left > 0) store_out(y + row * K + out_col, out_left, out);
    }
}

// ---- outer -------------------------------------------------------------------------------
// out[adapter] = sum over its rows of u[row][r] v[row][c], as [R][C], or with COLS [C][R]; u times the adapter's scale.
// A block has 64 columns of one adapter and a range of the rows; it gathers the adapter's rows, kList rows of the
// batch at a time, into a list, whose tiles of 32 its four waves take in turn: v through the wave's own LDS tile
// (16-byte copies in, the MFMA's 8 rows of a column out).  The waves add through LDS at the end.
constexpr int kList = 4096;
constexpr int kPitch = 72;  // elements of a tile's row in LDS: 64 and a shift of the banks

__device__ __forceinline__ void put_tile(uint16_t* to, const uint16_t* p, int left) {
    *reinterpret_cast<bf16x8*>(to) = load_frag(p, left).hi;
}
__device__ __forceinline__ void put_tile(float* to, const float* p, int left) {
    float v[8];
    load_f32(p, left, v);
    reinterpret_cast<f32x4*>(to)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4*>(to)[1] = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ Frag<uint16_t> column(const uint16_t* tile, int g, int col) {
    return gather_frag(tile + 8 * g * kPitch + col, kPitch, 8);
}
__device__ __forceinline__ Frag<float> column(const float* tile, int g, int col) {
    return gather_frag(tile + 8 * g * kPitch + col, kPitch, 8);
}

template <typename VT, bool COLS, int RN>
__global__ __launch_bounds__(256) void outer_kernel(const AdapterArgs a) {
    __shared__ uint16_t list[kList];
    __shared__ int counts[4];
    __shared__ __attribute__((aligned(16))) VT tiles[4][32 * kPitch];
    __shared__ f32x4 red[4][4 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i = lane & 15, g = lane >> 4;
    const VT* v = reinterpret_cast<const VT*>(a.x);
    const int32_t C = a.C, R = a.R;
    const int col0 = blockIdx.x * 64;
    const int aid = blockIdx.z;
    const float sc = a.scale ? a.scale[aid] : 1.0f;
    const int64_t r_lo = (int64_t)blockIdx.y * a.per_split;
    const int64_t r_hi = a.rows - r_lo < a.per_split ? a.rows : r_lo + a.per_split;
    VT* tile = tiles[wave];

    f32x4 acc[RN][4];
#pragma unroll
    for (int n = 0; n < RN; ++n)
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[n][f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (int64_t base = r_lo; base < r_hi; base += kList) {
        // the adapter's rows among these kList: each wave lists a quarter, behind those of the waves before it
        constexpr int kMine = kList / 4 / 64;
        const int64_t first = base + wave * (kList / 4);
        uint32_t found = 0;
        int count = 0;
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int64_t row = first + 64 * k + lane;
            const bool is = row < r_hi && a.index[row < r_hi ? row : r_lo] == aid;
            found |= (uint32_t)is << k;
            count += __popcll(__ballot(is));
        }
        __syncthreads();  // the list's readers of the round before are done
        if (lane == 0) counts[wave] = count;
        __syncthreads();
        int at = 0, n = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            at += k < wave ? counts[k] : 0;
            n += counts[k];
        }
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const bool is = found >> k & 1;
            const uint64_t m = __ballot(is);
            if (is) list[at + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)(wave * (kList / 4) + 64 * k + lane);
            at += __popcll(m);
        }
        __syncthreads();
        for (int t = wave * 32; t < n; t += 128) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int lr = 8 * k + (lane >> 3), e = 8 * (lane & 7);
                const bool in = t + lr < n;
                const int64_t row = base + (in ? list[t + lr] : 0);
                const int left = in ? C - col0 - e : 0;
                put_tile(tile + lr * kPitch + e, v + row * C + col0 + e, left);
            }
            Frag<float> uf[RN];
#pragma unroll
            for (int n2 = 0; n2 < RN; ++n2) {
                float u[8];
                const int r = 16 * n2 + i;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int lr = t + 8 * g + j;
                    u[j] = lr < n && r < R ? sc * a.part[(base + list[lr]) * R + r] : 0.0f;
                }
                uf[n2] = split8(u);
            }
            // the tile is the wave's own: its stores before these reads, in program order
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const Frag<VT> vf = column(tile, g, 16 * f + i);
#pragma unroll
                for (int n2 = 0; n2 < RN; ++n2) acc[n2][f] = product(uf[n2], vf, acc[n2][f]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    float* out = a.out + ((int64_t)blockIdx.y * a.S + aid) * R * C;
#pragma unroll
    for (int n = 0; n < RN; ++n) {
        __syncthreads();
#pragma unroll
        for (int f = 0; f < 4; ++f) red[wave][f * 64 + lane] = acc[n][f];
        __syncthreads();
        const f32x4 s = (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
        const int c = col0 + 16 * wave + i;  // thread = (column tile wave, lane)
        if (c < C) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 16 * n + 4 * g + j;
                if (r < R) out[COLS ? (int64_t)c * R + r : (int64_t)r * C + c] = s[j];
            }
        }
    }
}

// ---- launches ----------------------------------------------------------------------------
int tiles16(int32_t R) { return R <= 16 ? 1 : R <= 32 ? 2 : R <= 64 ? 4 : 8; }

template <typename XT, typename WT, bool ACROSS>
void shrink(const AdapterArgs& a, const AdapterPlan& p, hipStream_t s) {
    const dim3 grid((unsigned)((a.rows + 16 * p.row_tiles - 1) / (16 * p.row_tiles)), (unsigned)p.splits, (unsigned)p.slots);
#define TBN_SHRINK(rn, rt) hipLaunchKernelGGL((shrink_kernel<XT, WT, ACROSS, rn, rt>), grid, dim3(256), 0, s, a)
    switch (tiles16(a.R) * 8 + p.row_tiles) {
        case 9: TBN_SHRINK(1, 1); break;
        case 12: TBN_SHRINK(1, 4); break;
        case 17: TBN_SHRINK(2, 1); break;
        case 20: TBN_SHRINK(2, 4); break;
        case 33: TBN_SHRINK(4, 1); break;
        case 34: TBN_SHRINK(4, 2); break;
        default: TBN_SHRINK(8, 1);
    }
#undef TBN_SHRINK
}

template <typename WT, typename OT, bool ACROSS>
void expand(const AdapterArgs& a, hipStream_t s) {
    const int64_t blocks = (a.C + 255) / 256, tiles = (a.rows + 15) / 16;
    int64_t y = 2048 / blocks;  // eight blocks of a CU at once
    y = y < 1 ? 1 : y > tiles ? tiles : y;
    if (y > 65535) y = 65535;
    const dim3 grid((unsigned)blocks, (unsigned)y);
#define TBN_EXPAND(rk) hipLaunchKernelGGL((expand_kernel<WT, OT, ACROSS, rk>), grid, dim3(256), 0, s, a)
    if (a.R <= 32) TBN_EXPAND(1);
    else if (a.R <= 64) TBN_EXPAND(2);
    else TBN_EXPAND(4);
#undef TBN_EXPAND
}

template <typename VT, bool COLS>
void outer(const AdapterArgs& a, int32_t splits, hipStream_t s) {
    const dim3 grid((unsigned)((a.C + 63) / 64), (unsigned)splits, (unsigned)a.S);
#define TBN_OUTER(rn) hipLaunchKernelGGL((outer_kernel<VT, COLS, rn>), grid, dim3(256), 0, s, a)
    switch (tiles16(a.R)) {
        case 1: TBN_OUTER(1); break;
        case 2: TBN_OUTER(2); break;
        case 4: TBN_OUTER(4); break;
        default: TBN_OUTER(8);
    }
#undef TBN_OUTER
}

}  // namespace

AdapterPlan plan_adapter_shrink(int64_t rows, int32_t C, int32_t R, int32_t S) {
    AdapterPlan p;
    const bool few = rows <= kAdapterFewRows;
    p.row_tiles = few ? 1 : R <= 32 ? 4 : R <= 64 ? 2 : 1;
    p.slots = few ? (int32_t)(S < 16 ? S : 16) : 1;
    if (p.slots > rows) p.slots = (int32_t)rows;
    const int64_t tiles = (rows + 16 * p.row_tiles - 1) / (16 * p.row_tiles) * p.slots;
    int64_t splits = 1024 / tiles;
    const int64_t most = (C + 255) / 256;  // two rounds of the four waves at least
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    p.per_split = (int32_t)(((C + splits - 1) / splits + 127) / 128 * 128);
    p.splits = (C + p.per_split - 1) / p.per_split;
    return p;
}

int32_t adapter_outer_splits(int64_t rows, int32_t C, int32_t S, int64_t* per_split) {
    const int64_t blocks = (int64_t)((C + 63) / 64) * S;
    int64_t splits = 1024 / blocks;
    const int64_t most = (rows + 511) / 512;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    *per_split = ((rows + splits - 1) / splits + 31) / 32 * 32;
    return (int32_t)((rows + *per_split - 1) / *per_split);
}

hipError_t launch_adapter_shrink(const AdapterArgs& args, const AdapterPlan& p, int across, hipStream_t s) {
    AdapterArgs a = args;
    a.per_split = p.per_split;
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

hipError_t launch_adapter_outer(const AdapterArgs& args, int32_t splits, int64_t per_split, int cols, float* partial,
                                float* out, hipStream_t s) {
    AdapterArgs a = args;
    a.per_split = per_split;
    a.out = splits > 1 ? partial : out;
    if (cols) a.x_f32 ? outer<float, true>(a, splits, s) : outer<uint16_t, true>(a, splits, s);
    else a.x_f32 ? outer<float, false>(a, splits, s) : outer<uint16_t, false>(a, splits, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    const int64_t count = (int64_t)a.S * a.R * a.C;
    return launch_split_reduce(partial, splits, count, count, out, 0, s);
}

}  // namespace tbn
