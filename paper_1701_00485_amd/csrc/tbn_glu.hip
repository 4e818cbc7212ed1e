// tbn_glu.hip -- the gated block of two-bit filters: f gates and f others over the same c features,
//   g = alpha_g (x W~_g),  u = alpha_u (x W~_u),  h = act(g) u,
// both projections, the activation and the product in one kernel; and the gradient dg = dh u act'(g), du = dh act(g), from
// the g and u that the forward pass kept or, with the same products again, from x.
//
// The codes of the 2 f filters are packed as those of one layer, gates first (TBN2, see tbn.h).
#include "tbn_kernels.h"
#include "tbn_nt.h"

namespace tbn {

namespace {

// ---- activations, in fp32 ----------------------------------------------------------------
// act(g) and, for the backward pass, its derivative.
//   silu  g s, s = 1 / (1 + e^-g);            s (1 + g (1 - s))
//   gelu  g phi, phi = (1 + erf(g / sqrt 2)) / 2;   phi + g e^(-g^2 / 2) / sqrt(2 pi)
//   relu  max(g, 0);                          1 where g > 0, else 0
template <bool SLOPE>
__device__ __forceinline__ float activate(int act, float g, float* slope) {
    if (act == TBN_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        if (SLOPE) *slope = s * (1.0f + g * (1.0f - s));
        return g * s;
    }
    if (act == TBN_ACT_GELU) {
        const float phi = 0.5f * (1.0f + erff(g * 0.70710678f));
        if (SLOPE) *slope = phi + g * expf(-0.5f * g * g) * 0.39894228f;
        return g * phi;
    }
    if (SLOPE) *slope = g > 0.0f ? 1.0f : (g != g ? g : 0.0f);
    return g > 0.0f || g != g ? g : 0.0f;
}

__device__ __forceinline__ void unpack8(u32x4 r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = bf16_bits_to_f32(r[e] & 0xFFFFu), v[2 * e + 1] = __uint_as_float(r[e] & 0xFFFF0000u);
}

// Eight values of a row whose first has index `at`, `n` of them real; `whole`: all, and 16-byte aligned.
__device__ __forceinline__ void get8(const uint16_t* p, int64_t at, int n, bool whole, float (&v)[8]) {
    if (whole) {
        unpack8(*reinterpret_cast<const u32x4*>(p + at), v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? bf16_bits_to_f32(p[at + e]) : 0.0f;
}
__device__ __forceinline__ void put8(uint16_t* p, int64_t at, int n, bool whole, const float (&v)[8]) {
    if (whole) {
        *reinterpret_cast<u32x4*>(p + at) =
            u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[at + e] = (uint16_t)f32_to_bf16_bits(v[e]);
}
__device__ __forceinline__ void put8(float* p, int64_t at, int n, bool whole, const float (&v)[8]) {
    if (whole) {
        reinterpret_cast<f32x4*>(p + at)[0] = f32x4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<f32x4*>(p + at)[1] = f32x4{v[4], v[5], v[6], v[7]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[at + e] = v[e];
}

// What follows g and u of columns k .. k + 7 of row m (n of them real): h, the kept projections or the gradients.
template <int ACT>
__device__ __forceinline__ void finish8(const GluArgs& a, int64_t m, int32_t k, int n, bool whole, const float (&g)[8], const float (&u)[8]) {
    const int64_t o = m * a.f + k, og = m * 2 * a.f + k;
    float h[8];
    if (a.dh) {
        float dh[8], dg[8], du[8];
        get8(a.dh, o, n, whole, dh);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float slope;
            const float y = activate<true>(ACT, g[e], &slope);
            dg[e] = dh[e] * u[e] * slope;
            du[e] = dh[e] * y;
            h[e] = y * u[e];
        }
        put8(a.gu, og, n, whole, dg);
        put8(a.gu, og + a.f, n, whole, du);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = activate<false>(ACT, g[e], nullptr) * u[e];
        if (a.gu) {
            put8(a.gu, og, n, whole, g);
            put8(a.gu, og + a.f, n, whole, u);
        }
    }
    if (!a.h) return;
    if (a.h_f32)
        put8(reinterpret_cast<float*>(a.h), o, n, whole, h);
    else
        put8(reinterpret_cast<uint16_t*>(a.h), o, n, whole, h);
}

// ... of one column.
template <int ACT>
__device__ __forceinline__ void finish1(const GluArgs& a, int64_t m, int32_t k, float g, float u) {
    const int64_t o = m * a.f + k, og = m * 2 * a.f + k;
    float h, first = g, second = u;
    if (a.dh) {
        float slope;
        const float dh = bf16_bits_to_f32(a.dh[o]), y = activate<true>(ACT, g, &slope);
        first = dh * u * slope;
        second = dh * y;
        h = y * u;
    } else {
        h = activate<false>(ACT, g, nullptr) * u;
    }
    if (a.gu) {
        a.gu[og] = (uint16_t)f32_to_bf16_bits(first);
        a.gu[og + a.f] = (uint16_t)f32_to_bf16_bits(second);
    }
    if (!a.h) return;
    if (a.h_f32)
        reinterpret_cast<float*>(a.h)[o] = h;
    else
        reinterpret_cast<uint16_t*>(a.h)[o] = (uint16_t)f32_to_bf16_bits(h);
}

// ---- many rows ---------------------------------------------------------------------------
// A block owns BM rows and NH gates with the NH others of the same columns, so that a lane holds the g and the u of an
// output.  Rows of x go through LDS as in tbn_nt.h (64 features a stage, a ring of STAGES); of the 2 NH filters the
// stage's codes, 16 bytes each, decoded in registers into bf16 pairs, two operations a pair.
// GROUPS groups of such waves, each with a part of the stages and a ring of its own, serve tiles that are too few to fill the GPU; the
// first adds the others' sums.
template <int BM, int NH, int WAVES_M, int WAVES_N, int STAGES, int GROUPS, int ACT>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N * GROUPS, BM * NH >= 32768 || GROUPS > 1 ? 1 : 2) void glu_kernel(const GluArgs a) {
    constexpr int WAVES = WAVES_M * WAVES_N;
    constexpr int WM = BM / WAVES_M, WN = NH / WAVES_N, TM = WM / 32, TH = WN / 32, TN = 2 * TH;
    constexpr int STAGE = BM * 128 + 2 * NH * 16, CODES = 2 * NH / 64;  // 1 KiB copies of codes a stage
    constexpr int PITCH = WN + 4;
    static_assert(CODES >= 1 && CODES <= WAVES && WAVES % CODES == 0, "a copy a wave");
    constexpr int RING = STAGES * STAGE, QUADS = TM * TN * 4;
    static_assert(GROUPS * RING >= WAVES * 2 * 32 * PITCH * 4 + 2 * NH * 4, "staging fits in the ring");
    typedef NtRows<BM, WAVES> Rows;
    constexpr int COPIES = Rows::COPIES + 1;
    static_assert((GROUPS - 1) * QUADS * 16 * 64 * WAVES <= GROUPS * RING, "sums fit in the rings");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[GROUPS * RING];
    const int tid = threadIdx.x, lane = tid & 63;
    const int group = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(tid / (64 * WAVES)) : 0;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) - group * WAVES;
    const int wm = wave / WAVES_N, wn = wave % WAVES_N, half = lane >> 5, l32 = lane & 31;
    const uint32_t tiles_n = (uint32_t)((a.f + NH - 1) / NH), tiles_m = (uint32_t)((a.rows + BM - 1) / BM);
    uint32_t tm, tn;
    nt_tile((uint32_t)xcd_remap(blockIdx.x, gridDim.x), tiles_m, tiles_n, &tm, &tn);
    const int64_t m0 = (int64_t)tm * BM;
    const int32_t k0 = (int32_t)(tn * NH);

    const int seg = (lane & 7) ^ ((4 * (wave & 1)) | ((lane >> 4) & 3));
    const uint32_t row_bytes = (uint32_t)a.c * 2;
    Rows rows;
    rows.init(a.x, m0, a.rows, row_bytes, wave, lane, seg);
    const int nb = (a.c + 63) / 64;  // stages, and blocks of codes of a filter
    const int each = (nb + GROUPS - 1) / GROUPS, first = min(group * each, nb), n = min(each, nb - first);  // of this group
    // this lane's filter of the gates, then the others (past the last filter: other codes or none, never stored)
    const int piece = wave % CODES, of = 64 * piece + lane;
    const int32_t filter = k0 + (of < NH ? of : a.f + of - NH);
    const v4i rsrc_c = make_rsrc(a.codes, (uint32_t)((int64_t)((2 * a.f + 63) / 64) * nb * 1024));
    const uint32_t code_off = (uint32_t)((int64_t)(filter / 64) * nb * 1024 + (filter % 64) * 16);
    uint8_t* const ring = smem + group * RING;
    const uint32_t base = lds_addr(ring);
    int islot = 0;
    auto issue = [&](int s, int j0, int j1) {
        const uint32_t lds = base + (uint32_t)(islot * STAGE);
        const uint32_t kb = (uint32_t)(first + s) * 128u;
        const uint32_t at = kb + 16u * seg < row_bytes ? kb : kb | 0x80000000u;
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
            if (j < j0 || j >= j1) continue;
            if (j < Rows::COPIES)
                rows.issue(j, lds, at, wave);
            else
                dma_b128(rsrc_c, lds + BM * 128 + piece * 1024, code_off + (uint32_t)(first + s) * 1024u);
        }
        if (j1 == COPIES) islot = islot + 1 == STAGES ? 0 : islot + 1;
    };

    const int sw = (l32 >> 1) & 7;
    const int arow = (wm * WM + l32) * 128, bcol = BM * 128 + (wn * WN + l32) * 16;
    uint32_t mask[4], shl[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        mask[j] = 0x01010101u << (4 * half + j);
        shl[j] = 7 - 4 * half - j;
    }
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][t][v] = 0.0f;

#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if (s < n) issue(s, 0, COPIES);
    int cslot = 0;
    for (int s = 0; s < each; ++s) {
        if (s + STAGES - 2 < n)
            wait_vmcnt((STAGES - 2) * COPIES);
        else
            wait_vmcnt(0);
        __syncthreads();
        if (s + STAGES - 1 < n) issue(s + STAGES - 1, 0, COPIES);
        if (GROUPS > 1 && s >= n) continue;
        const uint8_t* st = ring + cslot * STAGE;
        cslot = cslot + 1 == STAGES ? 0 : cslot + 1;
        u32x4 raw[TN];
#pragma unroll
        for (int t = 0; t < TN; ++t)
            raw[t] = *reinterpret_cast<const u32x4*>(st + bcol + ((t < TH ? 0 : NH) + 32 * (t % TH)) * 16);
        u32x4 x[2][TM];
        bf16x8 w[2][TN];
        auto read = [&](int u, int k) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
                x[k][i] = *reinterpret_cast<const u32x4*>(st + arow + 32 * 128 * i + 16 * ((2 * u + half) ^ sw));
        };
        auto decode = [&](int u, int k) {
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                u32x4 d;
#pragma unroll
                for (int j = 0; j < 4; ++j) d[j] = ((raw[t][u] & mask[j]) << shl[j]) + 0x3F803F80u;
                w[k][t] = as_bf16x8(d);
            }
        };
        read(0, 0);
        decode(0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u + 1 < 4) {
                read(u + 1, (u + 1) & 1);
                decode(u + 1, (u + 1) & 1);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int t = 0; t < TN; ++t) acc[i][t] = mfma32(w[u & 1][t], as_bf16x8(x[u & 1][i]), acc[i][t]);
            if (u + 1 < 4) {
#pragma unroll
                for (int k = 0; k < TM * TN; ++k) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (k < TM) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, TM >= 4 ? 2 : 8 / TM, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // ---- lane l of tile (i, t) holds row 32 i + l % 32 and, for each v / 4, columns 32 t + 8 (v / 4) + 4 (l / 32) + 0..3;
    //      32 rows of g and u at a time are turned in LDS, so that a lane has 8 columns of a row ----
    __syncthreads();
    if constexpr (GROUPS > 1) {
        f32x4* const at = reinterpret_cast<f32x4*>(smem) + wave * 64 + lane;
        if (group) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int t = 0; t < TN; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        at[((group - 1) * QUADS + (i * TN + t) * 4 + g) * WAVES * 64] =
                            f32x4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
        }
        __syncthreads();
        if (!group) {
#pragma unroll
            for (int k = 0; k < GROUPS - 1; ++k)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int t = 0; t < TN; ++t)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const f32x4 v = at[(k * QUADS + (i * TN + t) * 4 + g) * WAVES * 64];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][t][4 * g + e] += v[e];
                        }
        }
        __syncthreads();
    }
    float* alpha = reinterpret_cast<float*>(smem + WAVES * 2 * 32 * PITCH * 4);  // of the gates, then of the others
    for (int i = tid; i < 2 * NH; i += 64 * WAVES * GROUPS) {
        const int32_t k = k0 + i % NH;
        alpha[i] = k < a.f ? a.alpha[(i < NH ? 0 : a.f) + k] : 0.0f;
    }
    __syncthreads();
    if (group) return;
    float* sg = reinterpret_cast<float*>(smem) + wave * 2 * 32 * PITCH;
    float* su = sg + 32 * PITCH;
    constexpr int CG = WN / 8, RPP = 64 / CG;
    const int cl = 8 * (lane % CG);
    const int32_t k = k0 + wn * WN + cl;
    const bool whole = a.f % 8 == 0;
    float ag[8], au[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) ag[e] = alpha[wn * WN + cl + e], au[e] = alpha[NH + wn * WN + cl + e];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int t = 0; t < TH; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int o = l32 * PITCH + 32 * t + 8 * g + 4 * half;
                *reinterpret_cast<f32x4*>(sg + o) = f32x4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
                *reinterpret_cast<f32x4*>(su + o) =
                    f32x4{acc[i][t + TH][4 * g], acc[i][t + TH][4 * g + 1], acc[i][t + TH][4 * g + 2], acc[i][t + TH][4 * g + 3]};
            }
        __builtin_amdgcn_wave_barrier();
        if (!whole) {  // rows begin anywhere: a value a lane, side by side
            constexpr int ROWS = 64 / WN;
            const int c = lane % WN;
            const float a1 = alpha[wn * WN + c], a2 = alpha[NH + wn * WN + c];
#pragma unroll 1
            for (int r = lane / WN; r < 32; r += ROWS) {
                const int64_t m = m0 + wm * WM + 32 * i + r;
                if (m < a.rows && k0 + wn * WN + c < a.f) finish1<ACT>(a, m, k0 + wn * WN + c, sg[r * PITCH + c] * a1, su[r * PITCH + c] * a2);
            }
            __builtin_amdgcn_wave_barrier();
            continue;
        }
#pragma unroll 1
        for (int p = 0; p < 32 / RPP; ++p) {
            const int r = p * RPP + lane / CG;
            const int64_t m = m0 + wm * WM + 32 * i + r;
            float g[8], u[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 vg = *reinterpret_cast<const f32x4*>(sg + r * PITCH + cl + 4 * h), vu = *reinterpret_cast<const f32x4*>(su + r * PITCH + cl + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) g[4 * h + e] = vg[e] * ag[4 * h + e], u[4 * h + e] = vu[e] * au[4 * h + e];
            }
            if (m < a.rows && k < a.f) finish8<ACT>(a, m, k, 8, true, g, u);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- up to 16 rows -----------------------------------------------------------------------
// The codes are read once and bound it.  A block owns 16 NG gates and the others of the same columns; its waves divide the
// features.  Lane (f = l % 16, q = l / 16) reads, of filter f of each group, the 16 bytes of element block ib + q and, of row f
// of x, the same 64 features; matrix instruction s of a step takes elements 8 s .. 8 s + 7 of each block (the order of the
// elements is the same in both operands, which is all that a sum asks).  The waves' sums meet in LDS.
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Elements 8 h .. 8 h + 7 of a packed word as bf16 pairs, two operations a pair.
template <int H>
__device__ __forceinline__ bf16x8 decode_half(uint32_t w) {
    u32x4 d;
#pragma unroll
    for (int j = 0; j < 4; ++j) d[j] = ((w & (0x01010101u << (4 * H + j))) << (7 - 4 * H - j)) + 0x3F803F80u;
    return as_bf16x8(d);
}

template <int NG, int WAVES, int DEPTH, bool STAGED, int ACT>
__global__ __launch_bounds__(64 * WAVES) void glu_few_kernel(const GluArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint16_t xl[];  // STAGED: [rows + 1][steps 256], the last row zero
    __shared__ f32x4 sums[WAVES][2 * NG][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int f = lane & 15, q = lane >> 4;
    const int32_t k0 = (int32_t)blockIdx.x * 16 * NG;
    const int nb = (a.c + 63) / 64;     // element blocks
    const int steps = (nb + 3) / 4;     // four a step, one a lane group
    const int s0 = (int)((int64_t)steps * wave / WAVES), s1 = (int)((int64_t)steps * (wave + 1) / WAVES);
    const u32x4* wp[2 * NG];
#pragma unroll
    for (int g = 0; g < 2 * NG; ++g) {
        const int32_t k = min(k0 + 16 * (g % NG) + f, a.f - 1) + (g < NG ? 0 : a.f);
        wp[g] = reinterpret_cast<const u32x4*>(a.codes) + (int64_t)(k / 64) * nb * 64 + k % 64;
    }
    const bool have = f < a.rows;
    const uint16_t* xp = a.x + (int64_t)(have ? f : 0) * a.c;
    f32x4 acc[2 * NG];
#pragma unroll
    for (int g = 0; g < 2 * NG; ++g) acc[g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    u32x4 w[DEPTH][2 * NG], x[STAGED ? 1 : DEPTH][8];
    const uint16_t* const xs = xl + (have ? f : (int)a.rows) * steps * 256;
    auto load = [&](int d, int s) {
        const int ib = 4 * s + q;
        if constexpr (!STAGED) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = ib * 64 + 8 * e;
                x[d][e] = u32x4{0u, 0u, 0u, 0u};
                if (have && c < a.c) x[d][e] = *reinterpret_cast<const u32x4*>(xp + c);
            }
        }
#pragma unroll
        for (int g = 0; g < 2 * NG; ++g) w[d][g] = __builtin_nontemporal_load(wp[g] + (int64_t)(ib < nb ? ib : nb - 1) * 64);
    };
    auto multiply = [&](int d, int s) {
        if constexpr (STAGED) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[0][e] = *reinterpret_cast<const u32x4*>(xs + (4 * s + q) * 64 + 8 * e);
        }
        const int dx = STAGED ? 0 : d;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int g = 0; g < 2 * NG; ++g) {
                acc[g] = mfma16(decode_half<0>(w[d][g][e]), as_bf16x8(x[dx][2 * e]), acc[g]);
                acc[g] = mfma16(decode_half<1>(w[d][g][e]), as_bf16x8(x[dx][2 * e + 1]), acc[g]);
            }
    };
    if constexpr (STAGED) {
        // the first loads of x before those of the codes: writing them to LDS waits for them alone
        const int per = steps * 32, pieces = ((int)a.rows + 1) * per;  // 16-byte pieces of a row, and all
        u32x4 v[4];
        auto get = [&](int i0) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + 64 * WAVES * u, r = i / per, c = (i - r * per) * 8;
                v[u] = u32x4{0u, 0u, 0u, 0u};
                if (i < pieces && r < a.rows && c < a.c) v[u] = *reinterpret_cast<const u32x4*>(a.x + (int64_t)r * a.c + c);
            }
        };
        auto put = [&](int i0) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i0 + 64 * WAVES * u < pieces) reinterpret_cast<u32x4*>(xl)[i0 + 64 * WAVES * u] = v[u];
        };
        get(threadIdx.x);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (s0 + d < s1) load(d, s0 + d);
        put(threadIdx.x);
        for (int i0 = threadIdx.x + 64 * WAVES * 4; i0 < pieces; i0 += 64 * WAVES * 4) {
            get(i0);
            put(i0);
        }
        __syncthreads();
    } else {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (s0 + d < s1) load(d, s0 + d);
    }
    for (int s = s0; s < s1; s += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (s + d >= s1) break;
            multiply(d, s + d);
            if (s + d + DEPTH < s1) load(d, s + d + DEPTH);
        }
    }
#pragma unroll
    for (int g = 0; g < 2 * NG; ++g) sums[wave][g][lane] = acc[g];
    __syncthreads();
    // lane (f, q) holds row f, columns 4 q .. 4 q + 3 of each 16
    for (int i = wave; i < NG; i += WAVES) {
        f32x4 g = sums[0][i][lane], u = sums[0][NG + i][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) {
            g += sums[v][i][lane];
            u += sums[v][NG + i][lane];
        }
        const int32_t k = k0 + 16 * i + 4 * q;
        if (!have || k >= a.f) continue;
        float g8[8] = {0, 0, 0, 0, 0, 0, 0, 0}, u8[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const int n = a.f - k < 4 ? a.f - k : 4;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) g8[e] = g[e] * a.alpha[k + e], u8[e] = u[e] * a.alpha[a.f + k + e];
        finish8<ACT>(a, f, k, n, false, g8, u8);
    }
}

// ---- from kept projections ---------------------------------------------------------------
template <int ACT>
__global__ __launch_bounds__(256) void glu_bwd_kernel(const GluArgs a, const uint16_t* __restrict__ gu, uint32_t groups) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = i / groups;
    if (m >= a.rows) return;
    const int32_t k = (int32_t)(i - m * groups) * 8;
    const int n = a.f - k < 8 ? a.f - k : 8;
    const bool whole = a.f % 8 == 0;
    float g[8], u[8];
    get8(gu, m * 2 * a.f + k, n, whole, g);
    get8(gu, m * 2 * a.f + a.f + k, n, whole, u);
    finish8<ACT>(a, m, k, n, whole, g, u);
}

template <int BM, int NH, int WM, int WN, int STAGES, int GROUPS, int ACT>
hipError_t launch_tiles(const GluArgs& a, hipStream_t s) {
    const int64_t blocks = (a.rows + BM - 1) / BM * ((a.f + NH - 1) / NH);
    hipLaunchKernelGGL((glu_kernel<BM, NH, WM, WN, STAGES, GROUPS, ACT>), dim3((unsigned)blocks), dim3(64 * WM * WN * GROUPS), 0, s, a);
    return hipGetLastError();
}

template <int ACT>
hipError_t launch(const GluArgs& a, const uint16_t* gu, hipStream_t s) {
    if (gu) {
        const uint32_t groups = (uint32_t)(a.f + 7) / 8;
        hipLaunchKernelGGL((glu_bwd_kernel<ACT>), dim3((unsigned)((a.rows * groups + 255) / 256)), dim3(256), 0, s, a, gu, groups);
        return hipGetLastError();
    }
    if (a.rows <= 16) {
        const int64_t groups = (a.f + 15) / 16;
        const int lds = ((int)a.rows + 1) * ((a.c + 255) / 256) * 512;  // of x and a row of zeros
#define TBN_FEW(ng, waves, depth, staged)                                                                                           \
    hipLaunchKernelGGL((glu_few_kernel<ng, waves, depth, staged, ACT>), dim3((unsigned)((groups + ng - 1) / ng)), dim3(64 * waves), \
                       staged ? lds : 0, s, a)
        if (a.rows <= 4 && lds <= 48 * 1024) {
            if (groups >= 1024)
                TBN_FEW(2, 8, 2, true);
            else
                TBN_FEW(1, 4, 2, true);
        } else if (groups >= 1024) {
            TBN_FEW(4, 8, 1, false);
        } else if (groups >= 512) {
            TBN_FEW(2, 4, 2, false);
        } else {
            TBN_FEW(1, 4, 2, false);
        }
#undef TBN_FEW
        return hipGetLastError();
    }
    auto tiles = [&](int64_t m, int64_t n) { return (a.rows + m - 1) / m * ((a.f + n - 1) / n); };
    if (tiles(256, 128) >= 192) return launch_tiles<256, 128, 2, 4, 4, 1, ACT>(a, s);
    if (tiles(128, 128) >= 192) return launch_tiles<128, 128, 2, 4, 4, 1, ACT>(a, s);
    if (tiles(128, 64) >= 192) return launch_tiles<128, 64, 2, 2, 4, 1, ACT>(a, s);
    if (tiles(64, 64) > 256 || a.c <= 1024) return launch_tiles<64, 64, 2, 2, 4, 1, ACT>(a, s);
    if (tiles(64, 64) > 128) return launch_tiles<64, 64, 2, 2, 4, 4, ACT>(a, s);
    return launch_tiles<64, 32, 2, 1, 4, 4, ACT>(a, s);
}

}  // namespace

hipError_t launch_glu(const GluArgs& a, const uint16_t* gu, int act, hipStream_t s) {
    if (act == TBN_ACT_SILU) return launch<TBN_ACT_SILU>(a, gu, s);
    if (act == TBN_ACT_GELU) return launch<TBN_ACT_GELU>(a, gu, s);
    return launch<TBN_ACT_RELU>(a, gu, s);
}

}  // namespace tbn
