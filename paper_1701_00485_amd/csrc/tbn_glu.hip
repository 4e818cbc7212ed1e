// tbn_glu.hip -- the gated block of two-bit filters: f gates and f others over the same c features,
//   g = alpha_g (x W~_g),  u = alpha_u (x W~_u),  h = act(g) u,
// both projections, the activation and the product in one kernel; and the gradient dg = dh u act'(g), du = dh act(g), from
// the g and u that the forward pass kept or, with the same products again, from x.
//
// The codes of the 2 f filters are packed as those of one layer, gates first (TBN2, see tbn.h).
#include <algorithm>
#include <type_traits>

#include "tbn_kernels.h"
#include "tbn_nt.h"

namespace tbn {

namespace {

// ---- activations, in fp32 ----------------------------------------------------------------
// act(g) and, for the backward pass, its derivative.
//   silu  g s, s = 1 / (1 + e^-g);            s (1 + g (1 - s))
//   gelu  g phi, phi = (1 + erf(g / sqrt 2)) / 2;   phi + g e^(-g^2 / 2) / sqrt(2 pi)
//   relu  max(g, 0);                          1 where g > 0, else 0
// silu's exponential is the hardware's 2^t of t = -|g| log2 e rounded, times 1 + (-|g| - t ln 2), what the rounding left (else e^-80 is off
// by 30 steps of fp32; now every silu of a bf16 gate by at most 1.9e-7 of itself).  Of -|g| it never overflows, and 1 - s is a quotient too, not
// a difference.  8192 x 4096 -> 2 x 8192: 826 us, with 2^(-g log2 e) alone 816; 777 x 1000 -> 2 x 1333 13.4 and 12.8.
// gelu's Phi(-|g|) is e^(-g^2 / 2), made the same way, times r P(r), r = 1 / (1 + 0.35 |g|): P is of degree 8, fitted to
// erfcx(|g| / sqrt 2) / 2 over |g| <= 13.5, where the exponential leaves fp32, to 3.2e-8 of itself: every gelu of a bf16 gate within
// 3.4e-7.  From 1 + erff it has no digit left at g = -5.6, and 777 x 1000 -> 2 x 1333 takes 15.4 us in place of 14.2; by erfcf 17.1.
template <bool SLOPE>
__device__ __forceinline__ float activate(int act, float g, float* slope) {
    if (act == TBN_ACT_SILU) {
        const float a = fminf(fabsf(g), 128.0f);  // (e^-128 is 0 here; of NaN anything, which g carries on)
        const float t = -1.44269504f * a, e = __builtin_amdgcn_exp2f(t);
        const float p = fmaf(e, fmaf(1.90465421e-9f, t, fmaf(-0.69314718f, t, -a)), e);  // e^-|g|; ln 2 in two parts
        const float y = __builtin_amdgcn_rcpf(1.0f + p), q = p * y;
        const float s = g < 0.0f ? q : y;
        if (SLOPE) *slope = s * (1.0f + g * (g < 0.0f ? y : q));
        return g * s;
    }
    if (act == TBN_ACT_GELU) {
        const float a = fminf(fabsf(g), 16.0f);  // (e^-128 is 0 here; of NaN anything, which g carries on)
        const float w = a * a, t = -0.72134752f * w, e = __builtin_amdgcn_exp2f(t);
        float rest = fmaf(1.90465421e-9f, t, fmaf(-0.69314718f, t, -0.5f * w));
        rest = fmaf(-0.5f, fmaf(a, a, -w), rest);
        const float p = fmaf(e, rest, e);  // e^(-g^2 / 2)
        const float r = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
        float poly = -0.0291259624f;
        for (float c : {0.143872693f, -0.255505502f, 0.158930317f, -0.0229377989f, 0.105433196f, 0.119852379f, 0.13985908f, 0.139621571f})
            poly = fmaf(poly, r, c);
        const float below = p * (r * poly);  // Phi(-|g|)
        const float phi = g < 0.0f ? below : 1.0f - below;
        if (SLOPE) *slope = phi + g * p * 0.39894228f;
        return g * phi;
    }
    if (SLOPE) *slope = g > 0.0f ? 1.0f : (g != g ? g : 0.0f);
    return g > 0.0f || g != g ? g : 0.0f;
}

__device__ __forceinline__ void unpack8(u32x4 r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = bf16_bits_to_f32(r[e] & 0xFFFFu), v[2 * e + 1] = __uint_as_float(r[e] & 0xFFFF0000u);
}

// Eight values of a row whose first has index `at`: 16-byte aligned, anywhere, or `n` of them.
enum Eight { EVEN, WHOLE, PART };
template <Eight E>
__device__ __forceinline__ void get8(const uint16_t* p, int64_t at, int n, float (&v)[8]) {
    if constexpr (E == PART) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? bf16_bits_to_f32(p[at + e]) : 0.0f;
    } else {
        typedef typename std::conditional<E == EVEN, u32x4, u32x4_at2>::type V;
        unpack8(*reinterpret_cast<const V*>(p + at), v);
    }
}
template <Eight E>
__device__ __forceinline__ void put8(uint16_t* p, int64_t at, int n, const float (&v)[8]) {
    if constexpr (E == PART) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[at + e] = (uint16_t)f32_to_bf16_bits(v[e]);
    } else {
        typedef typename std::conditional<E == EVEN, u32x4, u32x4_at2>::type V;
        *reinterpret_cast<V*>(p + at) =
            u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
}
template <Eight E>
__device__ __forceinline__ void put8(float* p, int64_t at, int n, const float (&v)[8]) {
    if constexpr (E == PART) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[at + e] = v[e];
    } else {
        typedef typename std::conditional<E == EVEN, f32x4, f32x4_at4>::type V;
        reinterpret_cast<V*>(p + at)[0] = f32x4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<V*>(p + at)[1] = f32x4{v[4], v[5], v[6], v[7]};
    }
}

// What follows g and u of columns k .. k + 7 of row m (n of them real): h, the kept projections or the gradients.
template <int ACT, Eight E>
__device__ __forceinline__ void finish8(const GluArgs& a, int64_t m, int32_t k, int n, const float (&g)[8], const float (&u)[8]) {
    const int64_t o = m * a.f + k, og = m * 2 * a.f + k;
    float h[8];
    if (a.dh) {
        float dh[8], dg[8], du[8];
        get8<E>(a.dh, o, n, dh);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float slope;
            const float y = activate<true>(ACT, g[e], &slope);
            dg[e] = dh[e] * u[e] * slope;
            du[e] = dh[e] * y;
            h[e] = y * u[e];
        }
        put8<E>(a.gu, og, n, dg);
        put8<E>(a.gu, og + a.f, n, du);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = activate<false>(ACT, g[e], nullptr) * u[e];
        if (a.gu) {
            put8<E>(a.gu, og, n, g);
            put8<E>(a.gu, og + a.f, n, u);
        }
    }
    if (!a.h) return;
    if (a.h_f32)
        put8<E>(reinterpret_cast<float*>(a.h), o, n, h);
    else
        put8<E>(reinterpret_cast<uint16_t*>(a.h), o, n, h);
}

// ... whichever way the rows lie.
template <int ACT>
__device__ __forceinline__ void finish8(const GluArgs& a, int64_t m, int32_t k, int n, const float (&g)[8], const float (&u)[8]) {
    if (a.f % 8 == 0)
        finish8<ACT, EVEN>(a, m, k, n, g, u);
    else if (n == 8)
        finish8<ACT, WHOLE>(a, m, k, n, g, u);
    else
        finish8<ACT, PART>(a, m, k, n, g, u);
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
// stage's codes, 16 bytes each, decoded in registers into bf16 pairs, two operations a pair, between the matrix instructions that
// bound it: 8192 x 4096 -> 2 x 8192 in 784 to 828 us, 1.33 to 1.40 PFLOP/s (copies issued at a stage's begin and operands made in a row: 857 of then 800).
// Two blocks of 128 x 128 a compute unit, each with a barrier a stage, do as well as one of 256 x 128.
// GROUPS groups of such waves, each with a part of the stages and a ring of its own, serve tiles that are too few to fill the GPU; the
// first adds the others' sums.
template <int BM, int NH, int WAVES_M, int WAVES_N, int STAGES, int GROUPS, int ACT>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N * GROUPS, GROUPS > 1 ? 1 : 2) void glu_kernel(const GluArgs a) {
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
    uint32_t copy_lds = 0, copy_x = 0, copy_codes = 0;  // of the stage whose copies are issued (past the last one: zeros, as in tbn_nt.h)
    auto aim = [&](int s) {
        const uint32_t past = s < n ? 0u : 0x80000000u, at = (uint32_t)(first + s) * 128u;
        copy_lds = base + (uint32_t)(islot * STAGE);
        copy_x = at + 16u * seg < row_bytes ? at | past : at | 0x80000000u;
        copy_codes = code_off + (uint32_t)(first + s) * 1024u | past;
        islot = islot + 1 == STAGES ? 0 : islot + 1;
    };
    auto copy = [&](int j) {
        if (j < Rows::COPIES)
            rows.issue(j, copy_lds, copy_x, wave);
        else
            dma_b128(rsrc_c, copy_lds + BM * 128 + piece * 1024, copy_codes);
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

    auto pin = [&]() {  // as in tbn_nt.h
        if constexpr (TM * TN >= 16) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int t = 0; t < TN; ++t) asm volatile("" : "+a"(acc[i][t]));
        }
    };
    u32x4 raw[TN], x[2][TM], w[2][TN];
    auto codes = [&](const uint8_t* st, int t) { raw[t] = *reinterpret_cast<const u32x4*>(st + bcol + ((t < TH ? 0 : NH) + 32 * (t % TH)) * 16); };
    auto read = [&](const uint8_t* st, int u, int i) {
        x[u & 1][i] = *reinterpret_cast<const u32x4*>(st + arow + 32 * 128 * i + 16 * ((2 * u + half) ^ sw));
    };
    auto decode = [&](int u, int d) {  // word d of the filters' operands of step u
        const int t = d / 4, j = d % 4;
        w[u & 1][t][j] = ((raw[t][u] & mask[j]) << shl[j]) + 0x3F803F80u;
    };
    // Step u of a stage, while the operands of step v of the stage at `st` are made: the next step of the same stage, or, in a
    // stage's last step, the first one of the next, whose codes are read first; then copies are issued too.
    constexpr int MUL = TM * TN, WORDS = 4 * TN, LAST = 3;
    auto step = [&](int u, const uint8_t* st, int v, bool last) {
        constexpr bool MANY = MUL >= 8;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!MANY) {
            if (last) {
#pragma unroll
                for (int t = 0; t < TN; ++t) codes(st, t);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) read(st, v, i);
            if (!last) {
#pragma unroll
                for (int d = 0; d < WORDS; ++d) decode(v, d);
            }
        }
#pragma unroll
        for (int k = 0; k < MUL; ++k) {
            const int i = k / TN, t = k % TN;
            acc[i][t] = mfma32(as_bf16x8(w[u & 1][t]), as_bf16x8(x[u & 1][i]), acc[i][t]);
            if constexpr (MANY) {
                if (last) {
#pragma unroll
                    for (int c = 2 * k * TN / MUL; c < 2 * (k + 1) * TN / MUL && c < TN; ++c) codes(st, c);
                }
#pragma unroll
                for (int r = k * TM / MUL; r < (k + 1) * TM / MUL; ++r) read(st, v, r);
                if (last) {
#pragma unroll
                    for (int d = (2 * k - MUL) * WORDS / MUL; d < (2 * k + 2 - MUL) * WORDS / MUL; ++d)
                        if (d >= 0) decode(v, d);
#pragma unroll
                    for (int j = k * COPIES / MUL; j < (k + 1) * COPIES / MUL; ++j) copy(j);
                } else {
#pragma unroll
                    for (int d = k * WORDS / MUL; d < (k + 1) * WORDS / MUL; ++d) decode(v, d);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (!MANY) {
            if (last) {
#pragma unroll
                for (int j = 0; j < COPIES; ++j) copy(j);
#pragma unroll
                for (int d = 0; d < WORDS; ++d) decode(v, d);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };

#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
        aim(s);
#pragma unroll
        for (int j = 0; j < COPIES; ++j) copy(j);
    }
    wait_vmcnt((STAGES - 1) * COPIES);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TN; ++t) codes(ring, t);
#pragma unroll
    for (int i = 0; i < TM; ++i) read(ring, 0, i);
#pragma unroll
    for (int d = 0; d < WORDS; ++d) decode(0, d);
    pin();
    int slot = 0;
    for (int s = 0; s < each; ++s) {
        const uint8_t* st = ring + slot * STAGE;
        slot = slot + 1 == STAGES ? 0 : slot + 1;
        if (GROUPS == 1 || s < n) {
#pragma unroll
            for (int u = 0; u < LAST; ++u) step(u, st, u + 1, false);
        }
        // this wave's copies of the next stage have landed, its reads of this one are done, and so are the other waves'
        wait_vmcnt((STAGES - 2) * COPIES);
        __syncthreads();
        if (GROUPS > 1 && s >= n) continue;
        aim(s + STAGES);  // into this stage's place
        step(LAST, ring + slot * STAGE, 0, true);
    }
    pin();
    wait_vmcnt(0);

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
    const int n8 = a.f - k < 8 ? a.f - k : 8;
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
            if (m < a.rows && n8 > 0) finish8<ACT>(a, m, k, n8, g, u);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- up to 16 rows -----------------------------------------------------------------------
// The codes are read once, 59 MB of 4096 -> 2 x 28672 in 18.4 us for 1 row (3.2 TB/s), in 21.4 us for 16; their reading and their
// decoding bound it together, two vector operations a pair (not decoded, 16 rows take 15.6 us; with x of one row read alone 21.1).  Lane
// (f = l % 16, q = l / 16) reads, of filter f of 16, the 16 bytes of element block ib + q and, of row f of x, the same 64
// features; matrix instruction s of a step takes elements 8 s .. 8 s + 7 of each block (the order of the elements is the
// same in both operands, which is all that a sum asks).
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Elements 8 h .. 8 h + 7 of a packed word as bf16 pairs, two operations a pair.
template <int H>
__device__ __forceinline__ bf16x8 decode_half(uint32_t w) {
    u32x4 d;
#pragma unroll
    for (int j = 0; j < 4; ++j) d[j] = ((w & (0x01010101u << (4 * H + j))) << (7 - 4 * H - j)) + 0x3F803F80u;
    return as_bf16x8(d);
}

// Of up to 4096 SL features: a block, one a compute unit, owns a range of the groups of 16 gates and the others of the same columns.
// Wave (i, j) of its KS x GS keeps x's steps i, i + KS, .. of 256 features in registers and streams the codes of groups j, j + GS, ..,
// four (SL 2: two) ahead; the KS sums of an output meet in LDS, four groups a wave at a time.  Without x in registers, a block for
// each 64 gates or 16 (glu_few_kernel): 26.5 us for 16 rows of 4096 -> 2 x 28672, and 3.9 for 1 x 512 -> 2 x 1024, 3.5 here.
template <int SL, int ACT>
__global__ __launch_bounds__(1024) void glu_stream_kernel(const GluArgs a, int KS, int GS) {
    constexpr int BATCH = 4, AHEAD = SL == 1 ? 4 : 2;
    __shared__ __attribute__((aligned(16))) float part[BATCH * 16 * 512];  // [BATCH GS groups][KS][gates, others][16 rows][16 columns]
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = wave / KS, i = wave - j * KS;
    const int f = lane & 15, q = lane >> 4;
    const int nb = (a.c + 63) / 64;  // element blocks, four a step, one a lane group
    const int groups = (a.f + 15) / 16;
    const int g0 = (int)((int64_t)groups * blockIdx.x / gridDim.x), g1 = (int)((int64_t)groups * (blockIdx.x + 1) / gridDim.x);
    const int rounds = (g1 - g0 + GS - 1) / GS;
    const u32x4* const codes = reinterpret_cast<const u32x4*>(a.codes);
    int ib[SL];
#pragma unroll
    for (int s = 0; s < SL; ++s) ib[s] = 4 * (i + KS * s) + q;
    u32x4 w[AHEAD][SL][2], x[SL][8];
    auto load = [&](int d, int r) {
        const int k = min((g0 + j + GS * r) * 16 + f, a.f - 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int filter = k + (h ? a.f : 0);
            const u32x4* const p = codes + (int64_t)(filter / 64) * nb * 64 + filter % 64;
#pragma unroll
            for (int s = 0; s < SL; ++s) w[d][s][h] = __builtin_nontemporal_load(p + (int64_t)min(ib[s], nb - 1) * 64);
        }
    };
    // A step's 512 bytes of each row, two rows a load, are turned in this wave's 8 KiB of LDS.  Read as the matrix instruction wants
    // them, 16 bytes of a line by each lane, 16 rows fetch each line eight times (16 x 4096 -> 2 x 8192: 14.1 us, 10.1 turned);
    // up to 4 rows stay in the cache, and turning them costs 0.5 to 2 us.
    uint8_t* const turn = reinterpret_cast<uint8_t*>(part) + wave * 8192;
    auto ahead = [&]() {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d)
            if (d < rounds) load(d, d);
    };
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(a.x), 0, (int)(a.rows * a.c * 2), 0x00020000);
    auto get = [&](int row, int c) {  // zeros past the row's end and past the last row
        return __builtin_amdgcn_raw_buffer_load_b128(rx, c < a.c ? (row * a.c + c) * 2 : (int)0x80000000, 0, 0);
    };
    if (a.rows <= 4) {
#pragma unroll
        for (int s = 0; s < SL; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[s][e] = get(f, ib[s] * 64 + 8 * e);
        ahead();
    } else {
        u32x4 v[SL][8];
#pragma unroll
        for (int s = 0; s < SL; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[s][e] = get(2 * e + (lane >> 5), (i + KS * s) * 256 + 8 * (lane & 31));
        ahead();
#pragma unroll
        for (int s = 0; s < SL; ++s) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = 2 * e + (lane >> 5);
                *reinterpret_cast<u32x4*>(turn + row * 512 + 16 * ((lane & 31) ^ row)) = v[s][e];
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < 8; ++e) x[s][e] = *reinterpret_cast<const u32x4*>(turn + f * 512 + 16 * ((8 * q + e) ^ f));
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
    }
    for (int r0 = 0; r0 < rounds; r0 += BATCH) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (r0 + b >= rounds) break;
            f32x4 acc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < SL; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        acc[h] = mfma16(decode_half<0>(w[b % AHEAD][s][h][e]), as_bf16x8(x[s][2 * e]), acc[h]);
                        acc[h] = mfma16(decode_half<1>(w[b % AHEAD][s][h][e]), as_bf16x8(x[s][2 * e + 1]), acc[h]);
                    }
            if (r0 + b + AHEAD < rounds) load(b % AHEAD, r0 + b + AHEAD);
            // lane (f, q) holds row f, columns 4 q .. 4 q + 3
#pragma unroll
            for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(part + (((b * GS + j) * KS + i) * 2 + h) * 256 + f * 16 + 4 * q) = acc[h];
        }
        __syncthreads();
        const int outputs = min(BATCH, rounds - r0) * GS * 256;
        for (int o = threadIdx.x; o < outputs; o += 64 * KS * GS) {
            const int row = o / 16 % 16, k = (g0 + GS * r0 + o / 256) * 16 + o % 16;
            if (row >= a.rows || k >= min(g1 * 16, a.f)) continue;
            const float ag = a.alpha[k], au = a.alpha[a.f + k];
            const float* const v = part + o / 256 * KS * 512 + o % 256;
            float g = v[0], u = v[256];
#pragma unroll 4
            for (int n = 1; n < KS; ++n) g += v[512 * n], u += v[512 * n + 256];
            finish1<ACT>(a, row, k, g * ag, u * au);
        }
        if (r0 + BATCH < rounds) __syncthreads();
    }
}

// Of more features: a block owns 16 NG gates and the others of the same columns, its waves a range of the features each, and x is read
// with the codes.
template <int NG, int WAVES, int DEPTH, int ACT>
__global__ __launch_bounds__(64 * WAVES) void glu_few_kernel(const GluArgs a) {
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
    u32x4 w[DEPTH][2 * NG], x[DEPTH][8];
    auto load = [&](int d, int s) {
        const int ib = 4 * s + q;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = ib * 64 + 8 * e;
            x[d][e] = u32x4{0u, 0u, 0u, 0u};
            if (have && c < a.c) x[d][e] = *reinterpret_cast<const u32x4*>(xp + c);
        }
#pragma unroll
        for (int g = 0; g < 2 * NG; ++g) w[d][g] = __builtin_nontemporal_load(wp[g] + (int64_t)(ib < nb ? ib : nb - 1) * 64);
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (s0 + d < s1) load(d, s0 + d);
    for (int s = s0; s < s1; s += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (s + d >= s1) break;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int g = 0; g < 2 * NG; ++g) {
                    acc[g] = mfma16(decode_half<0>(w[d][g][e]), as_bf16x8(x[d][2 * e]), acc[g]);
                    acc[g] = mfma16(decode_half<1>(w[d][g][e]), as_bf16x8(x[d][2 * e + 1]), acc[g]);
                }
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
        finish8<ACT, PART>(a, f, k, n, g8, u8);
    }
}

// ---- from kept projections ---------------------------------------------------------------
// A thread takes 8 columns of a row: dh, g and u in, dg and du out, 10 bytes an element, which bound it (8192 x 8192: 134 us, 5.0 TB/s).
template <int ACT>
__global__ __launch_bounds__(256) void glu_bwd_kernel(const GluArgs a, const uint16_t* __restrict__ gu, uint32_t groups) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = i / groups;
    if (m >= a.rows) return;
    const int32_t k = (int32_t)(i - m * groups) * 8;
    const int n = a.f - k < 8 ? a.f - k : 8;
    float g[8], u[8];
    if (a.f % 8 == 0) {
        get8<EVEN>(gu, m * 2 * a.f + k, n, g);
        get8<EVEN>(gu, m * 2 * a.f + a.f + k, n, u);
    } else if (n == 8) {
        get8<WHOLE>(gu, m * 2 * a.f + k, n, g);
        get8<WHOLE>(gu, m * 2 * a.f + a.f + k, n, u);
    } else {
        get8<PART>(gu, m * 2 * a.f + k, n, g);
        get8<PART>(gu, m * 2 * a.f + a.f + k, n, u);
    }
    finish8<ACT>(a, m, k, n, g, u);
}

template <int BM, int NH, int WM, int WN, int STAGES, int GROUPS, int ACT>
hipError_t launch_tiles(const GluArgs& a, hipStream_t s) {
    const int64_t blocks = (a.rows + BM - 1) / BM * ((a.f + NH - 1) / NH);
    hipLaunchKernelGGL((glu_kernel<BM, NH, WM, WN, STAGES, GROUPS, ACT>), dim3((unsigned)blocks), dim3(64 * WM * WN * GROUPS), 0, s, a);
    return hipGetLastError();
}

template <int SL, int ACT>
hipError_t launch_stream(const GluArgs& a, hipStream_t s) {
    const int steps = (a.c + 255) / 256, groups = (a.f + 15) / 16;
    const int KS = (steps + SL - 1) / SL, GS = std::max(1, std::min((groups + 255) / 256, 16 / KS));
    hipLaunchKernelGGL((glu_stream_kernel<SL, ACT>), dim3((unsigned)std::min(groups, 256)), dim3(64 * KS * GS), 0, s, a, KS, GS);
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
        if (a.c <= 256 * 16) return launch_stream<1, ACT>(a, s);
        if (a.c <= 256 * 32) return launch_stream<2, ACT>(a, s);
        // 16 x 8192 -> 2 f, NG 1, 2, 4: f 28672 98.8, 66.6, 46.4 us; 14336 55.2, 35.5, 25.2; 8192 29.8, 18.7, 23.6; 4096 16.7, 17.7, 22.8
        const int64_t groups = (a.f + 15) / 16;
#define TBN_FEW(ng, waves, depth) \
    hipLaunchKernelGGL((glu_few_kernel<ng, waves, depth, ACT>), dim3((unsigned)((groups + ng - 1) / ng)), dim3(64 * waves), 0, s, a)
        if (groups >= 768)
            TBN_FEW(4, 8, 1);
        else if (groups >= 512)
            TBN_FEW(2, 4, 2);
        else
            TBN_FEW(1, 4, 2);
#undef TBN_FEW
        return hipGetLastError();
    }
    // The largest tile of which there are enough for the 256 compute units: 160 of 128 x 128 (up to three units in eight are idle), 192 of
    // 128 x 64 (one in four); else 64 x 64, up to 256 of them, one a unit, in groups of waves that divide the stages where these are many, and up to
    // 128 as 64 x 32 so.  Times in us:
    //   rows x c -> 2 x f          128x128  128x64  64x64  64x64 x 4  64x32 x 4
    //   8192 x 4096 -> 2 x 8192      800      936    1051                         (256 x 128 by four or eight waves: 798, 814)
    //    768 x 4096 -> 2 x 4096       51.0     54.2    54.2    63.9      88.8     192 tiles of 128 x 128
    //    640 x 4096 -> 2 x 4096       49.5     52.4    51.3    60.9      74.3     160
    //    512 x 4096 -> 2 x 4096       48.2     34.7    39.9    46.2      61.6     256 tiles of 128 x 64
    //    777 x 1000 -> 2 x 1333       21.6     14.9    14.2    19.7      22.7     147
    //    256 x 4096 -> 2 x 4096       49.0     31.9    25.4    23.4      32.2     256 tiles of 64 x 64
    //    200 x 1536 -> 2 x 4096       23.5     15.4    11.9    12.2      17.7     256
    //     64 x 4096 -> 2 x 8192       47.6     31.3    23.8    20.2      16.5     128
    //     17 x  512 -> 2 x 1024       11.1      8.1     7.1     8.7       6.9      16
    auto tiles = [&](int64_t m, int64_t n) { return (a.rows + m - 1) / m * ((a.f + n - 1) / n); };
    if (tiles(128, 128) >= 160) return launch_tiles<128, 128, 2, 2, 4, 1, ACT>(a, s);
    if (tiles(128, 64) >= 192) return launch_tiles<128, 64, 2, 2, 4, 1, ACT>(a, s);
    if (tiles(64, 64) <= 128 && a.c >= 512) return launch_tiles<64, 32, 2, 1, 4, 4, ACT>(a, s);
    if (tiles(64, 64) <= 256 && a.c >= 2048) return launch_tiles<64, 64, 2, 2, 4, 4, ACT>(a, s);
    return launch_tiles<64, 64, 2, 2, 4, 1, ACT>(a, s);
}

}  // namespace

hipError_t launch_glu(const GluArgs& a, const uint16_t* gu, int act, hipStream_t s) {
    if (act == TBN_ACT_SILU) return launch<TBN_ACT_SILU>(a, gu, s);
    if (act == TBN_ACT_GELU) return launch<TBN_ACT_GELU>(a, gu, s);
    return launch<TBN_ACT_RELU>(a, gu, s);
}

}  // namespace tbn
