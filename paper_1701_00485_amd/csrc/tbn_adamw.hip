// tbn_adamw.hip -- AdamW (decoupled weight decay) over many tensors in one launch, the moments in 32 bits or as
// 8-bit codes.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   w = w - lr decay w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by HBM: 28 bytes a weight with fp32 states and gradients; with 8-bit states 12 (the weight and two codes, read
// and written; the scales are 16 bytes for 256 weights) and the gradient's 2 or 4; all of it read and written once.
// Measured: 268 M weights with fp32 states 1400 us (5.4 TB/s), with 8-bit ones and bf16 gradients 780 us (4.8 TB/s;
// 890 with a round's loads at a time); ResNet-18's 62 tensors, 8 bits, 42 us (4.5 TB/s); 1.7 M weights in 4 tensors 9 us,
// 1000 weights 2.4.  The tensors' pointers are kernel arguments (62 tensors a launch), so that nothing is copied to
// the device and a captured step replays with them; a block takes 1, 2 or 4 rounds of 1024 elements of one tensor, which
// it finds by a look at all tensors' first blocks at once.
//
// 8-bit states: m and r = sqrt(v) are E4M3 codes times a scale, one for every 256 elements of a tensor (the
// largest magnitude / 448); the root, because it has half the range of v in powers of two, so that what is small
// in a block stays above zero (a code spans 2^17.8).  The arithmetic is fp32 throughout; only the stored
// states are rounded, and by chance, up with the probability of the distance: rounded to nearest, a moment that
// moves by 0.1% a step never leaves its code (the steps of a code are 6 to 12%).  The random bits are a hash of
// seed, step, tensor and element, the same on every run.  A wave holds the 256 elements of a scale, 4 a lane.
#include <type_traits>

#include "tbn_device.h"
#include "tbn_kernels.h"

namespace tbn {

namespace {

typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
typedef uint32_t u32_a1 __attribute__((aligned(1)));

// Two rounds of xor-shift and multiplication (by the odd neighbours of 2^32 times the golden section and of the
// fractional part of sqrt 2): every bit of the result depends on every bit of h.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x9E3779B1u;
    h = (h ^ (h >> 15)) * 0x6A09E667u;
    return h ^ (h >> 16);
}

__device__ __forceinline__ float4 load4(const float* p) {
    const f32x4 v = *reinterpret_cast<const f32x4_a4*>(p);
    return float4{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ float4 load4(const uint16_t* p) {
    const u32x2 v = *reinterpret_cast<const u32x2_a2*>(p);
    return float4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                  __uint_as_float(v.y & 0xFFFF0000u)};
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return bf16_bits_to_f32(*p); }

// The update's factors: of the moments, of the decay, of the step and of the root.
struct Factors {
    float b1, a1, b2, a2, decay, rate, root, eps;
};

// b^t by squaring, in fp64 (t >= 1).
__device__ __forceinline__ double power(double b, uint32_t t) {
    double r = 1.0;
    for (; t; t >>= 1) {
        if (t & 1) r *= b;
        b *= b;
    }
    return r;
}

// Every product and sum of the moments is rounded by itself, as elementary operations do: the codes that 8-bit states
// are rounded to are then the same in any IEEE arithmetic (a fused multiply-add moves one in a million across its
// rounding border, and the largest of a block with its scale).
__device__ __forceinline__ void update(float& w, float& m, float& v, float& r, float g, const Factors& f) {
#pragma clang fp contract(off)
    m = f.b1 * m + f.a1 * g;
    v = f.b2 * v + f.a2 * (g * g);
    r = sqrtf(v);
    w = __builtin_fmaf(-f.decay, w, w) - f.rate * m / __builtin_fmaf(r, f.root, f.eps);
}

// x as the fp32 value of an E4M3 code, |x| <= 448 but for rounding: up with the probability rnd / 2^20 of the rest
// below the 3 fraction bits.  Below 2^-6 the codes keep the steps 2^-9 of the smallest normal ones: there
// 2^-6 is added first, which puts these steps where the cut is.  Not finite: NaN.
__device__ __forceinline__ float random_e4m3(float x, uint32_t rnd) {
#pragma clang fp contract(off)
    float a = __builtin_fabsf(x);
    const bool finite = a < __builtin_inff();
    const float low = a < 0x1p-6f ? 0x1p-6f : 0.0f;
    a = __uint_as_float((__float_as_uint(a + low) + rnd) & 0xFFF00000u) - low;
    a = fminf(a, 448.0f);
    return finite ? __builtin_copysignf(a, x) : __builtin_nanf("");
}

__device__ __forceinline__ float4 decode4(uint32_t c, float scale) {
    return float4{__builtin_amdgcn_cvt_f32_fp8((int)c, 0) * scale, __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * scale,
                  __builtin_amdgcn_cvt_f32_fp8((int)c, 2) * scale, __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * scale};
}

__device__ __forceinline__ uint32_t encode4(const float (&x)[4], float inv, const uint32_t (&rnd)[4]) {
#pragma clang fp contract(off)
    float q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = random_e4m3(x[j] * inv, rnd[j]);
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);  // exact: q are values of codes
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
}

// The largest finite magnitude over the wave's 256 values, by lane permutations within the vector unit: pairs, quads,
// eights and sixteens by mirrors, then rows of 16 into the next ones; lane 63 has seen all.
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_with(float t) {
    const int other = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, t), __builtin_bit_cast(int, t), CTRL, ROWS, 0xF, false);
    return fmaxf(t, __builtin_bit_cast(float, other));
}
__device__ __forceinline__ float wave_top(const float (&x)[4]) {
    float t = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = __builtin_fabsf(x[j]);
        t = a < __builtin_inff() ? fmaxf(t, a) : t;
    }
    t = max_with<0xB1, 0xF>(t);   // quad_perm [1, 0, 3, 2]
    t = max_with<0x4E, 0xF>(t);   // quad_perm [2, 3, 0, 1]
    t = max_with<0x141, 0xF>(t);  // row_half_mirror
    t = max_with<0x140, 0xF>(t);  // row_mirror
    t = max_with<0x142, 0xA>(t);  // row_bcast:15 into rows 1 and 3
    t = max_with<0x143, 0xC>(t);  // row_bcast:31 into rows 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, t), 63));
}

template <typename GT, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwBatch b) {
    // the tensor of this block: the last one whose first block is not behind it (a lane a tensor)
    const int lane = threadIdx.x & 63;
    static_assert(kAdamwTensors <= 64, "a lane a tensor");
    const uint64_t begun = __ballot(lane < b.n && b.t[lane < b.n ? lane : 0].first_block <= (int32_t)blockIdx.x);
    const int lo = __builtin_amdgcn_readfirstlane(63 - __clzll((long long)begun));
    const AdamwTensor& t = b.t[lo];
    const int64_t count = t.count;
    const int64_t base = (int64_t)((int32_t)blockIdx.x - t.first_block) * ((int64_t)b.rounds * kAdamwRound);

    const uint32_t step = b.step_dev ? (uint32_t)*b.step_dev : b.step;
    const double lr = b.lr_dev ? (double)*b.lr_dev : b.lr;
    __shared__ double bias[2];
    double c1 = b.c1, c2 = b.c2;
    if (b.step_dev) {
        if (threadIdx.x == 0) {
            bias[0] = 1.0 - power(b.beta1, step);
            bias[1] = 1.0 - power(b.beta2, step);
        }
        __syncthreads();
        c1 = bias[0];
        c2 = bias[1];
    }
    Factors f;
    f.b1 = (float)b.beta1;
    f.a1 = (float)(1.0 - b.beta1);
    f.b2 = (float)b.beta2;
    f.a2 = (float)(1.0 - b.beta2);
    f.decay = (float)(lr * (double)t.weight_decay);
    f.rate = (float)(lr / c1);
    f.root = 1.0f / sqrtf((float)c2);
    f.eps = (float)b.eps;

    float* const pw = t.w;
    const GT* const pg = reinterpret_cast<const GT*>(t.g);
    if constexpr (!EIGHT) {
        float* const pm = reinterpret_cast<float*>(t.m);
        float* const pv = reinterpret_cast<float*>(t.v);
#pragma unroll 2
        for (int k = 0; k < b.rounds; ++k) {
            const int64_t i = base + k * kAdamwRound + threadIdx.x * 4;
            if (i + 4 <= count) {
                float4 w = load4(pw + i), m = load4(pm + i), v = load4(pv + i);
                const float4 g = load4(pg + i);
                float r;
                update(w.x, m.x, v.x, r, g.x, f);
                update(w.y, m.y, v.y, r, g.y, f);
                update(w.z, m.z, v.z, r, g.z, f);
                update(w.w, m.w, v.w, r, g.w, f);
                *reinterpret_cast<f32x4_a4*>(pw + i) = f32x4{w.x, w.y, w.z, w.w};
                *reinterpret_cast<f32x4_a4*>(pm + i) = f32x4{m.x, m.y, m.z, m.w};
                *reinterpret_cast<f32x4_a4*>(pv + i) = f32x4{v.x, v.y, v.z, v.w};
            } else if (i < count) {  // the last 1 to 3: their loads go out together, the last one's again
                float w[3], m[3], v[3], g[3], r;
#pragma unroll
                for (int j = 0; j < 3; ++j) {
                    const int64_t e = i + j < count ? i + j : count - 1;
                    w[j] = pw[e];
                    m[j] = pm[e];
                    v[j] = pv[e];
                    g[j] = load1(pg + e);
                }
#pragma unroll
                for (int j = 0; j < 3; ++j) {
                    update(w[j], m[j], v[j], r, g[j], f);
                    if (i + j >= count) break;
                    pw[i + j] = w[j];
                    pm[i + j] = m[j];
                    pv[i + j] = v[j];
                }
            }
        }
    } else {
        uint8_t* const pm = reinterpret_cast<uint8_t*>(t.m);
        uint8_t* const pv = reinterpret_cast<uint8_t*>(t.v);
        const uint32_t key = mix(mix(mix(b.seed) ^ step) ^ (uint32_t)(b.first + lo));
        // a round: the wave's 256 elements of one scale
        struct Round {
            float4 w, g;
            uint32_t m, v;
            float ms, vs;
        };
        const int64_t blk0 = base / 256 + (threadIdx.x >> 6);
        auto load = [&](int k) {
            Round r;
            const int64_t i = base + k * kAdamwRound + threadIdx.x * 4;
            r.ms = t.m_scale[blk0 + 4 * k];
            r.vs = t.v_scale[blk0 + 4 * k];
            r.w = load4(pw + i);
            r.g = load4(pg + i);
            r.m = *reinterpret_cast<const u32_a1*>(pm + i);
            r.v = *reinterpret_cast<const u32_a1*>(pv + i);
            return r;
        };
        // ... with the first `left` of the lane's 4 elements inside the tensor
        auto step_round = [&](int k, Round& r, int left) {
            const int64_t i = base + k * kAdamwRound + threadIdx.x * 4;
            float w[4] = {r.w.x, r.w.y, r.w.z, r.w.w}, g[4] = {r.g.x, r.g.y, r.g.z, r.g.w}, m[4], v[4], root[4];
            const float4 m4 = decode4(r.m, r.ms), r4 = decode4(r.v, r.vs);
            m[0] = m4.x; m[1] = m4.y; m[2] = m4.z; m[3] = m4.w;
            v[0] = r4.x * r4.x; v[1] = r4.y * r4.y; v[2] = r4.z * r4.z; v[3] = r4.w * r4.w;
            uint32_t rm[4], rv[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                update(w[j], m[j], v[j], root[j], g[j], f);
                if (j >= left) m[j] = root[j] = 0.0f;
                const uint32_t h = mix((uint32_t)(i + j) ^ key);
                rm[j] = h & 0xFFFFFu;
                rv[j] = h >> 12;
            }
            const float tm = wave_top(m), tv = wave_top(root);
            // a block below 2^-100 is kept as zeros (1 / top has to be finite)
            const bool zm = tm < 0x1p-100f, zv = tv < 0x1p-100f;
            r.m = encode4(m, zm ? 0.0f : 448.0f * (1.0f / tm), rm);
            r.v = encode4(root, zv ? 0.0f : 448.0f * (1.0f / tv), rv);
            r.ms = zm ? 0.0f : tm * (1.0f / 448.0f);
            r.vs = zv ? 0.0f : tv * (1.0f / 448.0f);
            r.w = float4{w[0], w[1], w[2], w[3]};
            if ((threadIdx.x & 63) == 0) {
                t.m_scale[blk0 + 4 * k] = r.ms;
                t.v_scale[blk0 + 4 * k] = r.vs;
            }
        };
        auto whole = [&](auto rounds) {
            constexpr int N = decltype(rounds)::value;
            Round r[N];
#pragma unroll
            for (int k = 0; k < N; ++k) r[k] = load(k);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                step_round(k, r[k], 4);
                const int64_t i = base + k * kAdamwRound + threadIdx.x * 4;
                *reinterpret_cast<f32x4_a4*>(pw + i) = f32x4{r[k].w.x, r[k].w.y, r[k].w.z, r[k].w.w};
                *reinterpret_cast<u32_a1*>(pm + i) = r[k].m;
                *reinterpret_cast<u32_a1*>(pv + i) = r[k].v;
            }
        };
        if (base + (int64_t)b.rounds * kAdamwRound <= count) {
            if (b.rounds == 4) whole(std::integral_constant<int, 4>());
            else if (b.rounds == 2) whole(std::integral_constant<int, 2>());
            else whole(std::integral_constant<int, 1>());
            return;
        }
        for (int k = 0; k < b.rounds; ++k) {  // the tensor's end
            const int64_t i = base + k * kAdamwRound + threadIdx.x * 4;
            if ((blk0 + 4 * k) * 256 >= count) break;  // uniform in the wave
            const int left = i + 4 <= count ? 4 : (i < count ? (int)(count - i) : 0);
            Round r = {};
            if (left == 4) {
                r = load(k);
            } else {
                r.ms = t.m_scale[blk0 + 4 * k];
                r.vs = t.v_scale[blk0 + 4 * k];
                float w[3], g[3];
#pragma unroll
                for (int j = 0; j < 3; ++j) {  // behind the end the tensor's last one, not used
                    const int64_t e = i + j < count ? i + j : count - 1;
                    w[j] = pw[e];
                    g[j] = load1(pg + e);
                    r.m |= (uint32_t)pm[e] << (8 * j);
                    r.v |= (uint32_t)pv[e] << (8 * j);
                }
                r.w = float4{w[0], w[1], w[2], 0.0f};
                r.g = float4{g[0], g[1], g[2], 0.0f};
            }
            step_round(k, r, left);
            const float w[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j >= left) break;
                pw[i + j] = w[j];
                pm[i + j] = (uint8_t)(r.m >> (8 * j));
                pv[i + j] = (uint8_t)(r.v >> (8 * j));
            }
        }
    }
}

}  // namespace

hipError_t launch_adamw(const AdamwBatch& b, int64_t blocks, int g_bf16, int eight, hipStream_t stream) {
    const dim3 grid((unsigned)blocks);
    if (eight) {
        if (g_bf16) hipLaunchKernelGGL((adamw_kernel<uint16_t, true>), grid, dim3(256), 0, stream, b);
        else hipLaunchKernelGGL((adamw_kernel<float, true>), grid, dim3(256), 0, stream, b);
    } else {
        if (g_bf16) hipLaunchKernelGGL((adamw_kernel<uint16_t, false>), grid, dim3(256), 0, stream, b);
        else hipLaunchKernelGGL((adamw_kernel<float, false>), grid, dim3(256), 0, stream, b);
    }
    return hipGetLastError();
}

}  // namespace tbn
