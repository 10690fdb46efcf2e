// AdamW over many tensors at once, with the gradients' clipping, states in 32 bits or in FP8, and FP8 copies of the new weights, for gfx950 (MI355X).
//
//   g = c grad, c = min(1, max_norm / (norm + 1e-6)) or 1
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   p' = p - lr (wd p + (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps))
//   q = encode(p' s),  amax = max |p'|
//
// States in FP8: m and r = sqrt(v) in E4M3, 128 elements of a tensor with one factor each for m and r (448 over the block's largest magnitude).  r and not
// v is kept, since E4M3's range of 2^18 is then one of 2^36 of v.  Both are rounded stochastically: b2 near 1 moves r by far less than half
// a step of 3 mantissa bits at a time, so that rounding to nearest would leave it where it is for ever, while the expected value of what is stored here
// is what was computed.  Only r > 0 never becomes 0, which would make the next step's m / (sqrt(v) + eps) one over eps.  The weights are updated from the states
// before they are rounded.
#include "gemm_common.hpp"
#include "cast_common.hpp"
#include "fp8_stochastic.hpp"

#include <algorithm>

namespace fp8mm {
namespace {

constexpr int kAdamThreads = 256, kUnroll = 4;
constexpr unsigned kAdamChunk = kAdamThreads * 4 * kUnroll;     // elements
constexpr unsigned kParamF32 = 0x80000000u, kGradF32 = 0x40000000u;
constexpr int kAdamTensors = 50;

// Tensor t owns the chunks end[t - 1] .. end[t] - 1; size[t]: elements of its last chunk and the types; index[t]: its place in the caller's list.
struct AdamTensors {
    void* p[kAdamTensors];
    const void* g[kAdamTensors];
    void* m[kAdamTensors];
    void* v[kAdamTensors];
    float* m_scale[kAdamTensors];
    float* v_scale[kAdamTensors];
    uint8_t* q[kAdamTensors];
    float decay[kAdamTensors];
    unsigned end[kAdamTensors], size[kAdamTensors];
    int index[kAdamTensors];
    int count;
};
struct AdamScalars {
    const float* lr;
    const int64_t* step;
    const float* norm;
    const float* q_scale;
    float* q_amax;
    double beta1, beta2;
    float eps, max_norm;
    unsigned seed_lo, seed_hi;
    int q_fmt, skip_nonfinite;
};
static_assert(sizeof(AdamTensors) + sizeof(AdamScalars) < 4000, "kernel arguments");

// What is the same for all elements.
struct AdamStep { float clip, b1, o1, b2, o2, lr, k1, k2, eps; };

__device__ __forceinline__ double power(double b, uint64_t t)
{
    double r = 1.0;
    for (; t; t >>= 1, b *= b) if (t & 1) r *= b;
    return r;
}

// Four neighbouring values, `left` (1 to 4) of them there, the rest 0.
template <bool F32>
__device__ __forceinline__ void load4(const void* p, size_t at, int left, float (&x)[4])
{
    if (F32) {
        const float* f = (const float*)p + at;
        if (left >= 4) {
            const u32x4 v = __builtin_nontemporal_load((const u32x4_any*)f);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = as_f32(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i < left ? f[i] : 0.0f;
        }
    } else {
        const unsigned short* h = (const unsigned short*)p + at;
        if (left >= 4) {
            const u32x2 v = __builtin_nontemporal_load((const u32x2_any*)h);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = as_f32(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i < left ? as_f32((unsigned)h[i] << 16) : 0.0f;
        }
    }
}

template <bool F32>
__device__ __forceinline__ void store4(void* p, size_t at, int left, const float (&x)[4])
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    if (F32) {
        float* f = (float*)p + at;
        if (left >= 4) __builtin_nontemporal_store((u32x4){as_u32(x[0]), as_u32(x[1]), as_u32(x[2]), as_u32(x[3])}, (u32x4_any*)f);
        else {
#pragma unroll
            for (int i = 0; i < 3; ++i) if (i < left) f[i] = x[i];
        }
    } else {
        unsigned short* h = (unsigned short*)p + at;
        const unsigned a = __builtin_bit_cast(unsigned, __builtin_convertvector((f2){x[0], x[1]}, bf2)), b = __builtin_bit_cast(unsigned, __builtin_convertvector((f2){x[2], x[3]}, bf2));
        if (left >= 4) __builtin_nontemporal_store((u32x2){a, b}, (u32x2_any*)h);
        else {
#pragma unroll
            for (int i = 0; i < 3; ++i) if (i < left) h[i] = (unsigned short)((i >> 1 ? b : a) >> (16 * (i & 1)));
        }
    }
}

typedef unsigned word_any __attribute__((aligned(1)));

__device__ __forceinline__ unsigned load4_bytes(const uint8_t* p, int left)
{
    if (left >= 4) return *(const word_any*)p;
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) if (i < left) w |= (unsigned)p[i] << (8 * i);
    return w;
}
__device__ __forceinline__ void store4_bytes(uint8_t* p, int left, unsigned w)
{
    if (left >= 4) { *(word_any*)p = w; return; }
#pragma unroll
    for (int i = 0; i < 3; ++i) if (i < left) p[i] = (uint8_t)(w >> (8 * i));
}

// The largest magnitude over the 32 lanes that hold a block, as bits (a NaN's sort above infinity's).
__device__ __forceinline__ float block_top(const float (&x)[4])
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, as_u32(x[i]) & 0x7fffffffu);
#pragma unroll
    for (int d = 1; d <= 16; d <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
    return as_f32(top);
}

// The states are what the next step starts from: sums and products rounded one by one, so that they are the same however they are compiled.
#pragma clang fp contract(off)
__device__ __forceinline__ void moments(const AdamStep& s, const float (&g)[4], float (&m)[4], float (&v)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = g[i] * s.clip;
        m[i] = m[i] * s.b1 + x * s.o1;
        v[i] = v[i] * s.b2 + x * x * s.o2;
    }
}
#pragma clang fp contract(fast)

// r: sqrt(v')
__device__ __forceinline__ void weights(const AdamStep& s, float decay, const float (&m)[4], const float (&r)[4], float (&p)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float u = m[i] * s.k1 * __builtin_amdgcn_rcpf(__builtin_fmaf(r[i], s.k2, s.eps));
        p[i] = __builtin_fmaf(-s.lr, __builtin_fmaf(decay, p[i], u), p[i]);
    }
}

// count elements (up to a chunk) from element `at` of tensor t on.  Returns the largest |p'| as bits.
template <bool P32, bool G32, bool STATES8>
__device__ __forceinline__ unsigned adam_chunk(const AdamTensors& list, const AdamScalars& a, const AdamStep& s, int t, size_t at, unsigned count, unsigned step_bits)
{
    void* const pp = list.p[t];
    const void* const pg = list.g[t];
    const float decay = list.decay[t];
    uint8_t* const q = list.q[t];
    const float qs = q ? a.q_scale[list.index[t]] : 0.0f;
    unsigned top = 0;
    float p[kUnroll][4], g[kUnroll][4], m[kUnroll][4], v[kUnroll][4], fm[kUnroll], fr[kUnroll];
    unsigned mw[kUnroll], rw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const unsigned e = (u * kAdamThreads + threadIdx.x) * 4;
        const int left = e < count ? (int)min(count - e, 4u) : 0;
        mw[u] = rw[u] = 0; fm[u] = fr[u] = 1.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[u][i] = g[u][i] = m[u][i] = v[u][i] = 0.0f;
        if (left > 0) {
            load4<P32>(pp, at + e, left, p[u]);
            load4<G32>(pg, at + e, left, g[u]);
            if (STATES8) {
                mw[u] = load4_bytes((const uint8_t*)list.m[t] + at + e, left);
                rw[u] = load4_bytes((const uint8_t*)list.v[t] + at + e, left);
                fm[u] = list.m_scale[t][(at + e) / 128];
                fr[u] = list.v_scale[t][(at + e) / 128];
            } else {
                load4<true>(list.m[t], at + e, left, m[u]);
                load4<true>(list.v[t], at + e, left, v[u]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const unsigned e = (u * kAdamThreads + threadIdx.x) * 4;
        const int left = e < count ? (int)min(count - e, 4u) : 0;
        if (STATES8) {
            const float im = 1.0f / fm[u], ir = 1.0f / fr[u];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[u][i] = decode_fp8<FP8_E4M3>(mw[u] >> (8 * i) & 255u) * im;
                const float r = decode_fp8<FP8_E4M3>(rw[u] >> (8 * i) & 255u) * ir;
                v[u][i] = r * r;
            }
        }
        moments(s, g[u], m[u], v[u]);
        float r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __builtin_sqrtf(v[u][i]);
        weights(s, decay, m[u], r, p[u]);
        if (STATES8) {
            // (what lies beyond the tensor's end is 0 in m and r)
            const float sm = scale_rule(block_top(m[u]), FP8_E4M3), sr = scale_rule(block_top(r), FP8_E4M3);
            if (left > 0) {
                const size_t four = (at + e) / 4;
                unsigned bits[4];
                philox4x32_10((unsigned)four, (unsigned)(four >> 32), step_bits, (unsigned)list.index[t], a.seed_lo, a.seed_hi, bits);
                unsigned wm = 0, wr = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    wm |= encode_sr_bits<FP8_E4M3>(m[u][i] * sm, bits[i] & 0xffffu) << (8 * i);
                    unsigned c = encode_sr_bits<FP8_E4M3>(r[i] * sr, bits[i] >> 16);
                    if (c == 0u && r[i] > 0.0f) c = 1u;
                    wr |= c << (8 * i);
                }
                store4_bytes((uint8_t*)list.m[t] + at + e, left, wm);
                store4_bytes((uint8_t*)list.v[t] + at + e, left, wr);
                if ((threadIdx.x & 31) == 0) {
                    list.m_scale[t][(at + e) / 128] = sm;
                    list.v_scale[t][(at + e) / 128] = sr;
                }
            }
        } else if (left > 0) {
            store4<true>(list.m[t], at + e, left, m[u]);
            store4<true>(list.v[t], at + e, left, v[u]);
        }
        if (left > 0) {
            store4<P32>(pp, at + e, left, p[u]);
            if (q) {
#pragma unroll
                for (int i = 0; i < 4; ++i) if (i < left) top = max(top, as_u32(p[u][i]) & 0x7fffffffu);
                const float y0 = p[u][0] * qs, y1 = p[u][1] * qs, y2 = p[u][2] * qs, y3 = p[u][3] * qs;
                store4_bytes(q + at + e, left, a.q_fmt == FP8_E4M3 ? encode4<FP8_E4M3>(y0, y1, y2, y3) : encode4<FP8_E5M2>(y0, y1, y2, y3));
            }
        }
    }
    return top;
}

template <class L>
__device__ __forceinline__ int adam_tensor_of(const L& list, unsigned chunk)
{
    int lo = 0, hi = list.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (chunk < list.end[mid]) hi = mid; else lo = mid + 1;
    }
    return lo;
}

template <bool STATES8>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamTensors list, AdamScalars a, unsigned chunks)
{
    AdamStep s;
    s.clip = 1.0f;
    if (a.norm) {
        const float n = *a.norm;
        if (a.skip_nonfinite && !(__builtin_fabsf(n) < __builtin_inff())) return;
        s.clip = a.max_norm / (n + 1e-6f);
        if (s.clip > 1.0f) s.clip = 1.0f;        // (NaN stays)
        if (n == __builtin_inff()) s.clip = 0.0f;
    }
    const int64_t t_step = *a.step;
    s.b1 = (float)a.beta1; s.o1 = (float)(1.0 - a.beta1);
    s.b2 = (float)a.beta2; s.o2 = (float)(1.0 - a.beta2);
    s.lr = *a.lr; s.eps = a.eps;
    s.k1 = (float)(1.0 / (1.0 - power(a.beta1, (uint64_t)t_step)));
    s.k2 = (float)(1.0 / __builtin_sqrt(1.0 - power(a.beta2, (uint64_t)t_step)));
    for (unsigned c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = adam_tensor_of(list, c);
        const unsigned begin = t ? list.end[t - 1] : 0, size = list.size[t], count = c + 1 == list.end[t] ? size & ~(kParamF32 | kGradF32) : kAdamChunk;
        const size_t at = (size_t)(c - begin) * kAdamChunk;
        unsigned top;
        if (size & kParamF32) top = size & kGradF32 ? adam_chunk<true, true, STATES8>(list, a, s, t, at, count, (unsigned)t_step) : adam_chunk<true, false, STATES8>(list, a, s, t, at, count, (unsigned)t_step);
        else top = size & kGradF32 ? adam_chunk<false, true, STATES8>(list, a, s, t, at, count, (unsigned)t_step) : adam_chunk<false, false, STATES8>(list, a, s, t, at, count, (unsigned)t_step);
        if (a.q_amax && list.q[t]) wave_amax_commit(top, a.q_amax + list.index[t]);
    }
}

// (under the same condition as the step itself)
__global__ void adamw_clear_kernel(float* q_amax, int count, const float* norm, int skip_nonfinite)
{
    if (skip_nonfinite && norm && !(__builtin_fabsf(*norm) < __builtin_inff())) return;
    for (int i = threadIdx.x; i < count; i += blockDim.x) q_amax[i] = 0.0f;
}

}  // namespace

int launch_adamw(const AdamwArgs& a)
{
    AdamScalars s{};
    s.lr = a.lr; s.step = a.step; s.norm = a.norm; s.q_scale = a.q_scale; s.q_amax = a.q ? a.q_amax : nullptr;
    s.beta1 = a.beta1; s.beta2 = a.beta2; s.eps = a.eps; s.max_norm = a.max_norm;
    s.seed_lo = (unsigned)a.seed; s.seed_hi = (unsigned)(a.seed >> 32);
    s.q_fmt = a.q_fmt; s.skip_nonfinite = a.skip_nonfinite;
    if (a.q_amax && a.count > 0) {
        enqueue(adamw_clear_kernel, dim3(1), dim3(256), 0, a.stream, a.q_amax, a.count, a.norm, a.skip_nonfinite);
        if (int e = check_launch("AdamW (maxima)")) return e;
    }
    for (int i = 0; i < a.count;) {
        AdamTensors list{};
        unsigned chunks = 0;
        for (; i < a.count && list.count < kAdamTensors; ++i) {
            if (a.n[i] == 0) continue;
            const size_t more = (a.n[i] + kAdamChunk - 1) / kAdamChunk;
            if (chunks + more > 0xf0000000ull) break;
            chunks += (unsigned)more;
            const int k = list.count++;
            list.p[k] = a.p[i]; list.g[k] = a.g[i]; list.m[k] = a.m[i]; list.v[k] = a.v[i];
            if (a.states8) { list.m_scale[k] = a.m_scale[i]; list.v_scale[k] = a.v_scale[i]; }
            list.q[k] = a.q ? a.q[i] : nullptr;
            list.decay[k] = a.weight_decay ? a.weight_decay[i] : 0.0f;
            list.end[k] = chunks;
            list.size[k] = (unsigned)(a.n[i] - (more - 1) * kAdamChunk) | (a.p_dtype[i] == FP8_F32 ? kParamF32 : 0u) | (a.g_dtype[i] == FP8_F32 ? kGradF32 : 0u);
            list.index[k] = i;
        }
        if (chunks == 0) continue;
        const dim3 grid(std::min<unsigned>(chunks, 1u << 16));
        if (a.states8) enqueue(adamw_kernel<true>, grid, dim3(kAdamThreads), 0, a.stream, list, s, chunks);
        else enqueue(adamw_kernel<false>, grid, dim3(kAdamThreads), 0, a.stream, list, s, chunks);
        if (int e = check_launch("AdamW")) return e;
    }
    return FP8_OK;
}

}  // namespace fp8mm
