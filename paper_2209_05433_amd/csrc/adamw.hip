// AdamW over many tensors at once, with the gradients' clipping, states in 32 bits or in FP8, and FP8 copies of the new weights, for gfx950 (MI355X).
//
//   g = c grad, c = min(1, max_norm (1 / (norm + 1e-6))) or 1
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   p' = p - lr (wd p + (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps))
//   q = encode(p' s),  amax = max |p'|
//
// States in FP8: m and r = sqrt(v) in E4M3, 128 elements of a tensor with one factor each for m and r.  r and not
// v is kept, since E4M3's range of 2^18 is then one of 2^36 of v.  Both are rounded stochastically: b2 near 1 moves r by far less than half
// a step of 3 mantissa bits at a time, so that rounding to nearest would leave it where it is for ever, while the expected value of what is stored here
// is what was computed.  Only r > 0 is never rounded to 0, which would make the next step's m / (sqrt(v) + eps) one over eps.  The weights are updated from the states
// before they are rounded.
//
// HBM bound: one pass, with everything the step needs of an element loaded once (p, g, m, v) and stored once (p, m, v, q); 27 bytes an element with states in 32 bits
// and 15 in FP8, bf16 gradients and copies: 10^9 elements in 4.90 ms (5.55 TB/s; a copy 5.15) and 2.91 to 2.96 ms (5.15 to 5.23 TB/s, the vector ALU busy nearly all the time: the
// generator's ten rounds for four elements, two factors and two roundings).
#include "gemm_common.hpp"
#include "cast_common.hpp"
#include "fp8_stochastic.hpp"

#include <algorithm>
#include <type_traits>

namespace fp8mm {
namespace {

// Threads of a workgroup, quadruples of elements of a thread (with one 1.1 of the time, with eight the same; 512 and 1024 threads: 1.04 to 1.4).
constexpr int kAdamThreads = 256, U = 4;
constexpr unsigned kAdamChunk = kAdamThreads * 4 * U;           // elements
constexpr unsigned kMostGrid = 1u << 16, kAllAtOnce = 4096;     // workgroups
constexpr unsigned kParamF32 = 0x80000000u, kGradF32 = 0x40000000u;
constexpr size_t kAdamStreamBytes = (size_t)512 << 20;
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
// (the update is m' / (k r + eps), with 1 / (1 - b1^t) in k and eps.  Both are times `unit`, 1 but where the denominator may have no normal reciprocal: k is at least 2^-54
// and k r less than 2^92, so by an eps below 2^-126, where the unit is 2^30, or near 2^126, where it is 2^-30)
struct AdamStep {
    float clip, b1, o1, b2, o2, lr, k, eps, unit;
    bool small_eps;         // a root of less than 2^-63 counts beside eps
};

__device__ __forceinline__ double power(double b, uint64_t t)
{
    double r = 1.0;
    for (; t; t >>= 1, b *= b) if (t & 1) r *= b;
    return r;
}

// Four neighbouring values from element `at` on, `left` (1 to 4) of them there, the rest 0.
template <bool F32, bool STREAM>
__device__ __forceinline__ void load4(const void* p, unsigned at, int left, float (&x)[4])
{
    if (F32) {
        const float* f = (const float*)p + at;
        if (left >= 4) {
            const u32x4 v = STREAM ? __builtin_nontemporal_load((const u32x4_any*)f) : *(const u32x4_any*)f;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = as_f32(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i < left ? f[i] : 0.0f;
        }
    } else {
        const unsigned short* h = (const unsigned short*)p + at;
        if (left >= 4) {
            const u32x2 v = STREAM ? __builtin_nontemporal_load((const u32x2_any*)h) : *(const u32x2_any*)h;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = as_f32(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i < left ? as_f32((unsigned)h[i] << 16) : 0.0f;
        }
    }
}

template <bool F32, bool STREAM>
__device__ __forceinline__ void store4(void* p, unsigned at, int left, const float (&x)[4])
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    if (F32) {
        float* f = (float*)p + at;
        if (left >= 4) {
            const u32x4 v = {as_u32(x[0]), as_u32(x[1]), as_u32(x[2]), as_u32(x[3])};
            if (STREAM) __builtin_nontemporal_store(v, (u32x4_any*)f); else *(u32x4_any*)f = v;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) if (i < left) f[i] = x[i];
        }
    } else {
        unsigned short* h = (unsigned short*)p + at;
        const unsigned a = __builtin_bit_cast(unsigned, __builtin_convertvector((f2){x[0], x[1]}, bf2)), b = __builtin_bit_cast(unsigned, __builtin_convertvector((f2){x[2], x[3]}, bf2));
        if (left >= 4) {
            if (STREAM) __builtin_nontemporal_store((u32x2){a, b}, (u32x2_any*)h); else *(u32x2_any*)h = (u32x2){a, b};
        } else {
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

// 1 / x to the nearest: the instruction's is an ulp off, one step by Newton takes that away (every mantissa was tried); x whose inverse is no normal
// number comes out as infinity or 0 times it.
__device__ __forceinline__ float inverse(float x)
{
    const float r = __builtin_amdgcn_rcpf(x);
    return __builtin_fmaf(__builtin_fmaf(-x, r, 1.0f), r, r);
}

// The factor of a block: 448 times the reciprocal of its largest magnitude, over the 32 lanes that hold it (a NaN's bits sort above infinity's); 1 where
// that is 0 or not finite, or the factor not.  Rows of 16 lanes by moves within the vector registers, the two rows by one exchange.
template <int CTRL>
__device__ __forceinline__ unsigned row_max(unsigned x)
{
    return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false));
}
// finite: whether every magnitude of the block is.
__device__ __forceinline__ float block_factor(const float (&x)[4], bool& finite)
{
    unsigned top = max(max(as_u32(x[0]) & 0x7fffffffu, as_u32(x[1]) & 0x7fffffffu), max(as_u32(x[2]) & 0x7fffffffu, as_u32(x[3]) & 0x7fffffffu));
    top = row_max<0x128>(top);          // rotations by 8, 4, 2 and 1 lanes
    top = row_max<0x124>(top);
    top = row_max<0x122>(top);
    top = row_max<0x121>(top);
    top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
    const float f = 448.0f * inverse(as_f32(top));
    finite = top < 0x7f800000u;
    return finite && f < __builtin_inff() ? f : 1.0f;          // (f of 0 is infinite)
}

// The square root of a normal number, 0, infinity or NaN to the nearest: the instruction's is an ulp off, so its neighbours are looked at.
__device__ __forceinline__ float root_of_normal(float x)
{
    float s = __builtin_amdgcn_sqrtf(x);
    const float below = as_f32(as_u32(s) - 1u), above = as_f32(as_u32(s) + 1u);
    const float at_below = __builtin_fmaf(-below, s, x), at_above = __builtin_fmaf(-above, s, x);
    s = at_below <= 0.0f ? below : s;
    return at_above > 0.0f ? above : s;        // (0, infinity and NaN: every comparison is false)
}

// The square roots of four numbers.  The instruction takes what lies below 2^-126 for 0: in a wave with such a number (a block that no gradient has reached for
// long: sqrt(v) of 1e-19 would be left as the smallest code with factor 1, 2e-3) it is brought up by 2^64, and its root down by 2^32, which is exact.
__device__ __forceinline__ void roots(const float (&x)[4], float (&r)[4])
{
    unsigned least = as_u32(x[0]) - 1u;        // (0 wraps round)
#pragma unroll
    for (int i = 1; i < 4; ++i) least = min(least, as_u32(x[i]) - 1u);
    if (__builtin_expect(__any(least < 0x007fffffu), 0)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool below = x[i] < 0x1p-126f;
            const float s = root_of_normal(below ? x[i] * 0x1p64f : x[i]);
            r[i] = below ? s * 0x1p-32f : s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = root_of_normal(x[i]);
    }
}

// Four finite values as E4M3, rounded stochastically by 16 bits each in the upper halves of r (the lower ones 0).
__device__ __forceinline__ unsigned encode_states(const float (&y)[4], const unsigned (&r)[4])
{
    int w = 0;
    w = __builtin_amdgcn_cvt_sr_fp8_f32(__builtin_amdgcn_fmed3f(y[0], 448.0f, -448.0f), r[0], w, 0);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(__builtin_amdgcn_fmed3f(y[1], 448.0f, -448.0f), r[1], w, 1);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(__builtin_amdgcn_fmed3f(y[2], 448.0f, -448.0f), r[2], w, 2);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(__builtin_amdgcn_fmed3f(y[3], 448.0f, -448.0f), r[3], w, 3);
    return (unsigned)w;
}
// The same for any values (the instructions do not take NaN and infinities as the format does).
__device__ __forceinline__ unsigned encode_any_states(const float (&y)[4], const unsigned (&r)[4])
{
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= encode_sr_bits<FP8_E4M3>(y[i], r[i] >> 16) << (8 * i);
    return w;
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
        const float u = m[i] * __builtin_amdgcn_rcpf(__builtin_fmaf(r[i], s.k, s.eps)) * s.unit;
        p[i] = __builtin_fmaf(-s.lr, __builtin_fmaf(decay, p[i], u), p[i]);
    }
}

// What a chunk of a tensor needs, the same for all lanes; pointers to its first element.
struct AdamChunk {
    char* p; const char* g; char* m; char* v;
    float *m_scale, *v_scale;
    uint8_t* q;
    float decay, q_scale;
    unsigned count, four_lo, four_hi, step_bits, index;      // elements; the counter's words
};

// Returns the largest |p'| as bits.  FULL: the chunk is a whole one.
template <bool P32, bool G32, bool STATES8, bool FULL, bool STREAM>
__device__ __forceinline__ unsigned adam_chunk(const AdamChunk& c, const AdamScalars& a, const AdamStep& s)
{
    unsigned top = 0;
    float p[U][4], g[U][4], m[U][4], v[U][4], fm[U], fr[U];
    unsigned mw[U], rw[U];
    auto left_of = [&](unsigned e) __attribute__((always_inline)) { return FULL ? 4 : e < c.count ? (int)min(c.count - e, 4u) : 0; };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned e = (u * kAdamThreads + threadIdx.x) * 4;
        const int left = left_of(e);
        if (!FULL) {
            mw[u] = rw[u] = 0; fm[u] = fr[u] = 1.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) p[u][i] = g[u][i] = m[u][i] = v[u][i] = 0.0f;
        }
        if (left > 0) {
            load4<P32, STREAM>(c.p, e, left, p[u]);
            load4<G32, STREAM>(c.g, e, left, g[u]);
            if (STATES8) {
                mw[u] = load4_bytes((const uint8_t*)c.m + e, left);
                rw[u] = load4_bytes((const uint8_t*)c.v + e, left);
                fm[u] = c.m_scale[e / FP8_STATE_BLOCK];
                fr[u] = c.v_scale[e / FP8_STATE_BLOCK];
            } else {
                load4<true, STREAM>(c.m, e, left, m[u]);
                load4<true, STREAM>(c.v, e, left, v[u]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned e = (u * kAdamThreads + threadIdx.x) * 4;
        const int left = left_of(e);
        if (STATES8) {
            float im = inverse(fm[u]), ir = inverse(fr[u]);
            // (a factor below 2^-126 or beyond 2^126, of a block that has nearly vanished: the division itself)
            if (__builtin_expect(__any(max(as_u32(fm[u]) - 0x00800000u, as_u32(fr[u]) - 0x00800000u) > 0x7e800000u - 0x00800000u), 0)) { im = 1.0f / fm[u]; ir = 1.0f / fr[u]; }
            typedef float f2 __attribute__((ext_vector_type(2)));
            const f2 m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mw[u], false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mw[u], true);
            const f2 r01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)rw[u], false), r23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)rw[u], true);
            m[u][0] = m01.x * im; m[u][1] = m01.y * im; m[u][2] = m23.x * im; m[u][3] = m23.y * im;
            const float r[4] = {r01.x * ir, r01.y * ir, r23.x * ir, r23.y * ir};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[u][i] = r[i] * r[i];
        }
        moments(s, g[u], m[u], v[u]);
        float r[4];
        if (STATES8 || s.small_eps) roots(v[u], r);
        else {              // (one below 2^-63 as 0: half an ulp of eps at most)
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_sqrtf(v[u][i]);
        }
        weights(s, c.decay, m[u], r, p[u]);
        if (STATES8) {
            // (what lies beyond the tensor's end is 0 in m and r)
            bool finite_m, finite_r;
            const float sm = block_factor(m[u], finite_m), sr = block_factor(r, finite_r);
            const bool finite = __all(finite_m & finite_r);
            if (left > 0) {
                unsigned bits[4], low[4];
                philox4x32_10(c.four_lo + e / 4, c.four_hi, c.step_bits, c.index, a.seed_lo, a.seed_hi, bits);
                float x[4], y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = m[u][i] * sm;
                    low[i] = bits[i] << 16;
                    bits[i] &= 0xffff0000u;
                    y[i] = r[i] * sr;
                    y[i] = r[i] > 0.0f ? __builtin_fmaxf(y[i], 0.001953125f) : y[i];
                }
                unsigned wm, wr;
                if (__builtin_expect(finite, 1)) { wm = encode_states(x, low); wr = encode_states(y, bits); }
                else { wm = encode_any_states(x, low); wr = encode_any_states(y, bits); }
                store4_bytes((uint8_t*)c.m + e, left, wm);
                store4_bytes((uint8_t*)c.v + e, left, wr);
                if ((threadIdx.x & 31) == 0) {
                    c.m_scale[e / FP8_STATE_BLOCK] = sm;
                    c.v_scale[e / FP8_STATE_BLOCK] = sr;
                }
            }
        } else if (left > 0) {
            store4<true, STREAM>(c.m, e, left, m[u]);
            store4<true, STREAM>(c.v, e, left, v[u]);
        }
        if (left > 0) {
            store4<P32, STREAM>(c.p, e, left, p[u]);
            if (c.q) {
                unsigned most = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) if (FULL || i < left) most = max(most, as_u32(p[u][i]) & 0x7fffffffu);
                top = max(top, most);
                const float y0 = p[u][0] * c.q_scale, y1 = p[u][1] * c.q_scale, y2 = p[u][2] * c.q_scale, y3 = p[u][3] * c.q_scale;
                unsigned w;
                // (elements beyond the end are not stored, whatever becomes of them)
                if (__all(__builtin_fabsf(as_f32(most) * c.q_scale) < __builtin_inff())) {
                    w = a.q_fmt == FP8_E4M3 ? cvt_pair<FP8_E4M3, true>(y2, y3, cvt_pair<FP8_E4M3, false>(y0, y1, 0u)) : cvt_pair<FP8_E5M2, true>(y2, y3, cvt_pair<FP8_E5M2, false>(y0, y1, 0u));
                } else {
                    w = a.q_fmt == FP8_E4M3 ? encode4_bits<FP8_E4M3>(y0, y1, y2, y3) : encode4_bits<FP8_E5M2>(y0, y1, y2, y3);
                }
                store4_bytes(c.q + e, left, w);
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

template <bool STATES8, bool STREAM>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamTensors list, AdamScalars a, unsigned chunks)
{
    AdamStep s;
    s.clip = 1.0f;
    if (a.norm) {
        const float n = *a.norm;
        if (a.skip_nonfinite && !(__builtin_fabsf(n) < __builtin_inff())) return;
        // (Not the quotient: a number over a tensor in torch is this, and a factor that differs by an ulp makes a fifth of all m' do, and now and then an element round the
        // other way: where it is a block's largest, the block's next factor differs by a fourteenth.)
        s.clip = a.max_norm * (1.0f / (n + 1e-6f));
        if (s.clip > 1.0f) s.clip = 1.0f;        // (NaN stays)
        if (n == __builtin_inff()) s.clip = 0.0f;
    }
    const int64_t t_step = *a.step;
    s.b1 = (float)a.beta1; s.o1 = (float)(1.0 - a.beta1);
    s.b2 = (float)a.beta2; s.o2 = (float)(1.0 - a.beta2);
    const double c1 = 1.0 - power(a.beta1, (uint64_t)t_step), c2 = 1.0 - power(a.beta2, (uint64_t)t_step);
    s.lr = *a.lr;
    const double k = c1 / __builtin_sqrt(c2), eps = c1 * (double)a.eps, unit = eps < 0x1p-126 ? 0x1p30 : eps > 0x1p125 ? 0x1p-30 : 1.0;
    s.k = (float)(k * unit);
    s.eps = (float)(eps * unit);
    s.unit = (float)unit;
    s.small_eps = !(eps >= k * 0x1p-38);
    __shared__ unsigned tops[kAdamThreads / 64];
    // neighbouring chunks, so that a workgroup's maximum is of one tensor mostly
    const unsigned share = chunks / gridDim.x, rest = chunks % gridDim.x, b = blockIdx.x;
    const unsigned first = b * share + min(b, rest), end = first + share + (b < rest ? 1u : 0u);
    unsigned top = 0;
    int t = adam_tensor_of(list, first);
    for (unsigned c = first; c < end; ++c) {
        if (c == list.end[t]) ++t;
        const unsigned begin = t ? list.end[t - 1] : 0, size = list.size[t], count = c + 1 == list.end[t] ? size & ~(kParamF32 | kGradF32) : kAdamChunk;
        const size_t at = (size_t)(c - begin) * kAdamChunk;
        const int pb = size & kParamF32 ? 4 : 2, gb = size & kGradF32 ? 4 : 2, sb = STATES8 ? 1 : 4;
        // (a chunk begins at a multiple of its size: the upper word of the counter is the same for all of it, and with it a part of the generator's first rounds)
        const AdamChunk k = {(char*)list.p[t] + at * pb, (const char*)list.g[t] + at * gb, (char*)list.m[t] + at * sb, (char*)list.v[t] + at * sb,
                             list.m_scale[t] + at / FP8_STATE_BLOCK, list.v_scale[t] + at / FP8_STATE_BLOCK, list.q[t] ? list.q[t] + at : nullptr, list.decay[t],
                             list.q[t] ? a.q_scale[list.index[t]] : 0.0f, count, (unsigned)(at / 4), (unsigned)(at >> 34), (unsigned)t_step, (unsigned)list.index[t]};
        auto run = [&](auto p32, auto g32) __attribute__((always_inline)) {
            return count == kAdamChunk ? adam_chunk<decltype(p32)::value, decltype(g32)::value, STATES8, true, STREAM>(k, a, s)
                                          : adam_chunk<decltype(p32)::value, decltype(g32)::value, STATES8, false, STREAM>(k, a, s);
        };
        const std::integral_constant<bool, true> yes;
        const std::integral_constant<bool, false> no;
        const unsigned of_chunk = size & kParamF32 ? (size & kGradF32 ? run(yes, yes) : run(yes, no)) : size & kGradF32 ? run(no, yes) : run(no, no);
        top = max(top, of_chunk);
        if (a.q_amax && k.q && (c + 1 == end || c + 1 == list.end[t])) {
            // One atomic a workgroup and tensor.  Where many workgroups are behind one another most find a larger value in the cell and leave it at that; where all are
            // at work at once they would only queue up for the look as well (864 workgroups, 96 MB: 33.8 us with it, 23.6 without, 18.2 without maxima).
            __syncthreads();
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
            if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
            __syncthreads();
            if (threadIdx.x == 0) {
                unsigned* cell = (unsigned*)a.q_amax + k.index;
                top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
                if (gridDim.x <= kAllAtOnce || top > __hip_atomic_load(cell, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(cell, top);
            }
            top = 0;
        }
    }
}

// (under the same condition as the step itself)
__global__ void adamw_clear_kernel(float* q_amax, int count, const float* norm, int skip_nonfinite)
{
    if (skip_nonfinite && norm && !(__builtin_fabsf(*norm) < __builtin_inff())) return;
    for (int i = threadIdx.x; i < count; i += blockDim.x) q_amax[i] = 0.0f;
}

}  // namespace

namespace {

template <bool STREAM>
int launch_lists(const AdamwArgs& a, const AdamScalars& s)
{
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
        const dim3 grid(std::min(chunks, kMostGrid));
        if (a.states8) enqueue((adamw_kernel<true, STREAM>), grid, dim3(kAdamThreads), 0, a.stream, list, s, chunks);
        else enqueue((adamw_kernel<false, STREAM>), grid, dim3(kAdamThreads), 0, a.stream, list, s, chunks);
        if (int e = check_launch("AdamW")) return e;
    }
    return FP8_OK;
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
    // Loads and stores that leave the caches alone where no cache holds the tensors anyway (us, ordinary / streaming, with copies and maxima: states in 32 bits 266 MB 45 / 49,
    // 383 MB 62 / 70, 482 MB 93 / 101, 574 MB 117 / 117, 673 MB 137 / 131, 1.36 GB 267 / 247, 27.2 GB 5110 / 4945; in FP8 149 MB 43 / 43, 270 MB 67 / 75, 377 MB 80 / 89,
    // 583 MB 142 / 132, 762 MB 179 / 162, 15.2 GB 3010 / 2916).
    size_t bytes = 0;
    for (int i = 0; i < a.count; ++i)
        bytes += a.n[i] * (size_t)((a.p_dtype[i] == FP8_F32 ? 8 : 4) + (a.g_dtype[i] == FP8_F32 ? 4 : 2) + (a.states8 ? 4 : 16) + (a.q && a.q[i] ? 1 : 0));
    return bytes >= kAdamStreamBytes ? launch_lists<true>(a, s) : launch_lists<false>(a, s);
}

}  // namespace fp8mm
