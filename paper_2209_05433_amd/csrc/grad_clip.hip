// Global norm of many gradient tensors, and their clipping to it, for gfx950 (MI355X).
//
//   norm = sqrt(sum over all tensors and elements of x^2);  out = x min(1, max_norm / (norm + 1e-6))
//
// The squares are added in 64 bits: no sum overflows or loses its small terms, however long the tensors or large their elements are
// (an fp32 square overflows beyond 1.8e19).  Every thread, workgroup and launch adds in a fixed order: the result is the same in every run.
//
// The tensors, up to a few hundred a launch, come in the kernel's arguments (no table in device memory that somebody would have to copy
// and keep); they are cut into chunks of kChunk elements, which a grid of at most kMostBlocks workgroups walks.  Bound by memory: 2 or 4
// bytes read an element for the norm, as many read and written for the clipping.  The clipping walks the chunks from the last to the
// first: what the norm has read last is still in the last-level cache.  2 GB of bf16: the norm at 5.7 TB/s (355 us), the clipping at
// 6.2 (650).  An empty tensor or a single one costs a search over the list, per chunk, that other workgroups hide (chunks one behind the other: 360).
#include "gemm_common.hpp"

#include <algorithm>

namespace fp8mm {
namespace {

constexpr int kThreads = 256;
constexpr unsigned kChunk = 16384;              // elements
constexpr int kMostBlocks = 2048;               // of the norm: partial sums in the workspace
constexpr unsigned kF32 = 0x80000000u;

// Workspace: the sum of the launches before; tickets, zero between launches (of groups of workgroups, a line each, and of the groups: a thousand
// workgroups that end together would queue up at one counter); partial sums.
constexpr unsigned kGroup = 32;
struct NormWorkspace {
    unsigned groups_done, pad;
    double before;
    unsigned rest[28];
    unsigned done[kMostBlocks / kGroup][32];
    double part[kMostBlocks];
};
static_assert(sizeof(NormWorkspace) <= FP8_GRAD_NORM_WORKSPACE_BYTES, "the workspace that callers provide");

// Tensor t owns the chunks end[t - 1] .. end[t] - 1; size[t]: elements of its last chunk, kF32 set for fp32.
template <int T, bool OUT>
struct Tensors {
    const void* x[T];
    void* out[OUT ? T : 1];
    unsigned end[T], size[T];
    int count;
};
typedef Tensors<240, false> NormTensors;        // (the arguments of a launch end at 4 KB)
typedef Tensors<160, true> ClipTensors;
static_assert(sizeof(NormTensors) < 4000 && sizeof(ClipTensors) < 4000, "kernel arguments");

template <class L>
__device__ __forceinline__ int tensor_of(const L& list, unsigned chunk)
{
    int lo = 0, hi = list.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (chunk < list.end[mid]) hi = mid; else lo = mid + 1;
    }
    return lo;
}

template <bool F32> struct Piece { static constexpr int N = F32 ? 4 : 8; };    // elements in 16 bytes

__device__ __forceinline__ float bf16_at(u32x4 v, int i) { return as_f32(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }

__device__ __forceinline__ double square(float f) { return (double)f * (double)f; }

// Sum of squares of `count` elements from `base` on, this thread's share.
template <bool F32>
__device__ __forceinline__ double squares(const void* base, unsigned count)
{
    constexpr int N = Piece<F32>::N, STEP = kThreads * N, U = kChunk / STEP;
    const char* p = (const char*)base;
    constexpr int ESZ = F32 ? 4 : 2;
    double s0 = 0.0, s1 = 0.0;
    auto add = [&](u32x4 v) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float a = F32 ? as_f32(v[i & 3]) : bf16_at(v, i), b = F32 ? as_f32(v[(i + 1) & 3]) : bf16_at(v, i + 1);
            s0 = __builtin_fma((double)a, (double)a, s0);
            s1 = __builtin_fma((double)b, (double)b, s1);
        }
    };
    if (count == kChunk) {
        u32x4 v[8];
#pragma unroll
        for (int h = 0; h < U / 8; ++h) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = *(const u32x4_any*)(p + (size_t)((8 * h + i) * STEP + threadIdx.x * N) * ESZ);
#pragma unroll
            for (int i = 0; i < 8; ++i) add(v[i]);
        }
    } else {
        unsigned at = threadIdx.x * N;
        for (; at + N <= count; at += STEP) add(*(const u32x4_any*)(p + (size_t)at * ESZ));
        for (unsigned i = at; i < count && i < at + N; ++i)
            s0 += square(F32 ? ((const float*)p)[i] : as_f32((unsigned)((const unsigned short*)p)[i] << 16));
    }
    return s0 + s1;
}

__device__ __forceinline__ double block_sum(double s, double* cells)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if ((threadIdx.x & 63) == 0) cells[threadIdx.x >> 6] = s;
    __syncthreads();
    return (cells[0] + cells[1]) + (cells[2] + cells[3]);
}

// first, last: of the launches that make up one call.
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(NormTensors list, unsigned chunks, bool first, bool last, float* norm_out, NormWorkspace* ws)
{
    __shared__ double cells[4];
    __shared__ bool closes;
    double s = 0.0;
    for (unsigned c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = tensor_of(list, c);
        const unsigned begin = t ? list.end[t - 1] : 0, size = list.size[t], count = c + 1 == list.end[t] ? size & ~kF32 : kChunk;
        const size_t at = (size_t)(c - begin) * kChunk;
        s += size & kF32 ? squares<true>((const float*)list.x[t] + at, count) : squares<false>((const unsigned short*)list.x[t] + at, count);
    }
    s = block_sum(s, cells);
    // The workgroup that is done last adds all partial sums in their order.  A partial sum is stored where every other workgroup sees it
    // (agent scope) and acknowledged before the ticket is drawn; no other data is exchanged.
    if (threadIdx.x == 0) {
        __hip_atomic_store(&ws->part[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        __builtin_amdgcn_s_waitcnt(0x0070);      // vmcnt(0), lgkmcnt(0)
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        const unsigned g = blockIdx.x / kGroup, groups = (gridDim.x + kGroup - 1) / kGroup, members = min(kGroup, gridDim.x - g * kGroup);
        bool l = false;
        if (__hip_atomic_fetch_add(&ws->done[g][0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == members - 1) {
            __hip_atomic_store(&ws->done[g][0], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            l = __hip_atomic_fetch_add(&ws->groups_done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
        }
        closes = l;
    }
    __syncthreads();
    if (!closes) return;
    double total = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads) total += __hip_atomic_load(&ws->part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    total = block_sum(total, cells);
    if (threadIdx.x == 0) {
        if (!first) total += ws->before;
        if (last) *norm_out = (float)__builtin_sqrt(total); else ws->before = total;
        __hip_atomic_store(&ws->groups_done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

template <bool F32>
__device__ __forceinline__ u32x4 scaled(u32x4 v, float f)
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (F32) r[i] = as_u32(as_f32(v[i]) * f);
        else r[i] = __builtin_bit_cast(unsigned, __builtin_convertvector((f2){bf16_at(v, 2 * i) * f, bf16_at(v, 2 * i + 1) * f}, bf2));
    }
    return r;
}

// Loads and stores that leave no line behind in the caches where no cache holds the tensors anyway (stores alone, or loads alone, gain nothing there).
// Norm and clipping together, ordinary / streaming (us): out of place 128 MB 64 / 66, 256 MB 140 / 125, 384 MB 213 / 185, 512 MB 283 / 245, 2 GB 1069 / 955;
// in place 128 MB 65 / 70, 256 MB 121 / 128, 384 MB 194 / 186, 512 MB 286 / 249, 2 GB 1092 / 980.
constexpr size_t kStreamBytes = (size_t)384 << 20;
template <bool STREAM> __device__ __forceinline__ u32x4 load_piece(const char* p)
{
    return STREAM ? __builtin_nontemporal_load((const u32x4_any*)p) : *(const u32x4_any*)p;
}
template <bool STREAM> __device__ __forceinline__ void store_piece(char* p, u32x4 v)
{
    if (STREAM) __builtin_nontemporal_store(v, (u32x4_any*)p); else *(u32x4_any*)p = v;
}

// (x and out may be one tensor: a thread stores only what it has loaded)
template <bool F32, bool STREAM>
__device__ __forceinline__ void scale_chunk(const void* x, void* out, unsigned count, float f)
{
    constexpr int N = Piece<F32>::N, STEP = kThreads * N, U = kChunk / STEP, ESZ = F32 ? 4 : 2;
    const char* p = (const char*)x;
    char* q = (char*)out;
    if (count == kChunk) {
        u32x4 v[8];
#pragma unroll
        for (int h = 0; h < U / 8; ++h) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = load_piece<STREAM>(p + (size_t)((8 * h + i) * STEP + threadIdx.x * N) * ESZ);
#pragma unroll
            for (int i = 0; i < 8; ++i) store_piece<STREAM>(q + (size_t)((8 * h + i) * STEP + threadIdx.x * N) * ESZ, scaled<F32>(v[i], f));
        }
    } else {
        unsigned at = threadIdx.x * N;
        for (; at + N <= count; at += STEP) *(u32x4_any*)(q + (size_t)at * ESZ) = scaled<F32>(*(const u32x4_any*)(p + (size_t)at * ESZ), f);
        for (unsigned i = at; i < count && i < at + N; ++i) {
            if (F32) ((float*)q)[i] = ((const float*)p)[i] * f;
            else ((unsigned short*)q)[i] = (unsigned short)scaled<false>((u32x4){((const unsigned short*)p)[i], 0u, 0u, 0u}, f)[0];
        }
    }
}

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(ClipTensors list, unsigned chunks, const float* norm, float max_norm, bool in_place)
{
    const float n = *norm;
    float f = max_norm / (n + 1e-6f);
    if (f > 1.0f) f = 1.0f;                      // (NaN stays)
    if (n == __builtin_inff()) f = 0.0f;         // (also where max_norm is infinite)
    if (in_place && f == 1.0f) return;           // x 1 = x
    for (unsigned c = blockIdx.x; c < chunks; c += gridDim.x) {
        // the list begins with the last tensor; its chunks from the last one on
        const int t = tensor_of(list, c);
        const unsigned begin = t ? list.end[t - 1] : 0, size = list.size[t], count = c == begin ? size & ~kF32 : kChunk;
        const size_t at = (size_t)(list.end[t] - 1 - c) * kChunk;
        if (size & kF32) scale_chunk<true, STREAM>((const float*)list.x[t] + at, (float*)list.out[t] + at, count, f);
        else scale_chunk<false, STREAM>((const unsigned short*)list.x[t] + at, (unsigned short*)list.out[t] + at, count, f);
    }
}

inline size_t chunks_of(size_t n) { return (n + kChunk - 1) / kChunk; }

// Tensors i, i + step, ... (backwards for step = -1) into the list until it is full; empty ones are left out.  Returns the chunks.
template <class L, int T>
unsigned fill(L& list, int& i, int end, int step, const void* const* x, void* const* out, const size_t* n, const int* dtype)
{
    unsigned chunks = 0;
    list.count = 0;
    for (; i != end && list.count < T; i += step) {
        if (n[i] == 0) continue;
        const size_t more = chunks_of(n[i]);
        if (chunks + more > 0xf0000000ull) break;
        chunks += (unsigned)more;
        list.x[list.count] = x[i];
        if (out) list.out[list.count] = out[i];
        list.end[list.count] = chunks;
        list.size[list.count] = (unsigned)(n[i] - (more - 1) * kChunk) | (dtype[i] == FP8_F32 ? kF32 : 0u);
        ++list.count;
    }
    return chunks;
}

}  // namespace

int launch_grad_norm(int count, const void* const* x, const size_t* n, const int* dtype, float* norm_out, void* workspace, hipStream_t stream)
{
    int i = 0;
    bool first = true;
    do {
        NormTensors list{};
        const unsigned chunks = fill<NormTensors, 240>(list, i, count, 1, x, nullptr, n, dtype);
        const unsigned grid = std::min<unsigned>(std::max(chunks, 1u), kMostBlocks);
        bool last = true;
        for (int j = i; j < count; ++j) last = last && n[j] == 0;
        enqueue(grad_norm_kernel, dim3(grid), dim3(kThreads), 0, stream, list, chunks, first, last, norm_out, (NormWorkspace*)workspace);
        if (int e = check_launch("gradient norm")) return e;
        if (last) break;
        first = false;
    } while (i < count);
    return FP8_OK;
}

int launch_grad_clip(int count, const void* const* x, const size_t* n, const int* dtype, void* const* out, const float* norm, float max_norm, hipStream_t stream)
{
    size_t bytes = 0;
    for (int i = 0; i < count && bytes < kStreamBytes; ++i) bytes += n[i] * (dtype[i] == FP8_F32 ? 4 : 2);
    for (int i = count - 1; i >= 0;) {
        ClipTensors list{};
        const unsigned chunks = fill<ClipTensors, 160>(list, i, -1, -1, x, out, n, dtype);
        if (chunks == 0) continue;
        bool in_place = true;
        for (int t = 0; t < list.count; ++t) in_place = in_place && list.out[t] == list.x[t];
        const dim3 grid(std::min<unsigned>(chunks, 1u << 16));
        if (bytes < kStreamBytes) enqueue(grad_clip_kernel<false>, grid, dim3(kThreads), 0, stream, list, chunks, norm, max_norm, in_place);
        else enqueue(grad_clip_kernel<true>, grid, dim3(kThreads), 0, stream, list, chunks, norm, max_norm, in_place);
        if (int e = check_launch("gradient clipping")) return e;
    }
    return FP8_OK;
}

}  // namespace fp8mm
