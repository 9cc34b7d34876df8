// hcw_clip.cu -- the norm over the gradients of all parameters, and clipping by it
// (hcw_clip_grads):
//
//   n = sqrt(sum over tensors i and elements j of g_ij^2),  c = min(1, max_norm / n),
//   out_ij = c g_ij
//
// Bound by memory: every element is read for the norm and, as the factor is not known before
// the last of them, read again and written for the product.  Two launches for up to 512 tensors,
// whatever their sizes: each tensor is cut into chunks, the chunks of all tensors are numbered
// through, and the CTAs take them in turn.  The second launch goes through them backwards, so that
// what the first one read last is found in L2.
//
// The squares of a warp's elements of one chunk (8 to 64 a thread) are added in fp32, everything above in
// fp64.  Squares of fp32 or bf16 gradients may leave fp32's range: a warp whose sum did, or lies where
// squares lose their last bits, takes its elements again with a power of two before them, so the norm
// is right to a few parts in 2^24 for any finite gradients.
#include "hcw.h"
#include "hcw_internal.h"

#include <math.h>

#include <algorithm>
#include <new>
#include <type_traits>

namespace hcw {

namespace {

constexpr int kCThreads = 512;
constexpr int kCParts = 1024;                    // CTAs of a launch at most
constexpr int kCTensors = 512;                   // tensors of a launch at most
constexpr long long kCMaxChunks = 1ll << 30;     // of a launch

struct ClipTensor {
    const void* g;
    void* out;
    long long n;
};

// The tensors of a launch, passed by value: 32 of them or 512.  Chunks have PER elements a thread.
template <int N>
struct ClipArgs {
    ClipTensor t[N];
    int first[N + 1];        // the tensor's first chunk; first[count]: chunks in all
    unsigned char f32[N];
    int count;
    double* parts;           // sums of squares, one of each CTA
    int n_parts;             // of all launches (second kernel)
    float max_norm;
    float* norm;             // null: another launch writes it
    int in_place;
};

// Elements before p's first 16-byte boundary (as many as the tensor has, at most).
__device__ __forceinline__ int head_of(const void* p, int es, long long n) {
    const int h = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / es;
    return h < n ? h : (int)n;
}

// The chunk's tensor: the last one whose first chunk is not past it.
template <int N>
__device__ __forceinline__ int tensor_of(const ClipArgs<N>& a, int chunk) {
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.first[mid] <= chunk)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

template <typename T>
struct Vec {   // 16 bytes of T
    static constexpr int n = 16 / sizeof(T);
};

__device__ __forceinline__ void unpack(const uint4& q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x);
    v[1] = __uint_as_float(q.y);
    v[2] = __uint_as_float(q.z);
    v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The thread's share of the elements [lo, hi) of g, whose vectors start at its element `head`:
// the sum of (f g)^2, and in *any whether one of them is not zero.
template <typename T, int PER>
__device__ __forceinline__ float squares(const T* g, long long lo, long long hi, float f, bool* any) {
    constexpr int VE = Vec<T>::n, NV = PER / VE;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t bits = 0;
    const long long vecs = (hi - lo) / VE;   // lo is on a boundary
    uint4 q[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const long long k = threadIdx.x + (long long)i * kCThreads;
        q[i] = k < vecs ? reinterpret_cast<const uint4*>(g + lo)[k] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float v[VE];
        unpack(q[i], v);
        bits |= q[i].x | q[i].y | q[i].z | q[i].w;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float x = v[e] * f;
            s[e & 3] = fmaf(x, x, s[e & 3]);
        }
    }
    const long long rest = lo + vecs * VE + threadIdx.x;
    if (rest < hi) {
        const float x = value(g + rest) * f;
        bits |= __float_as_uint(x) | (uint32_t)(x != 0.f);
        s[0] = fmaf(x, x, s[0]);
    }
    *any = bits != 0;
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// The elements of chunk c of a tensor of n: chunk 0 takes those before the first boundary too.
template <int PER>
__device__ __forceinline__ void chunk_span(long long c, int head, long long n, long long* lo,
                                           long long* hi) {
    *lo = head + c * (kCThreads * PER);
    *hi = *lo + kCThreads * PER < n ? *lo + kCThreads * PER : n;
    if (*lo > n) *lo = n;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The warp's share of a chunk, on every lane (fp64 is slow here: one sum a warp and chunk).
template <typename T, int PER>
__device__ __forceinline__ double chunk_squares(const ClipTensor& t, int c) {
    const T* g = static_cast<const T*>(t.g);
    const int head = head_of(g, sizeof(T), t.n);
    long long lo, hi;
    chunk_span<PER>(c, head, t.n, &lo, &hi);
    float edge = 0.f;
    if (c == 0 && (int)threadIdx.x < head) edge = value(g + threadIdx.x);
    bool any;
    const float s = warp_sum(squares<T, PER>(g, lo, hi, 1.f, &any) + edge * edge);
    // 2^-60 and above: what a square lost below 2^-149 is nothing beside it
    if (s >= 0x1p-60f && s < INFINITY) return (double)s;
    if (!__any_sync(0xffffffffu, any || edge != 0.f)) return 0.0;
    // squares that fp32 does not hold: with 2^90 (elements below 2^-30) or 2^-70 before the
    // elements; infinities and NaN stay
    const float f = s < 1.f ? 0x1p90f : 0x1p-70f;
    const float again = warp_sum(squares<T, PER>(g, lo, hi, f, &any) + (edge * f) * (edge * f));
    return (double)again * (s < 1.f ? 0x1p-180 : 0x1p140);
}

// A CTA's sum of squares.  Two CTAs an SM, so that a thread's 16 vectors stay in registers at once:
// 475 M bf16 gradients 137 us, 6.9 TB/s; 109 M fp32 65 us, 6.6 TB/s.
template <int N, int PER>
__global__ void __launch_bounds__(kCThreads, 2) clip_norm_kernel(const __grid_constant__ ClipArgs<N> a) {
    pdl_wait();
    pdl_trigger();
    __shared__ double part[kCThreads / 32];
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    const int chunks = a.first[a.count];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int i = tensor_of(a, c);
        const double s = a.f32[i] ? chunk_squares<float, PER>(a.t[i], c - a.first[i])
                                  : chunk_squares<__nv_bfloat16, PER>(a.t[i], c - a.first[i]);
        if (lane == 0) sum += s;
    }
    if (lane == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    sum = warp_sum(lane < kCThreads / 32 ? part[lane] : 0.0);
    if (lane == 0) a.parts[blockIdx.x] = sum;
}

// What the sum of squares says: the norm, the factor, and the factor as two (pre = 2^-40 apart where
// fp32 would hold the factor in fewer bits; what that takes below fp32's normal numbers ends at zero).
// fp64's own root and quotient take about a microsecond here: fp32's, with one correction each from their
// remainder in fp64, are right to their last bit but for ties.
struct Clip {
    float norm, factor, pre, rest;
};
__device__ __forceinline__ Clip clip_of(double sum, float max_norm) {
    Clip c = {(float)sum, 1.f, 1.f, 1.f};   // 0, infinity or NaN
    if (sum > 0.0 && sum < INFINITY) {
        const int e = ((__double2hiint(sum) >> 20) - 1023) & ~1, h = e / 2;
        const double lead = sum * __hiloint2double((1023 - e) << 20, 0);   // 1 .. 4
        const float r = sqrtf((float)lead);
        const double root = (double)r + (double)((float)(lead - (double)r * r) * 0.5f / r);
        c.norm = scalbnf((float)root, h);
        if (c.norm > max_norm) {
            // (a limit of few bits is scaled before the quotient would lose its own)
            const bool small = max_norm < 0x1p-60f;
            const float limit = small ? max_norm * 0x1p64f : max_norm, q0 = limit / r;
            const float q = (float)((double)q0 + (double)((float)((double)limit - q0 * root) / r));
            const int shift = small ? -h - 64 : -h;
            c.factor = c.rest = scalbnf(q, shift);
            if (c.factor < 0x1p-80f) {
                c.pre = 0x1p-40f;
                c.rest = scalbnf(q, shift + 40);
            }
        }
    }
    return c;
}

template <typename T, int PER>
__device__ __forceinline__ void chunk_scale(const ClipTensor& t, int c, float pre, float f) {
    constexpr int VE = Vec<T>::n, NV = PER / VE;
    const T* g = static_cast<const T*>(t.g);
    T* out = static_cast<T*>(t.out);
    const int head = head_of(g, sizeof(T), t.n);
    long long lo, hi;
    chunk_span<PER>(c, head, t.n, &lo, &hi);
    if (c == 0 && (int)threadIdx.x < head) put(out + threadIdx.x, value(g + threadIdx.x) * pre * f);
    const bool same = ((reinterpret_cast<uintptr_t>(out + lo)) & 15) == 0;
    const long long vecs = (hi - lo) / VE;
    uint4 q[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const long long k = threadIdx.x + (long long)i * kCThreads;
        if (k < vecs) q[i] = reinterpret_cast<const uint4*>(g + lo)[k];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const long long k = threadIdx.x + (long long)i * kCThreads;
        if (k >= vecs) continue;
        float v[VE];
        unpack(q[i], v);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] *= pre;
        if (same) {
            uint4 r;
            if constexpr (VE == 4) {
                r = make_uint4(__float_as_uint(v[0] * f), __float_as_uint(v[1] * f),
                               __float_as_uint(v[2] * f), __float_as_uint(v[3] * f));
            } else {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * e] * f, v[2 * e + 1] * f);
                    w[e] = *reinterpret_cast<const uint32_t*>(&p);
                }
                r = make_uint4(w[0], w[1], w[2], w[3]);
            }
            reinterpret_cast<uint4*>(out + lo)[k] = r;
        } else {   // the output lies otherwise than the input
#pragma unroll
            for (int e = 0; e < VE; ++e) put(out + lo + k * VE + e, v[e] * f);
        }
    }
    const long long rest = lo + vecs * VE + threadIdx.x;
    if (rest < hi) put(out + rest, value(g + rest) * pre * f);
}

// Every CTA takes the norm from the CTAs' sums itself, then its chunks from the last one back: 475 M bf16
// gradients 285 us alone, 6.7 TB/s; 305 behind the norm, 6.2 TB/s.
template <int N, int PER>
__global__ void __launch_bounds__(kCThreads, 2) clip_scale_kernel(const __grid_constant__ ClipArgs<N> a) {
    pdl_wait();
    pdl_trigger();
    __shared__ Clip shared_clip;
    if (threadIdx.x < 32) {
        double sum = 0.0;
        for (int i = threadIdx.x; i < a.n_parts; i += 32) sum += a.parts[i];
        sum = warp_sum(sum);
        if (threadIdx.x == 0) {
            const Clip c = clip_of(sum, a.max_norm);
            shared_clip = c;
            if (a.norm && blockIdx.x == 0) {
                a.norm[0] = c.norm;
                a.norm[1] = c.factor;
            }
        }
    }
    __syncthreads();
    const float f = shared_clip.factor, pre = shared_clip.pre, rest = shared_clip.rest;
    if (a.in_place && f == 1.f) return;
    const int chunks = a.first[a.count];
    for (int c = chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const int i = tensor_of(a, c);
        if (a.f32[i])
            chunk_scale<float, PER>(a.t[i], c - a.first[i], pre, rest);
        else
            chunk_scale<__nv_bfloat16, PER>(a.t[i], c - a.first[i], pre, rest);
    }
}

size_t clip_ws_bytes(int count) {
    const size_t launches = count > 0 ? ((size_t)count + kCTensors - 1) / kCTensors : 1;
    return launches * kCParts * sizeof(double);
}

struct ClipCall {
    const void* const* grads;
    void* const* out;
    const long long* sizes;
    const int* dtypes;
    int count;
    float max_norm;
    float* norm;
    double* parts;
};

// Chunks of the tensors [t0, t1), at most.
long long chunks_of(const ClipCall& c, int t0, int t1, int chunk) {
    long long n = 0;
    for (int i = t0; i < t1; ++i) n += (c.sizes[i] + chunk - 1) / chunk + 1;
    return n;
}

// The launches for the tensors [t0, t0 + count): the norm's, or the product's.
template <bool SCALE, int N, int PER>
cudaError_t clip_launch(const ClipCall& c, int t0, int count, double* parts, int* n_parts, float* norm,
                        cudaStream_t st) {
    constexpr int kChunk = kCThreads * PER;
    ClipArgs<N> a;
    a.count = count;
    int chunks = 0;
    for (int i = 0; i < count; ++i) {
        const int k = t0 + i, es = c.dtypes[k] == HCW_F32 ? 4 : 2;
        a.t[i].g = c.grads[k];
        a.t[i].out = c.out ? c.out[k] : const_cast<void*>(c.grads[k]);
        a.t[i].n = c.sizes[k];
        a.f32[i] = c.dtypes[k] == HCW_F32;
        a.first[i] = chunks;
        // the elements before the first boundary come on top of the first chunk's
        const uintptr_t at = reinterpret_cast<uintptr_t>(c.grads[k]);
        const long long head = std::min<long long>((long long)((16 - (at & 15)) & 15) / es, c.sizes[k]);
        const long long body = c.sizes[k] - head;
        chunks += (int)(body > 0 ? (body + kChunk - 1) / kChunk : c.sizes[k] > 0);
    }
    a.first[count] = chunks;
    a.parts = SCALE ? c.parts : parts;
    a.max_norm = c.max_norm;
    a.norm = norm;
    a.in_place = c.out == nullptr;
    const int most = std::min(kCParts, (PER == 64 ? 2 : 4) * device_sms());
    const int grid = std::max(1, std::min(chunks, most));
    if constexpr (SCALE) {
        a.n_parts = *n_parts;
        return launch_pdl(clip_scale_kernel<N, PER>, dim3(grid), dim3(kCThreads), 0, st, a);
    } else {
        *n_parts += grid;
        a.n_parts = 0;
        return launch_pdl(clip_norm_kernel<N, PER>, dim3(grid), dim3(kCThreads), 0, st, a);
    }
}

}  // namespace

}  // namespace hcw

using namespace hcw;

extern "C" size_t hcw_clip_grads_workspace_bytes(int count) {
    return count < 0 ? 0 : clip_ws_bytes(count);
}

extern "C" int hcw_clip_grads(const void* const* grads, void* const* out, const long long* sizes,
                              const int* dtypes, int count, float max_norm, float* norm,
                              void* workspace, size_t ws_bytes, void* stream) {
    if (count < 0 || !norm || !(max_norm >= 0.f)) return HCW_ERR_INVALID_ARG;
    if (count > 0 && (!grads || !sizes || !dtypes)) return HCW_ERR_INVALID_ARG;
    const size_t need = clip_ws_bytes(count);
    // the tensors' spans (inputs, outputs, then norm and workspace): no two share a byte
    struct Span {
        uintptr_t a, b;
        bool out;
    };
    const bool apart = out != nullptr;
    const size_t room = (size_t)count * (apart ? 2 : 1) + 2;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] < 0 || (dtypes[i] != HCW_BF16 && dtypes[i] != HCW_F32)) return HCW_ERR_INVALID_ARG;
        if (!sizes[i]) continue;
        if (!grads[i] || (apart && !out[i])) return HCW_ERR_INVALID_ARG;
        if (sizes[i] > 1ll << 44) return HCW_ERR_UNSUPPORTED;
        const uintptr_t mask = dtypes[i] == HCW_F32 ? 3 : 1;
        if ((reinterpret_cast<uintptr_t>(grads[i]) & mask) ||
            (apart && (reinterpret_cast<uintptr_t>(out[i]) & mask)))
            return HCW_ERR_ALIGNMENT;
    }
    if (!on_16_bytes(workspace) || !on_4_bytes(norm)) return HCW_ERR_ALIGNMENT;
    if (!workspace || ws_bytes < need) return HCW_ERR_WORKSPACE;
    ClipCall c = {grads, out, sizes, dtypes, count, max_norm, norm, static_cast<double*>(workspace)};
    for (int t = 0; t < count; t += kCTensors)
        if (chunks_of(c, t, std::min(count, t + kCTensors), kCThreads * 32) > kCMaxChunks)
            return HCW_ERR_UNSUPPORTED;
    Span few[160];
    Span* s = room <= 160 ? few : new (std::nothrow) Span[room];
    if (!s) return HCW_ERR_UNSUPPORTED;
    size_t k = 0;
    bool sorted = true;
    const auto add = [&](const void* p, size_t bytes, bool o) {
        if (!bytes) return;
        const uintptr_t a = reinterpret_cast<uintptr_t>(p);
        s[k] = {a, a + bytes, o};
        if (k && s[k - 1].a > a) sorted = false;
        ++k;
    };
    for (int i = 0; i < count; ++i) add(grads[i], (size_t)sizes[i] * (dtypes[i] == HCW_F32 ? 4 : 2), !apart);
    if (apart)
        for (int i = 0; i < count; ++i)
            add(out[i], (size_t)sizes[i] * (dtypes[i] == HCW_F32 ? 4 : 2), true);
    add(norm, 8, true);
    add(workspace, need, true);
    if (!sorted) std::sort(s, s + k, [](const Span& x, const Span& y) { return x.a < y.a; });
    // inputs that are only read may share memory
    uintptr_t in_end = 0, out_end = 0;
    bool meet = false;
    for (size_t i = 0; i < k; ++i) {
        if (s[i].a < out_end || (s[i].out && s[i].a < in_end)) meet = true;
        uintptr_t& end = s[i].out ? out_end : in_end;
        if (s[i].b > end) end = s[i].b;
    }
    if (s != few) delete[] s;
    if (meet) return HCW_ERR_ALIASING;

    const cudaStream_t st = (cudaStream_t)stream;
    int launches = 0, n_parts = 0;
    cudaError_t e = cudaSuccess;
    // Chunks of 64 elements a thread for the norm and 32 for the product, which has as many stores to make
    // (950 MB of bf16, whole calls in a graph: 437 us; 456 with 64 for the product, 447 with 32 for the norm);
    // of 8 while the longer ones would leave SMs with fewer than four CTAs (a one-layer student 6.7 us, with
    // long ones 7.4; 17 M fp32 elements 30 with long ones, 44 without.  Between the two the rule comes late:
    // 4.3 and 8.5 M fp32 elements 15.5 and 23.4 us, with long ones 10.7 and 15.6).
    const auto launch = [&](auto scale, int t) {
        constexpr bool kScale = decltype(scale)::value;
        constexpr int kPer = kScale ? 32 : 64;
        const int n = std::min(count - t, kCTensors);
        double* parts = c.parts + n_parts;
        float* to = kScale && t == 0 ? norm : nullptr;
        const bool few = chunks_of(c, t, t + n, kCThreads * 32) < 4ll * device_sms();
        ++launches;
        if (n <= 32)
            return few ? clip_launch<kScale, 32, 8>(c, t, n, parts, &n_parts, to, st)
                       : clip_launch<kScale, 32, kPer>(c, t, n, parts, &n_parts, to, st);
        return few ? clip_launch<kScale, kCTensors, 8>(c, t, n, parts, &n_parts, to, st)
                   : clip_launch<kScale, kCTensors, kPer>(c, t, n, parts, &n_parts, to, st);
    };
    for (int t = 0; e == cudaSuccess && (t == 0 || t < count); t += kCTensors) e = launch(std::false_type(), t);
    // the norm alone: one CTA without tensors writes it
    if (isinf(max_norm) && !apart) c.count = count = 0;
    for (int t = 0; e == cudaSuccess && (t == 0 || t < count); t += kCTensors) e = launch(std::true_type(), t);
    return count_launch(e, launches);
}
