// hcw_logits.cu -- edits of the logits before a symbol is drawn (hcw_logits_edit).  For symbol j
// of row b, with n_j its occurrences in the row's own part of the history and s_j whether it
// occurs anywhere in it:
//
//   z' = s_j ? (z > 0 ? z / r : z r) : z,   z'' = z' - f n_j - p [n_j > 0] + its slots' biases,
//   out = z'' where the mask lets j through, else -inf
//
// Bound by memory: the logits are read and written once.  One launch; a CTA takes a slice of a
// row's symbols, with a counter for each of them in shared memory.  Its logits are already on
// their way while it goes through the row's history and counts the symbols of its slice (whole
// numbers: the order of the atomics does not matter).  The biases are few and may name a symbol
// more than once: they are collected in the order of their slots, and the first slot of each symbol
// writes the symbol again when the rest of the slice is out, with the sum over its slots.
#include "hcw.h"
#include "hcw_internal.h"
#include "hcw_ptx.cuh"

#include <math.h>

#include <algorithm>
#include <mutex>

namespace hcw {

namespace {

constexpr int kErrInvalid = 1;        // HCW_ERR_INVALID_ARG in the error word
constexpr int kLMaxSlots = 1024;      // biases of a row
constexpr uint32_t kSeen = 1u << 31;  // in a counter: occurs in the prompt

struct LogitsArgs {
    const void* z;
    void* out;
    const int* history;      // [B][H] or null
    const int* lengths;      // [B] or null (H)
    const int* prompt;       // [B] or null (0)
    const float* rep;        // [B] or null (1)
    const float* freq;       // [B] or null (0)
    const float* pres;       // [B] or null (0)
    const int* bias_idx;     // [B][M] or null
    const float* bias;       // [B][M]
    const uint32_t* mask;    // [B][ceil(V / 32)] or null
    int B, V, H, M;
    int slices;              // of a row
    int lazy;                // in place, without a mask: only what changes is read and written
};

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

template <int VE>
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[VE]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (VE == 8) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            v[i] = __uint_as_float(w[i]);
        }
    }
}
template <int VE>
__device__ __forceinline__ uint4 pack(const float (&v)[VE]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (VE == 8)
            w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        else
            w[i] = __float_as_uint(v[i]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Penalty {
    float rep, freq, pres;
    __device__ __forceinline__ float operator()(float z, uint32_t c) const {
        if (!c) return z;
        const float n = (float)(c & ~kSeen);
        z = z > 0.f ? z / rep : z * rep;
        return z - freq * n - (n > 0.f ? pres : 0.f);
    }
};

// NT threads, NV vectors of 16 bytes each: a slice of NT NV vectors, from the boundary at or
// before the row's start.
template <typename T, int NT, int NV>
__global__ void __launch_bounds__(NT) logits_edit_kernel(const LogitsArgs a) {
    constexpr int VE = 16 / sizeof(T), S = NT * NV * VE;
    extern __shared__ __align__(16) uint32_t count[];   // [S]
    __shared__ int slot_id[kLMaxSlots];
    __shared__ float slot_bias[kLMaxSlots];
    __shared__ int found[NT / 32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const size_t start = (size_t)row * a.V;
    const int phase = (int)(start % VE);
    const T* z = static_cast<const T*>(a.z) + start;
    T* out = static_cast<T*>(a.out) + start;
    const int j0 = slice * S - phase;                    // the symbol of the slice's first place
    const int lo = max(j0, 0), hi = (int)min((long long)a.V, (long long)j0 + S);
    // the slice's vectors; those over an end of the row one by one
    uint4 q[NV];
    if (!a.lazy) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const long long j = (long long)j0 + (threadIdx.x + i * NT) * VE;
            q[i] = make_uint4(0, 0, 0, 0);
            if (j >= 0 && j + VE <= a.V) q[i] = *reinterpret_cast<const uint4*>(z + j);
        }
    }
    Penalty pen;
    pen.rep = a.rep ? a.rep[row] : 1.f;
    pen.freq = a.freq ? a.freq[row] : 0.f;
    pen.pres = a.pres ? a.pres[row] : 0.f;
    for (int i = threadIdx.x * 4; i < S; i += NT * 4)
        *reinterpret_cast<uint4*>(count + i) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    // the history
    if (a.history) {
        const int* h = a.history + (size_t)row * a.H;
        const int n = a.lengths ? min(max(a.lengths[row], 0), a.H) : a.H;
        const int own = a.prompt ? a.prompt[row] : 0;
        for (int t = threadIdx.x; t < n; t += NT) {
            const int id = h[t];
            if (id >= a.V) atomicExch(&g_error_word, kErrInvalid);
            if (id < lo || id >= hi) continue;
            if (t < own)
                atomicOr(&count[id - j0], kSeen);
            else
                atomicAdd(&count[id - j0], 1u);
        }
    }
    // the slice's biases, in the order of their slots
    int slots = 0;
    if (a.bias_idx) {
        for (int k0 = 0; k0 < a.M; k0 += NT) {
            const int k = k0 + threadIdx.x;
            const int id = k < a.M ? a.bias_idx[(size_t)row * a.M + k] : -1;
            if (id >= a.V) atomicExch(&g_error_word, kErrInvalid);
            const bool here = id >= lo && id < hi;
            const uint32_t some = __ballot_sync(0xffffffffu, here);
            if (lane == 0) found[warp] = __popc(some);
            __syncthreads();
            int at = slots, all = slots;
            for (int w = 0; w < NT / 32; ++w) {
                if (w < warp) at += found[w];
                all += found[w];
            }
            if (here) {
                at += __popc(some & ((1u << lane) - 1));
                slot_id[at] = id;
                slot_bias[at] = a.bias[(size_t)row * a.M + k];
            }
            slots = all;
            __syncthreads();
        }
    } else {
        __syncthreads();
    }
    const uint32_t* mask = a.mask ? a.mask + (size_t)row * ((a.V + 31) / 32) : nullptr;
    const auto passes = [&](int j) { return !mask || (mask[j >> 5] >> (j & 31) & 1); };
    // what the first slot of a symbol will write: its logit as it was, and its slots' sum
    constexpr int SL = (kLMaxSlots + NT - 1) / NT;
    float again[SL];
    int again_at[SL];
#pragma unroll
    for (int i = 0; i < SL; ++i) {
        const int k = threadIdx.x + i * NT;
        again_at[i] = -1;
        if (k >= slots) continue;
        const int id = slot_id[k];
        float sum = 0.f;
        bool first = true;
        for (int m = 0; m < slots; ++m) {
            if (slot_id[m] != id) continue;
            if (m < k) {
                first = false;
                break;
            }
            sum += slot_bias[m];
        }
        if (!first || !passes(id)) continue;
        again_at[i] = id;
        again[i] = pen(value(z + id), count[id - j0]) + sum;
    }
    if (a.bias_idx && z == out) __syncthreads();   // before the logits are written over
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = (threadIdx.x + i * NT) * VE;
        const long long jl = (long long)j0 + at;
        if (jl + VE <= lo || jl >= hi) continue;
        const int j = (int)jl;
        uint32_t c[VE], any = 0;
#pragma unroll
        for (int e = 0; e < VE; e += 4) {
            const uint4 p = *reinterpret_cast<const uint4*>(count + at + e);
            c[e] = p.x;
            c[e + 1] = p.y;
            c[e + 2] = p.z;
            c[e + 3] = p.w;
            any |= p.x | p.y | p.z | p.w;
        }
        if (a.lazy && !any) continue;
        if (j >= 0 && j + VE <= a.V) {
            if (a.lazy) q[i] = *reinterpret_cast<const uint4*>(z + j);
            float v[VE];
            unpack<VE>(q[i], v);
            if (any) {
#pragma unroll
                for (int e = 0; e < VE; ++e) v[e] = pen(v[e], c[e]);
            }
            if (mask) {
                uint32_t w = mask[j >> 5] >> (j & 31);
                if ((j & 31) + VE > 32) w |= mask[(j >> 5) + 1] << (32 - (j & 31));
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    if (!(w >> e & 1)) v[e] = -INFINITY;
            }
            *reinterpret_cast<uint4*>(out + j) = pack<VE>(v);
        } else {
            for (int e = 0; e < VE; ++e) {
                if (j + e < 0 || j + e >= a.V) continue;
                put(out + j + e, passes(j + e) ? pen(value(z + j + e), c[e]) : -INFINITY);
            }
        }
    }
    if (!a.bias_idx) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SL; ++i)
        if (again_at[i] >= 0) put(out + again_at[i], again[i]);
}

template <typename T, int NT, int NV>
cudaError_t launch_edit(LogitsArgs& a, cudaStream_t st) {
    constexpr int VE = 16 / sizeof(T), S = NT * NV * VE;
    auto kern = logits_edit_kernel<T, NT, NV>;
    if (S * 4 > 32768) {
        static std::once_flag once[64];
        static cudaError_t set_err[64];
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
        std::call_once(once[dev], [&] {
            set_err[dev] = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S * 4);
        });
        if (set_err[dev] != cudaSuccess) return set_err[dev];
    }
    // a row may start anywhere between two boundaries
    a.slices = (int)(((long long)a.V + VE - 1 + S - 1) / S);
    return launch_pdl(kern, dim3((unsigned)((long long)a.B * a.slices)), dim3(NT), S * 4, st, a);
}

// The slice: as large as leaves every SM a CTA or two, since each CTA goes through the whole history.
template <typename T>
cudaError_t edit(LogitsArgs& a, cudaStream_t st) {
    const long long bytes = (long long)a.B * a.V * sizeof(T), sms = device_sms();
    if (bytes <= sms * 2 * 128 * 16) return launch_edit<T, 128, 1>(a, st);
    if (bytes <= sms * 2 * 256 * 2 * 16) return launch_edit<T, 256, 2>(a, st);
    if constexpr (sizeof(T) == 4) {
        return launch_edit<T, 512, 8>(a, st);
    } else {
        return launch_edit<T, 512, 4>(a, st);
    }
}

}  // namespace

cudaError_t logits_error_word_read_clear(int* word) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(word, g_error_word, sizeof(int));
    if (e == cudaSuccess && *word) e = cudaMemcpyToSymbol(g_error_word, &zero, sizeof(int));
    return e;
}

}  // namespace hcw

using namespace hcw;

extern "C" int hcw_logits_edit(const void* z, int B, int V, int dtype, const int* history,
                               const int* lengths, const int* prompt, int H, const float* repetition,
                               const float* frequency, const float* presence, const int* bias_idx,
                               const float* bias, int M, const unsigned* mask, void* out,
                               void* stream) {
    if (B < 0 || V < 1 || H < 0 || M < 0 || (dtype != HCW_BF16 && dtype != HCW_F32))
        return HCW_ERR_INVALID_ARG;
    if (V > 1 << 24 || B > 1 << 20 || H > 1 << 28 || M > kLMaxSlots || (long long)B * V > 1ll << 40)
        return HCW_ERR_UNSUPPORTED;
    const void* all[] = {z, history, lengths, prompt, repetition, frequency, presence, bias_idx,
                         bias, mask, out};
    for (const void* p : all)
        if (!on_16_bytes(p)) return HCW_ERR_ALIGNMENT;
    const size_t zb = (size_t)B * V * (dtype == HCW_F32 ? 4 : 2), b4 = (size_t)B * 4;
    const struct {
        const void* p;
        size_t n;
    } in[] = {{history, b4 * H}, {lengths, b4}, {prompt, b4}, {repetition, b4}, {frequency, b4},
              {presence, b4}, {bias_idx, b4 * M}, {bias, b4 * M}, {mask, b4 * ((V + 31) / 32)}};
    for (const auto& q : in)
        if (spans_meet(out, zb, q.p, q.n)) return HCW_ERR_ALIASING;
    if (out != z && spans_meet(out, zb, z, zb)) return HCW_ERR_ALIASING;
    if (B == 0) return HCW_OK;
    if (!z || !out || (H > 0) != (history != nullptr) || (M > 0) != (bias_idx != nullptr) ||
        (bias_idx != nullptr) != (bias != nullptr) || (!history && (lengths || prompt)))
        return HCW_ERR_INVALID_ARG;
    LogitsArgs a = {};
    a.z = z;
    a.out = out;
    // without a penalty the history changes nothing
    a.history = repetition || frequency || presence ? history : nullptr;
    a.lengths = lengths;
    a.prompt = prompt;
    a.rep = repetition;
    a.freq = frequency;
    a.pres = presence;
    a.bias_idx = bias_idx;
    a.bias = bias;
    a.mask = mask;
    a.B = B;
    a.V = V;
    a.H = H;
    a.M = M;
    a.lazy = z == out && !mask;
    const cudaStream_t st = (cudaStream_t)stream;
    return count_launch(dtype == HCW_BF16 ? edit<__nv_bfloat16>(a, st) : edit<float>(a, st), 1);
}
