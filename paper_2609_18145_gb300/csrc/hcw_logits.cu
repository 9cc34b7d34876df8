// hcw_logits.cu -- edits of the logits before a symbol is drawn (hcw_logits_edit).  For symbol j
// of row b, with n_j its occurrences in the row's own part of the history and s_j whether it
// occurs anywhere in it:
//
//   z' = s_j ? (z > 0 ? z / r : z r) : z,   z'' = z' - f n_j - p [n_j > 0] + its slots' biases,
//   out = z'' where the mask lets j through, else -inf
//
// Bound by memory: the logits are read and written once.
//
// Few logits: one launch, in which a CTA takes a slice of a row's symbols with a counter for each in
// shared memory.  Many: the whole rows first, with the mask alone; then, a CTA a row, the few symbols
// that the history or a slot names, from a table of them.  Occurrences are whole numbers, for which
// the order of the atomics does not matter; biases are added in the order of their slots, by the thread
// of the symbol's first one.
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
constexpr uint32_t kMore = 1u << 30;  // in a named symbol's: has more than one slot

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

// f(symbol, t) for the history's entries from `from` on, eight of a thread's on their way at once.
template <int NT, typename F>
__device__ __forceinline__ void rest_of_history(const int* h, int from, int n, F f) {
    for (long long t0 = from + (int)threadIdx.x; t0 < n; t0 += 8 * NT) {
        int v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = t0 + i * NT < n ? h[t0 + i * NT] : -1;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (t0 + i * NT < n) f(v[i], (int)t0 + i * NT);
    }
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

// ------------------------------------------------------------------ one launch
// A slice of 256 vectors of 16 bytes, from the boundary at or before the row's start, for a CTA of as
// many threads.  What it needs is asked for at once, before the counters are cleared: its logits, its
// words of the mask, the first 1024 symbols of the history, the first 256 slots.  Bound by latency: a
// launch, one round of loads, three barriers (1 x 201 fp32 2.4 us, 8 x 131072 bf16 3.9).
template <typename T>
__global__ void __launch_bounds__(256) logits_edit_kernel(const LogitsArgs a) {
    constexpr int NT = 256, NH = 4, VE = 16 / sizeof(T), S = NT * VE;
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
    const int* h = a.history ? a.history + (size_t)row * a.H : nullptr;
    int past[NH];
    if (h) {   // (no condition at a load: those wait one for another; entries past n are not looked at)
#pragma unroll
        for (int i = 0; i < NH; ++i) past[i] = h[min((int)threadIdx.x + i * NT, a.H - 1)];
    }
    const int n = !h ? 0 : a.lengths ? min(max(a.lengths[row], 0), a.H) : a.H;
    const int own = a.prompt ? a.prompt[row] : 0;
    int id = -1;
    float id_bias = 0.f;
    if ((int)threadIdx.x < a.M) {
        id = a.bias_idx[(size_t)row * a.M + threadIdx.x];
        id_bias = a.bias[(size_t)row * a.M + threadIdx.x];
    }
    Penalty pen;
    pen.rep = a.rep ? a.rep[row] : 1.f;
    pen.freq = a.freq ? a.freq[row] : 0.f;
    pen.pres = a.pres ? a.pres[row] : 0.f;
    // the slice's vectors and their bits of the mask; vectors over an end of the row come one by
    // one later
    const uint32_t* mask = a.mask ? a.mask + (size_t)row * ((a.V + 31) / 32) : nullptr;
    const long long jl = (long long)j0 + threadIdx.x * VE;
    const bool inside = jl >= 0 && jl + VE <= a.V;
    uint4 q = make_uint4(0, 0, 0, 0);
    uint32_t bits = 0xffffffffu;
    if (inside) {
        if (!a.lazy) q = *reinterpret_cast<const uint4*>(z + jl);
        if (mask) {
            const int at = (int)jl & 31;
            bits = mask[jl >> 5] >> at;
            if (at + VE > 32) bits |= mask[(jl >> 5) + 1] << (32 - at);
        }
    }
    for (int i = threadIdx.x * 4; i < S; i += NT * 4)
        *reinterpret_cast<uint4*>(count + i) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const auto mark = [&](int symbol, int t) {
        if (symbol >= a.V) atomicExch(&g_error_word, kErrInvalid);
        if (symbol < lo || symbol >= hi) return;
        if (t < own)
            atomicOr(&count[symbol - j0], kSeen);
        else
            atomicAdd(&count[symbol - j0], 1u);
    };
#pragma unroll
    for (int i = 0; i < NH; ++i)
        if ((int)threadIdx.x + i * NT < n) mark(past[i], threadIdx.x + i * NT);
    rest_of_history<NT>(h, NH * NT, n, mark);
    // the slice's slots, in their order
    int slots = 0;
    for (int k0 = 0; k0 < a.M; k0 += NT) {
        if (k0) {
            const int k = k0 + threadIdx.x;
            id = k < a.M ? a.bias_idx[(size_t)row * a.M + k] : -1;
            id_bias = k < a.M ? a.bias[(size_t)row * a.M + k] : 0.f;
        }
        if (id >= a.V) atomicExch(&g_error_word, kErrInvalid);
        const bool here = id >= lo && id < hi;
        const uint32_t some = __ballot_sync(0xffffffffu, here);
        if (lane == 0) found[warp] = __popc(some);
        __syncthreads();
        int at = slots;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) {
            if (w < warp) at += found[w];
            slots += found[w];
        }
        if (here) {
            at += __popc(some & ((1u << lane) - 1));
            slot_id[at] = id;
            slot_bias[at] = id_bias;
        }
        __syncthreads();
    }
    if (!a.M) __syncthreads();
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
        const int symbol = slot_id[k];
        float sum = 0.f;
        bool first = true;
        for (int m = 0; m < slots; ++m) {
            if (slot_id[m] != symbol) continue;
            if (m < k) {
                first = false;
                break;
            }
            sum += slot_bias[m];
        }
        if (!first || !passes(symbol)) continue;
        again_at[i] = symbol;
        again[i] = pen(value(z + symbol), count[symbol - j0]) + sum;
    }
    if (a.M && z == out) __syncthreads();   // before the logits are written over
    if (jl + VE > lo && jl < hi) {
        const int at = threadIdx.x * VE, j = (int)jl;
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
        if (a.lazy && !any) {
        } else if (inside) {
            if (a.lazy) q = *reinterpret_cast<const uint4*>(z + j);
            float v[VE];
            unpack<VE>(q, v);
            if (any) {
#pragma unroll
                for (int e = 0; e < VE; ++e) v[e] = pen(v[e], c[e]);
            }
#pragma unroll
            for (int e = 0; e < VE; ++e)
                if (!(bits >> e & 1)) v[e] = -INFINITY;
            *reinterpret_cast<uint4*>(out + j) = pack<VE>(v);
        } else {
            for (int e = 0; e < VE; ++e) {
                if (j + e < 0 || j + e >= a.V) continue;
                put(out + j + e, passes(j + e) ? pen(value(z + j + e), c[e]) : -INFINITY);
            }
        }
    }
    if (!a.M) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SL; ++i)
        if (again_at[i] >= 0) put(out + again_at[i], again[i]);
}

// ------------------------------------------------------------------ two launches
// The whole row first: logits and mask, four vectors a thread.  A vector that the mask takes out
// entirely is not read; in place one that it lets through entirely is not touched.  Bound by memory:
// 256 x 131072 fp32 without a mask 40 us, 6.7 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) logits_mask_kernel(const LogitsArgs a) {
    constexpr int VE = 16 / sizeof(T), NV = 4;
    constexpr uint32_t kAll = (1u << VE) - 1;
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    const size_t start = (size_t)row * a.V;
    const int phase = (int)(start % VE);
    const T* z = static_cast<const T*>(a.z) + start;
    T* out = static_cast<T*>(a.out) + start;
    const uint32_t* mask = a.mask ? a.mask + (size_t)row * ((a.V + 31) / 32) : nullptr;
    const bool apart = a.z != a.out;
    const int j0 = (slice * NV * 256 + threadIdx.x) * VE - phase;
    uint32_t bits[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = j0 + i * 256 * VE;
        bits[i] = kAll;
        if (!mask || j + VE <= 0 || j >= a.V) continue;
        // the words of the vector's first and last symbol (the same one, unless it lies over a
        // word's end)
        const int f = max(j, 0), l = min(j + VE, a.V) - 1;
        const uint32_t u = mask[f >> 5], w = mask[l >> 5];
        bits[i] = __funnelshift_r(u, w, f & 31) << (f - j) & kAll;
    }
    uint4 q[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = j0 + i * 256 * VE;
        q[i] = make_uint4(0, 0, 0, 0);
        if (j >= 0 && j + VE <= a.V && bits[i] && (apart || bits[i] != kAll))
            q[i] = *reinterpret_cast<const uint4*>(z + j);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = j0 + i * 256 * VE;
        if (j + VE <= 0 || j >= a.V || (!apart && bits[i] == kAll)) continue;
        if (j >= 0 && j + VE <= a.V) {
            if (bits[i] != kAll) {
                constexpr uint32_t kOff = sizeof(T) == 2 ? 0xff80u : 0xff800000u;   // -inf
                uint32_t* const w = &q[i].x;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    if (bits[i] >> e & 1) continue;
                    if constexpr (sizeof(T) == 2)
                        w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | kOff << 16 : (w[e / 2] & 0xffff0000u) | kOff;
                    else
                        w[e] = kOff;
                }
            }
            *reinterpret_cast<uint4*>(out + j) = q[i];
        } else {
            for (int e = 0; e < VE; ++e) {
                if (j + e < 0 || j + e >= a.V) continue;
                if (bits[i] >> e & 1)
                    out[j + e] = z[j + e];
                else
                    put(out + j + e, -INFINITY);
            }
        }
    }
}

// Then the symbols that the history or a slot names, a CTA a row: a table of them in shared memory
// (open addressing), with each one's occurrences and first
// slot.  Which place a symbol gets depends on the order of the threads, what is found there does not.
// Where a row has more names than the table takes (HASH false) the table is indexed by the symbol,
// and CTAs share a row's symbols in ranges of kLRange.
// The table is cleared while the launch before may still be under way; everything else waits for it:
// what lies before that launch has ended by then, but only the wait makes its memory visible here.
constexpr int kLRange = 8192;
constexpr int kLNames = 4096;         // of a row's history, for the hashed table
constexpr int kLPlaces = 8192;        // of that table: five eighths of them taken at most
constexpr int kNoSlot = 0x7fffffff;

template <typename T, bool HASH, int NT>
__global__ void __launch_bounds__(NT) logits_named_kernel(const LogitsArgs a, int size) {
    constexpr int NH = kLNames / NT, NS = kLMaxSlots / NT;   // names a thread
    extern __shared__ __align__(16) int table[];   // [size]: counts, first slots, symbols
    uint32_t* const count = reinterpret_cast<uint32_t*>(table);
    int* const low = table + size;
    int* const key = table + 2 * size;             // HASH
    for (int i = threadIdx.x; i < size / 4; i += NT) {
        reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
        reinterpret_cast<int4*>(low)[i] = make_int4(kNoSlot, kNoSlot, kNoSlot, kNoSlot);
        if (HASH) reinterpret_cast<int4*>(key)[i] = make_int4(-1, -1, -1, -1);
    }
    pdl_wait();
    pdl_trigger();
    const int row = HASH ? blockIdx.x : blockIdx.x / a.slices;
    const int lo = HASH ? 0 : blockIdx.x % a.slices * kLRange;
    const int hi = HASH ? a.V : min(a.V, lo + kLRange);
    const T* z = static_cast<const T*>(a.z) + (size_t)row * a.V;
    T* out = static_cast<T*>(a.out) + (size_t)row * a.V;
    const int* h = a.history ? a.history + (size_t)row * a.H : nullptr;
    const int* bias_idx = a.bias_idx + (size_t)row * a.M;
    const float* bias = a.bias + (size_t)row * a.M;
    const uint32_t* mask = a.mask ? a.mask + (size_t)row * ((a.V + 31) / 32) : nullptr;
    // everything asked for at once
    // (no condition at a load: those wait one for another)
    int past[NH], slot[NS];
#pragma unroll
    for (int i = 0; i < NH; ++i) past[i] = h ? h[min((int)threadIdx.x + i * NT, a.H - 1)] : -1;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int k = threadIdx.x + i * NT;
        slot[i] = a.M ? bias_idx[min(k, a.M - 1)] : -1;
        if (k >= a.M) slot[i] = -1;
    }
    const int n = !h ? 0 : a.lengths ? min(max(a.lengths[row], 0), a.H) : a.H;
    const int own = a.prompt ? a.prompt[row] : 0;
    Penalty pen;
    pen.rep = a.rep ? a.rep[row] : 1.f;
    pen.freq = a.freq ? a.freq[row] : 0.f;
    pen.pres = a.pres ? a.pres[row] : 0.f;
    __syncthreads();
    // the symbol's place (made if it has none), or -1
    const auto place = [&](int symbol) {
        if (symbol >= a.V) atomicExch(&g_error_word, kErrInvalid);
        if (symbol < lo || symbol >= hi) return -1;
        if (!HASH) return symbol - lo;
        int p = (int)(((uint32_t)symbol * 2654435761u) >> 8) & (size - 1);
        for (;;) {
            int was = *(volatile int*)&key[p];
            if (was == -1) was = atomicCAS(&key[p], -1, symbol);
            if (was == -1 || was == symbol) return p;
            p = (p + 1) & (size - 1);
        }
    };
    const auto mark = [&](int p, int t) {
        if (t < own)
            atomicOr(&count[p], kSeen);
        else
            atomicAdd(&count[p], 1u);
    };
#pragma unroll
    for (int i = 0; i < NH; ++i) {
        const int t = threadIdx.x + i * NT;
        past[i] = t < n ? place(past[i]) : -1;
        if (past[i] >= 0) mark(past[i], t);
    }
    if (!HASH)
        rest_of_history<NT>(h, kLNames, n, [&](int symbol, int t) {
            const int p = place(symbol);
            if (p >= 0) mark(p, t);
        });
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int symbol = slot[i];
        slot[i] = symbol >= 0 ? place(symbol) : -1;
        if (slot[i] >= 0) atomicMin(&low[slot[i]], (int)threadIdx.x + i * NT);
    }
    __syncthreads();
    if (a.M) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (slot[i] >= 0 && low[slot[i]] != (int)threadIdx.x + i * NT)
                atomicOr(&count[slot[i]], kMore);
        __syncthreads();
    }
    // What will be written: a symbol without slots by whoever takes its count first, one with slots
    // by the first of them, with the sum over all in their order.
    const auto passes = [&](int j) { return !mask || (mask[j >> 5] >> (j & 31) & 1); };
    const auto taken = [&](int p, uint32_t* c) {
        *c = p >= 0 && low[p] == kNoSlot ? atomicExch(&count[p], 0u) : 0u;
        return !*c ? -1 : HASH ? key[p] : lo + p;
    };
    uint32_t c[NH], sc[NS];
    int at[NS];
    float v[NH], sv[NS], sum[NS];
#pragma unroll
    for (int i = 0; i < NH; ++i) past[i] = taken(past[i], &c[i]);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int p = slot[i];
        at[i] = -1;
        if (p < 0 || low[p] != (int)threadIdx.x + i * NT) continue;
        at[i] = HASH ? key[p] : lo + p;
        sc[i] = count[p];
    }
#pragma unroll
    for (int i = 0; i < NH; ++i) v[i] = value(z + max(past[i], 0));
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        sum[i] = a.M ? bias[min((int)threadIdx.x + i * NT, a.M - 1)] : 0.f;
        sv[i] = value(z + max(at[i], 0));
    }
    if (mask) {
        uint32_t w[NH], sw[NS];
#pragma unroll
        for (int i = 0; i < NH; ++i) w[i] = mask[max(past[i], 0) >> 5];
#pragma unroll
        for (int i = 0; i < NS; ++i) sw[i] = mask[max(at[i], 0) >> 5];
#pragma unroll
        for (int i = 0; i < NH; ++i)
            if (!(w[i] >> (past[i] & 31) & 1)) past[i] = -1;
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (!(sw[i] >> (at[i] & 31) & 1)) at[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        if (at[i] < 0 || !(sc[i] & kMore)) continue;
        for (int m = threadIdx.x + i * NT + 1; m < a.M; ++m)
            if (bias_idx[m] == at[i]) sum[i] += bias[m];
    }
#pragma unroll
    for (int i = 0; i < NH; ++i)
        if (past[i] >= 0) put(out + past[i], pen(v[i], c[i]));
#pragma unroll
    for (int i = 0; i < NS; ++i)
        if (at[i] >= 0) put(out + at[i], pen(sv[i], sc[i] & ~kMore) + sum[i]);
    if (!HASH)
        rest_of_history<NT>(h, kLNames, n, [&](int symbol, int) {
            uint32_t m;
            const int j = symbol >= lo && symbol < hi ? taken(symbol - lo, &m) : -1;
            if (j >= 0 && passes(j)) put(out + j, pen(value(z + j), m));
        });
}

template <typename T, bool HASH, int NT>
cudaError_t launch_named(const LogitsArgs& a, long long ctas, int size, cudaStream_t st) {
    auto kern = logits_named_kernel<T, HASH, NT>;
    static std::once_flag once[64];
    static cudaError_t set_err[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::call_once(once[dev], [&] {
        set_err[dev] = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                            HASH ? kLPlaces * 12 : kLRange * 8);
    });
    if (set_err[dev] != cudaSuccess) return set_err[dev];
    return launch_pdl(kern, dim3((unsigned)ctas), dim3(NT), (size_t)size * (HASH ? 12 : 8), st, a, size);
}

// One launch up to 2.5 MB of logits, where it is the shorter wait (1 x 201 2.5 us against 4.0 in two, 8 x
// 131072 bf16 3.9 against 5.2, 16 x 65536 5.1 against 7.1); above, its slices would each go through the
// history (64 x 32003 bf16 8.4 against 7.9, 256 x 32003 21 against 13, 256 x 131072 fp32 207 against 51).
// The named symbols' CTAs have 1024 threads while there are no more of them than SMs (64 x 32003 7.8 us
// against 10.8 with 512; 256 x 32003 13.4 against 12.7).  Times of a call in a graph.
template <typename T>
cudaError_t edit(LogitsArgs& a, cudaStream_t st, int* launches) {
    constexpr int VE = 16 / sizeof(T);
    const long long bytes = (long long)a.B * a.V * sizeof(T), sms = device_sms();
    *launches = 0;
    // (a row may start anywhere between two boundaries)
    if (bytes <= sms * 4 * 256 * 16) {
        a.slices = (int)(((long long)a.V + VE - 1 + 256 * VE - 1) / (256 * VE));
        ++*launches;
        return launch_pdl(logits_edit_kernel<T>, dim3((unsigned)((long long)a.B * a.slices)), dim3(256),
                          (size_t)256 * VE * 4, st, a);
    }
    const bool whole = a.z != a.out || a.mask;
    if (whole) {
        a.slices = (int)(((long long)a.V + VE - 1 + 1024 * VE - 1) / (1024 * VE));
        const cudaError_t e = launch_pdl(logits_mask_kernel<T>, dim3((unsigned)((long long)a.B * a.slices)),
                                         dim3(256), 0, st, a);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    const int names = (a.history ? a.H : 0) + a.M;
    if (!names) return cudaSuccess;
    ++*launches;
    if ((a.history && a.H > kLNames) || a.V <= kLRange) {
        a.slices = (a.V + kLRange - 1) / kLRange;
        const long long ctas = (long long)a.B * a.slices;
        const int size = std::min((a.V + 3) / 4 * 4, kLRange);
        return ctas <= sms ? launch_named<T, false, 1024>(a, ctas, size, st)
                           : launch_named<T, false, 512>(a, ctas, size, st);
    }
    int size = 256;
    while (5 * size < 8 * names) size *= 2;
    return a.B <= sms ? launch_named<T, true, 1024>(a, a.B, size, st)
                      : launch_named<T, true, 512>(a, a.B, size, st);
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
    const void* all[] = {history, lengths, prompt, repetition, frequency, presence, bias_idx, bias, mask};
    for (const void* p : all)
        if (!on_4_bytes(p)) return HCW_ERR_ALIGNMENT;
    if (!on_16_bytes(z) || !on_16_bytes(out)) return HCW_ERR_ALIGNMENT;
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
    int launches = 0;
    const cudaError_t e =
        dtype == HCW_BF16 ? edit<__nv_bfloat16>(a, st, &launches) : edit<float>(a, st, &launches);
    return count_launch(e, launches);
}
