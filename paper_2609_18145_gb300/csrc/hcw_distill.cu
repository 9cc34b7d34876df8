// hcw_distill.cu -- distillation from a teacher's top logits, loss and gradient in one
// pass over the student's logits (hcw_distill_loss).  Per row, with M the row's maximum:
//
//   p = softmax over the given slots of t / tau        (the teacher, K slots)
//   q = softmax(z / tau),  q1 = softmax(z)             (the student, V symbols)
//   loss = w [ a tau^2 sum_k p_k (log p_k - log q_{i_k}) + b (log sum exp(z) - z_y) ]
//   dz_j = w [ a tau (P q_j - sum_{k: i_k = j} p_k) + b (q1_j - [j = y]) ]
//
// (P = 1, or 0 for a row without slots).  Bound by memory: the logits are read once and
// the gradient is written once, 4 bytes a symbol in bf16.  A row stays on chip between
// its sums and its gradient: rows of a few thousand symbols in the registers of 1 to 8 warps,
// longer ones in the shared memory of a cluster of up to 8 CTAs, each summing its slice against its own
// maximum, the parts joined through distributed shared memory.  The dense part
// of the gradient goes out first; then the symbols that the teacher or the label names
// are written again with their share taken off, each by the one thread that owns the
// symbol's first slot, so nothing depends on the order of atomics and every output is
// rounded once, from fp32.
//
// A row starts anywhere (V may be odd): its first and last 16-byte vectors may hold symbols
// of its neighbours, which are masked when read and left alone when written.
#include "hcw.h"
#include "hcw_internal.h"
#include "hcw_ptx.cuh"

#include <math.h>
#include <mutex>

namespace hcw {

namespace {

constexpr int kDMaxK = 1024;          // slots of a row
constexpr int kDMaxV = 262144;        // 8 CTAs x 128 KB of fp32 logits
constexpr size_t kDSmem = 232448;     // shared memory of an SM
constexpr long long kDSlice = 65536;  // bytes of a row a CTA takes by choice
constexpr int kDWarpV = 8192;         // rows in registers up to here (bf16: half as many),
constexpr int kDWarpK = 64;           // and up to this many slots
constexpr int kDWarps = 8;            // warps of a CTA of the kernel for rows in registers
constexpr int kErrInvalid = 1;        // HCW_ERR_INVALID_ARG in the error word

struct DistillArgs {
    const void* z;
    const int* idx;         // [T][K] or null
    const float* teacher;   // [T][K]
    const int* target;      // [T] or null
    const float* weight;    // [T] or null (ones)
    float* loss;            // [T] or null
    void* dz;               // [T][V] or null
    int T, V, K;
    float inv_tau;          // 1 / tau
    float kl, ce;           // a tau^2 and b
    float kl_tau;           // a tau
};

constexpr float kLog2e = 1.4426950408889634f;

// The exponentials of a symbol: one (a single temperature in use), one at each of two
// temperatures, or, where the teacher's is 2, the one at temperature 1 as the square of the
// other.
enum DistillExps { kOne = 0, kTwo = 1, kSquare = 2 };

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A running maximum and the sums of exp((z - m) / tau) and exp(z - m) under it.
struct Stat {
    float m, s, s1;
};

// m as the subtrahend of the exponents: 0 for a part without any symbol, whose logits are
// all -inf (exp2(-inf - 0) = 0, where -inf - -inf would be NaN).
__device__ __forceinline__ float stat_base(float m) { return m == -INFINITY ? 0.f : m; }

template <int EXPS>
__device__ __forceinline__ Stat stat_join(const Stat& x, const Stat& y, float c) {
    Stat r;
    r.m = fmaxf(x.m, y.m);
    const float b = stat_base(r.m);
    const float dx = x.m == -INFINITY ? -INFINITY : x.m - b, dy = y.m == -INFINITY ? -INFINITY : y.m - b;
    // a part without symbols has no sum; one with NaN keeps it
    const float fx = ex2(dx * c), fy = ex2(dy * c);
    r.s = (x.m == -INFINITY ? x.s : x.s * fx) + (y.m == -INFINITY ? y.s : y.s * fy);
    if (EXPS != kOne) {
        const float gx = ex2(dx * kLog2e), gy = ex2(dy * kLog2e);
        r.s1 = (x.m == -INFINITY ? x.s1 : x.s1 * gx) + (y.m == -INFINITY ? y.s1 : y.s1 * gy);
    } else {
        r.s1 = r.s;
    }
    return r;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// The lanes' parts joined, on every lane: the maximum first, then one exponential a lane.
template <int EXPS>
__device__ __forceinline__ Stat stat_warp(Stat v, float c) {
    Stat r;
    r.m = warp_max(v.m);
    // a part without symbols has no sum (one with NaN keeps it)
    const float d = v.m == -INFINITY ? 0.f : v.m - stat_base(r.m);
    r.s = warp_sum(v.s * ex2(d * c));
    r.s1 = EXPS != kOne ? warp_sum(v.s1 * ex2(d * kLog2e)) : r.s;
    return r;
}

template <typename T>
__device__ __forceinline__ float logit(const T* p);
template <>
__device__ __forceinline__ float logit(const float* p) { return *p; }
template <>
__device__ __forceinline__ float logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The row's slots, in the caller's shared arrays: p[k] (0 for an empty slot), the symbol
// id[k] (-1), own[k]: the slots' sum for the symbol where slot k is its first one, else -1, and
// zk[k], the symbol's logit.  An index at or past V is reported and counts as empty.
struct Slots {
    float *p, *own, *zk;
    int* id;
};

// One warp: fills p and id from the row's slots; returns sum_k p_k log p_k, and in *any
// whether there is a slot with any probability.  The teacher's logits count by their distance
// from the largest, taken before anything is rounded at their own size.
__device__ __forceinline__ float slots_read(const DistillArgs& a, size_t row, const Slots& s,
                                            int lane, bool* any) {
    const int* idx = a.idx + row * a.K;
    const float* tl = a.teacher + row * a.K;
    const float c = a.inv_tau;
    float m = -INFINITY;
    for (int k0 = lane; k0 < a.K; k0 += 64) {   // two of each on their way at once
        int i[2];
        float t[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int k = k0 + 32 * q;
            i[q] = k < a.K ? idx[k] : -1;
            t[q] = k < a.K ? tl[k] : 0.f;
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int k = k0 + 32 * q;
            if (k >= a.K) continue;
            if (i[q] >= a.V) {
                atomicExch(&g_error_word, kErrInvalid);
                i[q] = -1;
            }
            const float x = i[q] >= 0 ? t[q] : -INFINITY;
            s.id[k] = i[q];
            s.p[k] = x;
            m = fmaxf(m, x);
        }
    }
    m = warp_max(m);
    const float b = stat_base(m);
    float sum = 0.f;
    for (int k = lane; k < a.K; k += 32)
        sum += s.id[k] >= 0 ? ex2((s.p[k] - b) * (c * kLog2e)) : 0.f;
    sum = warp_sum(sum);
    *any = sum != 0.f;   // NaN counts: it belongs in the result
    const float ls = *any ? logf(sum) : 0.f, inv = *any ? 1.f / sum : 0.f;
    float ent = 0.f;
    for (int k = lane; k < a.K; k += 32) {
        const float t = s.p[k] - b;
        const float p = *any && s.id[k] >= 0 ? ex2(t * (c * kLog2e)) * inv : 0.f;
        s.p[k] = p;
        if (p != 0.f) ent += p * (t * c - ls);
    }
    return warp_sum(ent);
}

// Slot k: the sum of the probabilities of its symbol's slots if it is the first of them,
// else -1 (also for an empty slot).
__device__ __forceinline__ float slot_owned(const Slots& s, int K, int k) {
    const int i = s.id[k];
    if (i < 0) return -1.f;
    float t = 0.f;
    for (int j = 0; j < K; ++j) {
        if (s.id[j] != i) continue;
        if (j < k) return -1.f;
        t += s.p[j];
    }
    return t;
}

// One warp: fills own, above 32 slots through a table of the symbols (open addressing, `size` a
// power of two of at least 2 K entries of symbol and first slot).  Which entry a symbol gets
// depends on the order of the threads, what is found there does not.
__device__ __forceinline__ void slots_own(const Slots& s, int K, int* table, int size, int lane) {
    __syncwarp();    // the lanes' p and id are there for the others
    if (K <= 32) {   // a slot a lane: the lanes with the same symbol
        const int id = lane < K ? s.id[lane] : -1;
        const uint32_t same = __match_any_sync(0xffffffffu, id);
        if (lane < K) {
            float t = -1.f;
            if (id >= 0 && __ffs(same) - 1 == lane) {
                t = 0.f;
                for (uint32_t m = same; m; m &= m - 1) t += s.p[__ffs(m) - 1];
            }
            s.own[lane] = t;
        }
        __syncwarp();
        return;
    }
    int* const key = table;
    int* const low = table + size;
    for (int i = lane; i < size; i += 32) {
        key[i] = -1;
        low[i] = 0x7fffffff;
    }
    __syncwarp();
    for (int k = lane; k < K; k += 32) {
        const int id = s.id[k];
        if (id < 0) continue;
        int h = (int)(((uint32_t)id * 2654435761u) >> 7) & (size - 1);
        for (;;) {
            const int was = atomicCAS(&key[h], -1, id);
            if (was == -1 || was == id) break;
            h = (h + 1) & (size - 1);
        }
        atomicMin(&low[h], k);
        s.own[k] = __int_as_float(h);
    }
    __syncwarp();
    // a symbol with a second slot: its entry's sign bit
    for (int k = lane; k < K; k += 32) {
        if (s.id[k] < 0) continue;
        const int h = __float_as_int(s.own[k]);
        if ((low[h] & 0x7fffffff) != k) atomicOr(&low[h], (int)0x80000000);
    }
    __syncwarp();
    for (int k = lane; k < K; k += 32) {
        if (s.id[k] < 0) {
            s.own[k] = -1.f;
            continue;
        }
        const int l = low[__float_as_int(s.own[k])];
        if ((l & 0x7fffffff) != k)
            s.own[k] = -1.f;
        else
            s.own[k] = l < 0 ? slot_owned(s, K, k) : s.p[k];
    }
    __syncwarp();
}

// ------------------------------------------------------------------ W warps a row
// NE symbols a lane: symbol lane + 32 W e (lane: of the row's 32 W), in bf16 above 256 symbols two
// neighbours at a time, from the even place at or before the row's start: coalesced whatever
// the row's alignment.  Everything the row needs from its index alone is loaded at once; the named
// symbols' logits come after the row, from L1.  Slots lane and lane + 32 stay in registers, in
// each of the row's warps; the first one writes the loss and the named symbols.  At most 64
// registers (8 symbols a lane: 40): two kernels of 128 took nearly twice as long.  bf16, loss
// and gradient, 16384 rows, us and TB/s: V = 201 10.8, 1.2; 1000 20, 3.2; 2048 33, 4.1; 4096
// 64, 4.2: bound by the issue of instructions, a row's slots and factors first of all.
template <typename T, int NE, int EXPS, int W>
__global__ void __launch_bounds__(32 * kDWarps, NE == 8 ? 6 : 4) distill_warp_kernel(const DistillArgs a) {
    __shared__ float sp[kDWarps][kDWarpK];
    __shared__ int si[kDWarps][kDWarpK];
    __shared__ float red[3][kDWarps];   // the warps' maxima and sums
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = warp % W, first = lane + 32 * part;   // the row's warp and lane
    // all of the row's threads are here, and what they wrote before is there for the others
    auto meet = [&]() {
        if (W > 1)
            asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / W), "n"(32 * W) : "memory");
        else
            __syncwarp();
    };
    pdl_wait();
    pdl_trigger();
    const long long row = (long long)blockIdx.x * (kDWarps / W) + warp / W;
    if (row >= a.T) return;
    const T* z = static_cast<const T*>(a.z) + (size_t)row * a.V;
    T* dz = a.dz ? static_cast<T*>(a.dz) + (size_t)row * a.V : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    int y = a.target ? a.target[row] : -1;
    int id[2];
    float p[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int k = lane + 32 * q;
        id[q] = k < a.K ? a.idx[row * a.K + k] : -1;
        p[q] = k < a.K ? a.teacher[row * a.K + k] : 0.f;
    }
    constexpr bool kPairs = sizeof(T) == 2 && NE > 8;
    const int odd = kPairs ? (int)(row & a.V & 1) : 0;   // the row starts at an odd place
    // the lane's pair e: its first symbol (-1: the second alone lies in the row)
    auto pair_at = [&](int e) { return 2 * (first + 32 * W * e) - odd; };
    float v[NE];
    if constexpr (kPairs) {
        // whole pairs, and apart from them a first or a last symbol on its own
        uint32_t q[NE / 2];
#pragma unroll
        for (int e = 0; e < NE / 2; ++e) {
            const int j = pair_at(e);
            q[e] = j >= 0 && j + 1 < a.V ? *reinterpret_cast<const uint32_t*>(z + j) : 0xff80ff80u;
        }
        const float head = odd ? logit(z) : -INFINITY, tail = logit(z + a.V - 1);
#pragma unroll
        for (int e = 0; e < NE / 2; ++e) {
            v[2 * e] = pair_at(e) == a.V - 1 ? tail : __uint_as_float(q[e] << 16);
            v[2 * e + 1] = __uint_as_float(q[e] & 0xffff0000u);
        }
        if (first == 0 && odd) v[1] = head;
    } else {
#pragma unroll
        for (int e = 0; e < NE; ++e)
            v[e] = first + 32 * W * e < a.V ? logit(z + first + 32 * W * e) : -INFINITY;
    }
    if (w == 0.f) {   // whatever the row holds
        if (dz)
            for (int j = first; j < a.V; j += 32 * W) put(dz + j, 0.f);
        if (first == 0 && a.loss) a.loss[row] = 0.f;
        return;
    }
    if (y >= a.V || id[0] >= a.V || id[1] >= a.V) atomicExch(&g_error_word, kErrInvalid);
    if (y >= a.V) y = -1;
    // maxima of the row and of the teacher's logits
    float mz = -INFINITY, mt = -INFINITY;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (id[q] >= a.V) id[q] = -1;
        p[q] = id[q] >= 0 ? p[q] : -INFINITY;
        mt = fmaxf(mt, p[q]);
    }
#pragma unroll
    for (int e = 0; e < NE; ++e) mz = fmaxf(mz, v[e]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mz = fmaxf(mz, __shfl_xor_sync(0xffffffffu, mz, o));
        mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
    }
    if (W > 1) {
        if (lane == 0) red[0][warp] = mz;
        meet();
        mz = red[0][warp - part];
#pragma unroll
        for (int i = 1; i < W; ++i) mz = fmaxf(mz, red[0][warp - part + i]);
    }
    const float c = a.inv_tau * kLog2e;
    const float base = stat_base(mz), bt = stat_base(mt);
    const float zy = y >= 0 ? logit(z + y) : 0.f;
    float zk[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) zk[q] = id[q] >= 0 ? logit(z + id[q]) : 0.f;
    // sums: the row's exponentials, the teacher's, and its sum of exp(t / tau) (t - z)
    float s = 0.f, s1 = 0.f, st = 0.f, stt = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) {
        const float x = ex2((v[e] - base) * c);
        s += x;
        if (EXPS == kTwo) s1 += ex2((v[e] - base) * kLog2e);
        if (EXPS == kSquare) s1 += x * x;
    }
    float et[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        et[q] = id[q] >= 0 ? ex2((p[q] - bt) * c) : 0.f;
        st += et[q];
        if (et[q] != 0.f) stt += et[q] * ((p[q] - bt) - (zk[q] - base));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        st += __shfl_xor_sync(0xffffffffu, st, o);
        stt += __shfl_xor_sync(0xffffffffu, stt, o);
        if (EXPS != kOne) s1 += __shfl_xor_sync(0xffffffffu, s1, o);
    }
    if (W > 1) {
        if (lane == 0) {
            red[1][warp] = s;
            red[2][warp] = s1;
        }
        meet();
        s = red[1][warp - part];
        s1 = red[2][warp - part];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            s += red[1][warp - part + i];
            s1 += red[2][warp - part + i];
        }
    }
    if (EXPS == kOne) s1 = s;
    bool any = st != 0.f;   // NaN counts: it belongs in the result
    if (s == 0.f) {         // no logit above -inf: nothing to learn from
        any = false;
        y = -1;
        s = s1 = 1.f;
    }
    const float inv_t = any ? 1.f / st : 0.f;
    if (first == 0 && a.loss) {
        // sum p (log p - log q) with log p = (t - bt) / tau - log st and log q = (z - base) / tau
        // - log s
        const float kl = any ? stt * inv_t * a.inv_tau - logf(st) + logf(s) : 0.f;
        a.loss[row] = w * (a.kl * kl + (y >= 0 ? a.ce * (logf(s1) - (zy - base)) : 0.f));
    }
    if (!dz) return;
    const float fq = any ? w * a.kl_tau / s : 0.f, f1 = y >= 0 ? w * a.ce / s1 : 0.f;
    auto dense = [&](float x) {
        const float e = ex2((x - base) * c);
        if (EXPS == kOne) return (fq + f1) * e;
        return fq * e + f1 * (EXPS == kSquare ? e * e : ex2((x - base) * kLog2e));
    };
    if constexpr (kPairs) {
#pragma unroll
        for (int e = 0; e < NE / 2; ++e) {
            const int j = pair_at(e);
            const float x = dense(v[2 * e]);
            if (j >= 0 && j + 1 < a.V)
                *reinterpret_cast<uint32_t*>(dz + j) = pack_bf16x2(x, dense(v[2 * e + 1]));
            if (j == a.V - 1) put(dz + j, x);
        }
        if (first == 0 && odd) put(dz, dense(v[1]));
    } else {
#pragma unroll
        for (int e = 0; e < NE; ++e)
            if (first + 32 * W * e < a.V) put(dz + first + 32 * W * e, dense(v[e]));
    }
    meet();   // the dense values are in place
    if (part) return;
    bool named = false;
    if (any) {
        // a slot's share of its symbol: every slot its own, as a rule
        const uint32_t m0 = __match_any_sync(0xffffffffu, id[0]);
        bool twice = id[0] >= 0 && (m0 & (m0 - 1));
        float own[2] = {id[0] >= 0 ? et[0] * inv_t : -1.f, id[1] >= 0 ? et[1] * inv_t : -1.f};
        if (a.K > 32) {
            const uint32_t m1 = __match_any_sync(0xffffffffu, id[1]);
            twice |= id[1] >= 0 && (m1 & (m1 - 1));
#pragma unroll 8
            for (int r = 0; r < 32; ++r) {
                const int o = __shfl_sync(0xffffffffu, id[1], lane ^ r);
                twice |= id[0] >= 0 && o == id[0];
            }
        }
        if (__any_sync(0xffffffffu, twice)) {
            const Slots sl = {sp[warp], nullptr, nullptr, si[warp]};
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                si[warp][lane + 32 * q] = id[q];
                sp[warp][lane + 32 * q] = et[q] * inv_t;
            }
            __syncwarp();
#pragma unroll
            for (int q = 0; q < 2; ++q) own[q] = slot_owned(sl, kDWarpK, lane + 32 * q);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (own[q] < 0.f) continue;
            const bool is_y = id[q] == y;
            named |= is_y;
            put(dz + id[q], dense(zk[q]) - w * (a.kl_tau * own[q] + (is_y ? a.ce : 0.f)));
        }
    }
    named = __any_sync(0xffffffffu, named);
    if (y >= 0 && !named && lane == 0) put(dz + y, dense(zy) - w * a.ce);
}

// ------------------------------------------------------------------ a cluster a row
// Long rows: a persistent cluster of C CTAs takes rows in turn, each CTA a slice of the row's
// 16-byte vectors.  A CTA's roles:
//   producer      bulk copies of the slices of the next rows into a ring of buffers
//   NT compute    pass A (row n + 1): maximum and sum of the slice, each warp sending
//     threads     its part to every CTA of the cluster (st.async, counted by an mbarrier);
//                 then pass B (row n), whose factors are there by now: the gradient, from
//                 the slice in shared memory
//   slot warps    rows in turn: the teacher's probabilities and the named symbols' logits;
//                 the row's parts joined, and its factors for pass B; the loss; and, behind
//                 the dense values of pass B, the named symbols
// so that no compute warp waits for another CTA's current row.  Rows of weight 0 are not
// read.  us and TB/s: 2048 x 131072 bf16 164, 6.5; 16384 x 8192 bf16 101, 5.3; 1000 x 32003 fp32
// 46, 5.6.
// At most this many slot warps: a row's slots take about 10 us from their first load to the
// last named symbol, of which a slot warp waits half for the row itself; 64 KB of logits
// and as much gradient pass through an SM in 3 us.
constexpr int slot_warps(int nt) { return nt == 512 ? 8 : nt == 256 ? 4 : 2; }
constexpr int kDMaxSlotWarps = 8;   // slot warps in use: a power of two up to this
// Buffers of parts, row n's in buffer n % kDStats.  A CTA sends row m's parts after its
// pass B of row m - 2, whose factors need every warp's pass A of row m - 2, which comes after
// that warp's pass B of row m - 4 and so after row m - 4 was joined: four buffers would hold
// all rows that may still be read.  A wait for a buffer's barrier tells only odd from even
// rounds, so the slot warp that waits for row n has to have seen row n - kDStats: the
// buffers are a multiple of the slot warps, which makes it the same warp.
constexpr int kDStats = 8;
static_assert(kDStats >= 4 && kDStats % kDMaxSlotWarps == 0, "buffers of parts");
constexpr int kDMaxBufs = 4;
constexpr unsigned long long kDTimeoutNs = 2000000000ull;

struct __align__(16) DistillBars {
    uint64_t full[kDMaxBufs];        // a row's slice has landed
    uint64_t empty[kDMaxBufs];       // pass B has read it
    uint64_t stat[kDStats];          // every warp of the cluster has sent its part
    uint64_t ready[kDMaxSlotWarps];     // the slot warp's factors for its row are set
    uint64_t dense[kDMaxSlotWarps];     // the dense values of its row are stored
    // pass B's subtrahend of the exponents, factor at the teacher's temperature (of both
    // softmaxes where they are one) and factor at temperature 1
    float4 factor[kDMaxSlotWarps];
    int abort;
};

struct DistillPlan {
    int C, C_log2, clusters, bufs, look, slice;   // slice: bytes of a buffer
    int table;                            // entries of a slot warp's symbol table
    int sw_log2;                          // log2 of the slot warps that take rows
    size_t smem;
};

// A warp's rows: first + i * step, i = 0, 1, ...; their weights come 32 at a time.
struct RowCursor {
    const float* weight;
    int row, T, step, i, lane;
    float mine;
    __device__ __forceinline__ RowCursor(const DistillArgs& a, int first, int step_, int lane_)
        : weight(a.weight), row(first), T(a.T), step(step_), i(0), lane(lane_), mine(1.f) {
        fetch();
    }
    __device__ __forceinline__ void fetch() {
        const long long r = (long long)row + (long long)lane * step;
        mine = weight && r < T ? weight[r] : 1.f;
    }
    __device__ __forceinline__ bool more() const { return row < T; }
    __device__ __forceinline__ float w() const { return __shfl_sync(0xffffffffu, mine, i); }
    __device__ __forceinline__ void next() {
        row = row <= T - step ? row + step : T;
        if (++i == 32) {
            i = 0;
            fetch();
        }
    }
    // to the first row from here on that counts; false when there is none
    __device__ __forceinline__ bool seek() {
        while (more() && w() == 0.f) next();
        return more();
    }
};

__device__ __forceinline__ float2 ex2_pair(uint64_t x) {
    const float2 f = f32x2_unpack(x);
    return make_float2(ex2(f.x), ex2(f.y));
}

// Sends one 16-byte value to the same place of CTA `rank`'s shared memory, counted by its
// mbarrier `bar`.
__device__ __forceinline__ void send16(const void* at, const uint64_t* bar, uint32_t rank, float x,
                                       float y, float z) {
    asm volatile(
        "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
        ::"r"(mapa_shared(at, rank)), "r"(__float_as_uint(x)), "r"(__float_as_uint(y)),
        "r"(__float_as_uint(z)), "r"(0u), "r"(mapa_shared(bar, rank))
        : "memory");
}

// The joined statistic of a row from its n parts (at most 4 a lane), on every lane, in a
// fixed order.
template <int EXPS>
__device__ __forceinline__ Stat stat_read(const float4* part, int n, int lane, float c) {
    float4 q[4];
    Stat v = {-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[i] = lane + 32 * i < n ? part[lane + 32 * i] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        v.m = fmaxf(v.m, q[i].x);
    }
    const float b = stat_base(v.m);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float d = q[i].x == -INFINITY ? 0.f : q[i].x - b;
        v.s += q[i].y * ex2(d * c);
        if (EXPS != kOne) v.s1 += q[i].z * ex2(d * kLog2e);
    }
    return stat_warp<EXPS>(v, c);
}

template <typename T, int NT, int EXPS>
__global__ void __launch_bounds__(NT + 32 + 32 * slot_warps(NT), NT == 512 ? 1 : NT == 256 ? 2 : 4)
    distill_row_kernel(const DistillArgs a, const DistillPlan pl) {
    constexpr int VE = 16 / (int)sizeof(T);   // symbols of a vector
    constexpr int NW = NT / 32;
    constexpr int G = 4;                      // vectors a thread holds at once
    extern __shared__ __align__(128) uint8_t dsm[];
    uint8_t* p = dsm + (size_t)pl.bufs * pl.slice;
    float4* const stats = reinterpret_cast<float4*>(p);   // [kDStats][C * NW]
    const int parts = pl.C * NW;
    p += (size_t)kDStats * parts * sizeof(float4);
    uint8_t* const slot_mem = p;
    const size_t slot_bytes = (size_t)a.K * 16 + (size_t)pl.table * 8;
    DistillBars* const bars =
        reinterpret_cast<DistillBars*>(p + ((slot_bytes + 15) & ~(size_t)15) * ((size_t)1 << pl.sw_log2));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
    const int rank = (int)blockIdx.x % pl.C, first = (int)blockIdx.x / pl.C;
    const float c = a.inv_tau * kLog2e;
    volatile int* abort = &bars->abort;
    if (tid == 0) {
        for (int i = 0; i < pl.bufs; ++i) {
            mbar_init(&bars->full[i], 1);
            mbar_init(&bars->empty[i], NW);
        }
        for (int i = 0; i < kDStats; ++i) mbar_init(&bars->stat[i], 1);
        for (int i = 0; i < slot_warps(NT); ++i) {
            mbar_init(&bars->ready[i], 1);
            mbar_init(&bars->dense[i], NW);
        }
        bars->abort = 0;
        fence_mbar_init();
    }
    __syncthreads();
    cluster_sync_all();
    pdl_wait();
    pdl_trigger();

    // A row's vectors: those its symbols touch, the first and the last perhaps shared with
    // the rows beside it.  [v0, v1): this CTA's; [i0, i1): those wholly of the row.
    struct Row {
        size_t at;       // the row's first symbol
        int skew;        // symbols of vector 0 before it
        int n, v0, v1, i0, i1;
    };
    auto row_of = [&](int row) {
        Row r;
        r.at = (size_t)row * a.V;
        r.skew = (int)(r.at % VE);
        r.n = (r.skew + a.V + VE - 1) / VE;
        const int per = (r.n + pl.C - 1) >> pl.C_log2;
        r.v0 = rank * per < r.n ? rank * per : r.n;
        r.v1 = r.v0 + per < r.n ? r.v0 + per : r.n;
        r.i0 = r.v0 == 0 && r.skew ? 1 : r.v0;
        r.i1 = r.v1 == r.n && (r.skew + a.V) % VE ? r.n - 1 : r.v1;
        return r;
    };
    // The symbol of a shared vector of this CTA's that a lane looks after (the first
    // vector's with lanes 0 .. VE - 1, the last one's with the next VE), or -1.
    auto edge_of = [&](const Row& r) {
        const bool last = lane >= VE;
        const int v = last ? r.n - 1 : 0;
        const int j = v * VE + (lane & (VE - 1)) - r.skew;
        const bool shared = last ? r.v1 == r.n && r.i1 < r.n && (r.n > 1 || !r.skew)
                                 : r.v0 == 0 && r.skew != 0;
        return lane < 2 * VE && shared && r.v0 < r.v1 && j >= 0 && j < a.V ? j : -1;
    };
    const T* const zb = static_cast<const T*>(a.z);
    T* const gb = static_cast<T*>(a.dz);

    if (warp == NW) {
        // ------------------------------------------------------------ producer
        const size_t end = (size_t)a.T * a.V;   // symbols
        int n = 0;
        uint32_t issued = 0;
        bool ok = true;
        RowCursor cur(a, first, pl.clusters, lane);
        for (; ok && cur.seek(); cur.next(), ++n) {
            const int b = n % pl.bufs;
            bool w = true;
            if (n >= pl.bufs)
                w = mbar_wait(&bars->empty[b], ((n / pl.bufs) & 1) ^ 1, abort, kDTimeoutNs);
            ok = __all_sync(0xffffffffu, w);
            if (!ok) break;
            const Row r = row_of(cur.row);
            uint8_t* dst = dsm + (size_t)b * pl.slice;
            const size_t s0 = r.at - r.skew + (size_t)r.v0 * VE;
            // whole vectors inside the tensor; the symbols after them one by one
            size_t whole = (size_t)(r.v1 - r.v0);
            if (whole && s0 + whole * VE > end) {
                --whole;
                const size_t s1 = s0 + whole * VE;
                if (s1 + lane < end)
                    reinterpret_cast<T*>(dst + whole * 16)[lane] = zb[s1 + lane];
                __syncwarp();
            }
            if (lane == 0) {
                mbar_arrive_expect_tx(&bars->full[b], (uint32_t)(whole * 16));
                issued |= 1u << b;
                if (whole)
                    asm volatile(
                        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes "
                        "[%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                        "l"(zb + s0), "r"((uint32_t)(whole * 16)), "r"(smem_u32(&bars->full[b]))
                        : "memory");
            }
        }
        if (lane == 0)
            // every copy has landed before the CTA leaves, also when the others gave up
            for (int b = 0; b < pl.bufs; ++b)
                if (issued & (1u << b)) {
                    const int last = (n - 1 - b) / pl.bufs;   // the buffer's last round
                    mbar_wait_drain(&bars->full[b], last & 1, kDTimeoutNs);
                }
    } else if (warp > NW) {
        // ------------------------------------------------------------ slot warps
        const int sw = warp - NW - 1, sw_n = 1 << pl.sw_log2;
        Slots sl;
        sl.p = reinterpret_cast<float*>(slot_mem + sw * ((slot_bytes + 15) & ~(size_t)15));
        sl.own = sl.p + a.K;
        sl.zk = sl.own + a.K;
        sl.id = reinterpret_cast<int*>(sl.zk + a.K);
        int* const table = sl.id + a.K;
        RowCursor cur(a, first, pl.clusters, lane);
        int n = 0;
        bool ok = sw < sw_n;
        for (; ok && cur.seek(); cur.next(), ++n) {
            if ((n & (sw_n - 1)) != sw) continue;
            const uint32_t phase = (n >> pl.sw_log2) & 1;
            const float w = cur.w();
            const Row r = row_of(cur.row);
            const T* z = zb + r.at;
            T* dz = gb ? gb + r.at : nullptr;
            auto mine = [&](int j) {
                const int v = (r.skew + j) / VE;
                return v >= r.v0 && v < r.v1;
            };
            int y = a.target ? a.target[cur.row] : -1;
            bool any = false;
            float ent = 0.f;
            if (a.K) ent = slots_read(a, (size_t)cur.row, sl, lane, &any);
            if (y >= a.V) {
                if (lane == 0) atomicExch(&g_error_word, kErrInvalid);
                y = -1;
            }
            // the named symbols' logits, on their way while the symbols are sorted out
            auto named_logit = [&](int k) {
                const int i = k < a.K ? sl.id[k] : -1;
                return i >= 0 && (rank == 0 || mine(i)) ? logit(z + i) : 0.f;
            };
            const float zy = y >= 0 && (rank == 0 || mine(y)) ? logit(z + y) : 0.f;
            const float x0 = named_logit(lane), x1 = named_logit(lane + 32);
            if (any && dz) slots_own(sl, a.K, table, pl.table, lane);
            if (lane < a.K) sl.zk[lane] = x0;
            if (lane + 32 < a.K) sl.zk[lane + 32] = x1;
#pragma unroll 4
            for (int k = lane + 64; k < a.K; k += 32) sl.zk[k] = named_logit(k);
            const bool w1 = mbar_wait_cluster(&bars->stat[n % kDStats], (n / kDStats) & 1, abort,
                                              kDTimeoutNs);
            ok = __all_sync(0xffffffffu, w1);
            if (!ok) break;
            Stat st = stat_read<EXPS>(stats + (n % kDStats) * parts, parts, lane, c);
            const float base = stat_base(st.m);
            if (st.s == 0.f) {   // no logit above -inf: nothing to learn from
                any = false;
                y = -1;
                st.s = st.s1 = 1.f;
            }
            const float fq = any ? w * a.kl_tau / st.s : 0.f, f1 = y >= 0 ? w * a.ce / st.s1 : 0.f;
            if (lane == 0) {
                bars->factor[sw] = make_float4(-base, EXPS != kOne ? fq : fq + f1, f1, 0.f);
                mbar_arrive(&bars->ready[sw]);
            }
            if (rank == 0 && a.loss) {
                // log-sums relative to the maximum, as the logits are: the row's own size
                // cancels first
                const float ls = logf(st.s), ls1 = logf(st.s1);
                float l = 0.f;
                if (any)
                    for (int k = lane; k < a.K; k += 32)
                        if (sl.p[k] != 0.f) l -= sl.p[k] * ((sl.zk[k] - base) * a.inv_tau - ls);
                l = warp_sum(l) + (any ? ent : 0.f);
                if (lane == 0)
                    a.loss[cur.row] =
                        w * (a.kl * l + (y >= 0 ? a.ce * (ls1 - (zy - base)) : 0.f));
            }
            const bool w2 = mbar_wait(&bars->dense[sw], phase, abort, kDTimeoutNs);
            ok = __all_sync(0xffffffffu, w2);
            if (!ok) break;
            if (!dz) continue;
            auto dense = [&](float x) {
                const float e = ex2((x - base) * c);
                return EXPS != kOne ? fq * e + f1 * ex2((x - base) * kLog2e) : (fq + f1) * e;
            };
            bool named = false;   // the label, by a slot
            if (any)
                for (int k = lane; k < a.K; k += 32) {
                    const float t = sl.own[k];
                    if (t < 0.f) continue;
                    const bool is_y = sl.id[k] == y;
                    named |= is_y;
                    if (mine(sl.id[k]))
                        put(dz + sl.id[k], dense(sl.zk[k]) - w * (a.kl_tau * t + (is_y ? a.ce : 0.f)));
                }
            named = __any_sync(0xffffffffu, named);
            if (y >= 0 && !named && lane == 0 && mine(y)) put(dz + y, dense(zy) - w * a.ce);
        }
    } else {
        // ------------------------------------------------------------ compute warps
        auto elem = [](const uint4& u, int e) {
            const uint32_t ws[4] = {u.x, u.y, u.z, u.w};
            if (sizeof(T) == 4) return __uint_as_float(ws[e]);
            return __uint_as_float(e & 1 ? ws[e >> 1] & 0xFFFF0000u : ws[e >> 1] << 16);
        };
        // two neighbouring symbols of a vector
        auto pair = [](const uint4& u, int i) {
            const uint32_t ws[4] = {u.x, u.y, u.z, u.w};
            return sizeof(T) == 2
                       ? bf16x2_to_f32x2(ws[i])
                       : f32x2_pack(__uint_as_float(ws[2 * i]), __uint_as_float(ws[2 * i + 1]));
        };
        const uint32_t ninf = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
        const uint64_t cc = f32x2_pack(c, c), ll = f32x2_pack(kLog2e, kLog2e);
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            const bool w = mbar_wait(bar, parity, abort, kDTimeoutNs);
            ok = __all_sync(0xffffffffu, w);
            return ok;
        };
        // buffers of the next row of either pass, and pass A's parity
        int ba = 0, bb = 0, pa = 0;
        auto pass_a = [&](int row, int n) {
            const int b = ba;
            if (!wait(&bars->full[b], pa)) return;
            if (++ba == pl.bufs) {
                ba = 0;
                pa ^= 1;
            }
            const Row r = row_of(row);
            const uint4* buf = reinterpret_cast<const uint4*>(dsm + (size_t)b * pl.slice);
            Stat st = {-INFINITY, 0.f, 0.f};
            for (int g = r.i0 + tid; g < r.i1; g += G * NT) {
                uint4 q[G];
#pragma unroll
                for (int k = 0; k < G; ++k)
                    q[k] = g + k * NT < r.i1 ? buf[g + k * NT - r.v0]
                                             : make_uint4(ninf, ninf, ninf, ninf);
                Stat u = {-INFINITY, 0.f, 0.f};
                if (sizeof(T) == 2) {
                    __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162*>(&ninf);
#pragma unroll
                    for (int k = 0; k < G; ++k) {
                        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q[k]);
                        m = __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
                    }
                    u.m = fmaxf(__low2float(m), __high2float(m));
                } else {
#pragma unroll
                    for (int k = 0; k < G; ++k)
#pragma unroll
                        for (int e = 0; e < VE; ++e) u.m = fmaxf(u.m, elem(q[k], e));
                }
                const float nb = -stat_base(u.m);
                const uint64_t nbb = f32x2_pack(nb, nb);
                uint64_t s = 0, s1 = 0;   // two sums side by side
#pragma unroll
                for (int k = 0; k < G; ++k)
#pragma unroll
                    for (int i = 0; i < VE / 2; ++i) {
                        const uint64_t d = f32x2_add(pair(q[k], i), nbb);
                        const float2 e = ex2_pair(f32x2_mul(d, cc));
                        s = f32x2_add(s, f32x2_pack(e.x, e.y));
                        if (EXPS == kTwo) {
                            const float2 f = ex2_pair(f32x2_mul(d, ll));
                            s1 = f32x2_add(s1, f32x2_pack(f.x, f.y));
                        }
                        if (EXPS == kSquare) {
                            const uint64_t f = f32x2_pack(e.x, e.y);
                            s1 = f32x2_fma(f, f, s1);
                        }
                    }
                const float2 sf = f32x2_unpack(s), sf1 = f32x2_unpack(s1);
                u.s = sf.x + sf.y;
                u.s1 = EXPS != kOne ? sf1.x + sf1.y : u.s;
                st = stat_join<EXPS>(st, u, c);
            }
            if (warp == 0) {
                const int j = edge_of(r);
                if (j >= 0) {
                    const float x = logit(reinterpret_cast<const T*>(buf) + (j + r.skew - r.v0 * VE));
                    const float d = x - stat_base(x);
                    st = stat_join<EXPS>(st, Stat{x, ex2(d * c), ex2(d * kLog2e)}, c);
                }
            }
            st = stat_warp<EXPS>(st, c);
            if (!gb) {   // read once
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->empty[b]);
            }
            uint64_t* const bar = &bars->stat[n % kDStats];
            float4* const at = stats + (n % kDStats) * parts + rank * NW + warp;
            if (tid == 0) mbar_arrive_expect_tx(bar, (uint32_t)(parts * sizeof(float4)));
            if (lane < pl.C) send16(at, bar, (uint32_t)lane, st.m, st.s, st.s1);
        };
        auto pass_b = [&](int row, int n) {
            const int sw = n & ((1 << pl.sw_log2) - 1), b = bb;
            if (++bb == pl.bufs) bb = 0;
            if (!wait(&bars->ready[sw], (n >> pl.sw_log2) & 1)) return;
            if (gb) {
                const Row r = row_of(row);
                const uint4* buf = reinterpret_cast<const uint4*>(dsm + (size_t)b * pl.slice);
                uint4* const dv = reinterpret_cast<uint4*>(gb + (r.at - r.skew));
                const float4 f = bars->factor[sw];
                const float nb = f.x;
                const uint64_t nbb = f32x2_pack(nb, nb), ff = f32x2_pack(f.y, f.y),
                               ff1 = f32x2_pack(f.z, f.z);
#pragma unroll 2
                for (int v = r.i0 + tid; v < r.i1; v += NT) {
                    const uint4 q = buf[v - r.v0];
                    uint32_t o[4];
#pragma unroll
                    for (int i = 0; i < VE / 2; ++i) {
                        const uint64_t d = f32x2_add(pair(q, i), nbb);
                        const float2 e = ex2_pair(f32x2_mul(d, cc));
                        const uint64_t ee = f32x2_pack(e.x, e.y);
                        uint64_t g = f32x2_mul(ee, ff);
                        if (EXPS == kTwo) {
                            const float2 e1 = ex2_pair(f32x2_mul(d, ll));
                            g = f32x2_fma(f32x2_pack(e1.x, e1.y), ff1, g);
                        }
                        if (EXPS == kSquare) g = f32x2_fma(f32x2_mul(ee, ee), ff1, g);
                        const float2 h = f32x2_unpack(g);
                        if (sizeof(T) == 2) {
                            o[i] = pack_bf16x2(h.x, h.y);
                        } else {
                            o[2 * i] = __float_as_uint(h.x);
                            o[2 * i + 1] = __float_as_uint(h.y);
                        }
                    }
                    dv[v] = make_uint4(o[0], o[1], o[2], o[3]);
                }
                if (warp == 0) {
                    const int j = edge_of(r);
                    if (j >= 0) {
                        const float d =
                            logit(reinterpret_cast<const T*>(buf) + (j + r.skew - r.v0 * VE)) + nb;
                        put(gb + r.at + j, EXPS != kOne ? f.y * ex2(d * c) + f.z * ex2(d * kLog2e)
                                               : f.y * ex2(d * c));
                    }
                }
            }
            __syncwarp();
            if (lane == 0) {
                if (gb) mbar_arrive(&bars->empty[b]);
                mbar_arrive(&bars->dense[sw]);
            }
        };
        RowCursor ca(a, first, pl.clusters, lane), cb(a, first, pl.clusters, lane);
        int na = 0, nb = 0;
        for (; ok && cb.more(); cb.next()) {
            const float w = cb.w();
            if (w == 0.f) {   // whatever the row holds
                if (gb) {
                    const Row r = row_of(cb.row);
                    uint4* const dv = reinterpret_cast<uint4*>(gb + (r.at - r.skew));
                    for (int v = r.i0 + tid; v < r.i1; v += NT) dv[v] = make_uint4(0u, 0u, 0u, 0u);
                    if (warp == 0) {
                        const int j = edge_of(r);
                        if (j >= 0) put(gb + r.at + j, 0.f);
                    }
                }
                if (rank == 0 && tid == 0 && a.loss) a.loss[cb.row] = 0.f;
                continue;
            }
            while (ok && na <= nb + pl.look && ca.seek()) {
                pass_a(ca.row, na);
                ++na;
                ca.next();
            }
            if (!ok) break;
            pass_b(cb.row, nb);
            ++nb;
        }
    }
    // No CTA leaves while another may still send to it.  A sent part that was waited for has come
    // by then; after giving up some were not.
    __syncwarp();
    cluster_sync_all();
    if (*abort) settle_after_abort();
}

template <typename T, int NT, int EXPS>
cudaError_t launch_distill_rows(const DistillArgs& a, DistillPlan pl, cudaStream_t st) {
    auto kern = distill_row_kernel<T, NT, EXPS>;
    static std::once_flag once[64];
    static cudaError_t set_err[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::call_once(once[dev], [&] {
        set_err[dev] = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                            (int)kDSmem);
    });
    if (set_err[dev] != cudaSuccess) return set_err[dev];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)pl.C);
    cfg.blockDim = dim3(NT + 32 + 32 * slot_warps(NT));
    cfg.dynamicSmemBytes = pl.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)pl.C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    // no more clusters than run at once (their SMs have to lie together, so this is not the
    // SMs over C): rows are dealt out in turn, and a late cluster's would come late.  Asked
    // once for a device, cluster size and shared memory, in steps of 4 KB.
    static std::mutex lock;
    static int fit[64][4][64];
    const int step = (int)((pl.smem + 4095) / 4096), lc = pl.C_log2;
    int n;
    {
        std::lock_guard<std::mutex> hold(lock);
        int& f = fit[dev][lc][step];
        if (!f) {
            cudaLaunchConfig_t q = cfg;
            q.numAttrs = 1;
            q.dynamicSmemBytes = (size_t)step * 4096 < kDSmem ? (size_t)step * 4096 : kDSmem;
            e = cudaOccupancyMaxActiveClusters(&n, kern, &q);
            if (e != cudaSuccess) return e;
            f = n > 0 ? n : 1;
        }
        n = f;
    }
    pl.clusters = a.T < n ? a.T : n;
    cfg.gridDim = dim3((unsigned)(pl.clusters * pl.C));
    return cudaLaunchKernelEx(&cfg, kern, a, pl);
}

template <typename T, int EXPS>
cudaError_t launch_distill(const DistillArgs& a, cudaStream_t st) {
    // Rows in registers, or in a cluster's shared memory (us, 16384 rows of bf16, 8192 of fp32; K = 32
    // at one temperature and K = 64 at two): bf16 V = 2048: 33, 72 and 41, 129; 4096: 64, 78 and 77,
    // 133; 8192: 125, 101; fp32 4096: 44, 51; 8192: 81, 95.
    if (a.V <= (sizeof(T) == 2 ? kDWarpV / 2 : kDWarpV) && a.K <= kDWarpK) {
        const dim3 block(32 * kDWarps);
        auto grid = [&](int w) { return dim3((unsigned)(((long long)a.T * w + kDWarps - 1) / kDWarps)); };
        if (a.V <= 256)
            return launch_pdl(distill_warp_kernel<T, 8, EXPS, 1>, grid(1), block, 0, st, a);
        if (a.V <= 1024)
            return launch_pdl(distill_warp_kernel<T, 32, EXPS, 1>, grid(1), block, 0, st, a);
        if (a.V <= 2048)
            return launch_pdl(distill_warp_kernel<T, 32, EXPS, 2>, grid(2), block, 0, st, a);
        if (a.V <= 4096)
            return launch_pdl(distill_warp_kernel<T, 32, EXPS, 4>, grid(4), block, 0, st, a);
        if constexpr (sizeof(T) == 4)
            return launch_pdl(distill_warp_kernel<T, 32, EXPS, 8>, grid(8), block, 0, st, a);
    }
    const int sms = device_sms();
    const long long bytes = (long long)a.V * (int)sizeof(T) + 32;
    DistillPlan pl;
    // the fewest CTAs a row whose slices fit 64 KB (8 at most); more while the rows alone
    // leave SMs without a CTA and a slice has 8 KB or more
    pl.C = 1;
    while (pl.C < 8 && bytes > pl.C * (kDSlice + 1024)) pl.C *= 2;
    while (pl.C < 8 && (long long)a.T * pl.C * 2 <= sms && bytes > pl.C * 8192ll) pl.C *= 2;
    pl.C_log2 = pl.C == 1 ? 0 : pl.C == 2 ? 1 : pl.C == 4 ? 2 : 3;
    // a slice: the row's vectors shared out, as a multiple of 128 bytes
    const long long vecs = ((long long)a.V + 16 / sizeof(T) - 1) / (16 / sizeof(T)) + 1;
    pl.slice = (int)(((vecs + pl.C - 1) / pl.C * 16 + 127) / 128 * 128);
    // eight vectors a thread: 512 threads and one CTA an SM for 64 KB, and so on down
    const int nt = pl.slice <= 17408 ? 128 : pl.slice <= 33792 ? 256 : 512;
    const int per_sm = nt == 128 ? 4 : nt == 256 ? 2 : 1;
    pl.table = 64;
    while (pl.table < 2 * a.K) pl.table *= 2;
    if (!a.K) pl.table = 0;
    const size_t slots = (((size_t)a.K * 16 + (size_t)pl.table * 8) + 15) & ~(size_t)15;
    const size_t room = kDSmem / per_sm - (per_sm > 1 ? 1024 : 0);
    // fewer slot warps where their slots would take a quarter of the room
    pl.sw_log2 = nt == 512 ? 3 : nt == 256 ? 2 : 1;
    while (pl.sw_log2 && (slots << pl.sw_log2) > room / 4) --pl.sw_log2;
    const size_t fixed = (size_t)kDStats * pl.C * (nt / 32) * 16 + (slots << pl.sw_log2) +
                         sizeof(DistillBars);
    pl.bufs = 3;
    while (pl.bufs > 1 && fixed + (size_t)pl.bufs * pl.slice > room) --pl.bufs;
    if (pl.bufs == 1 && 2 * (size_t)pl.slice + fixed <= kDSmem) pl.bufs = 2;
    pl.look = pl.bufs > 1;
    pl.smem = fixed + (size_t)pl.bufs * pl.slice;
    pl.clusters = 0;   // the launch's
    if (nt == 128) return launch_distill_rows<T, 128, EXPS>(a, pl, st);
    if (nt == 256) return launch_distill_rows<T, 256, EXPS>(a, pl, st);
    return launch_distill_rows<T, 512, EXPS>(a, pl, st);
}

}  // namespace

cudaError_t distill_error_word_read_clear(int* word) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(word, g_error_word, sizeof(int));
    if (e == cudaSuccess && *word) e = cudaMemcpyToSymbol(g_error_word, &zero, sizeof(int));
    return e;
}

}  // namespace hcw

using namespace hcw;

extern "C" int hcw_distill_loss(const void* z, const int* idx, const float* teacher,
                                const int* target, const float* weight, int T, int V, int K,
                                int dtype, float temperature, float kl_scale, float ce_scale,
                                float* loss, void* dz, void* stream) {
    if (T < 0 || V < 1 || K < 0 || (dtype != HCW_BF16 && dtype != HCW_F32) ||
        !(temperature > 0.f) || !isfinite(temperature) || !isfinite(kl_scale) ||
        !isfinite(ce_scale))
        return HCW_ERR_INVALID_ARG;
    // a grid holds the rows times the CTAs of a row
    if (V > kDMaxV || K > kDMaxK || T > 0x7fffffff / 8) return HCW_ERR_UNSUPPORTED;
    const auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    if (!aligned(z) || !aligned(idx) || !aligned(teacher) || !aligned(target) || !aligned(weight) ||
        !aligned(loss) || !aligned(dz))
        return HCW_ERR_ALIGNMENT;
    const size_t zb = (size_t)T * V * (dtype == HCW_F32 ? 4 : 2), kb = (size_t)T * K * 4,
                 tb = (size_t)T * 4;
    const auto meet = [](const void* a, size_t na, const void* b, size_t nb) {
        if (!a || !b || !na || !nb) return false;
        const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
        return x < y + nb && y < x + na;
    };
    const struct {
        const void* p;
        size_t n;
    } in[] = {{z, zb}, {idx, kb}, {teacher, kb}, {target, tb}, {weight, tb}};
    for (const auto& q : in)
        if (meet(loss, tb, q.p, q.n) || meet(dz, zb, q.p, q.n)) return HCW_ERR_ALIASING;
    if (meet(loss, tb, dz, zb)) return HCW_ERR_ALIASING;
    if (T == 0) return HCW_OK;
    if (!z || (!loss && !dz) || (K > 0) != (idx != nullptr) ||
        (idx != nullptr) != (teacher != nullptr))
        return HCW_ERR_INVALID_ARG;
    DistillArgs a = {};
    a.z = z;
    a.idx = kl_scale != 0.f ? idx : nullptr;
    a.teacher = teacher;
    a.target = ce_scale != 0.f ? target : nullptr;
    a.weight = weight;
    a.loss = loss;
    a.dz = dz;
    a.T = T;
    a.V = V;
    a.K = a.idx ? K : 0;
    a.inv_tau = 1.f / temperature;
    a.kl = kl_scale * temperature * temperature;
    a.kl_tau = kl_scale * temperature;
    a.ce = ce_scale;
    const cudaStream_t st = (cudaStream_t)stream;
    // the label's softmax is at temperature 1: a second sum where the teacher's is not
    const int exps = !(a.idx && a.target) || temperature == 1.f ? kOne
                     : temperature == 2.f                        ? kSquare
                                                                 : kTwo;
    // without the teacher's part only the label's softmax is left
    if (!a.idx) a.inv_tau = 1.f;
    cudaError_t e;
    if (dtype == HCW_BF16)
        e = exps == kOne   ? launch_distill<__nv_bfloat16, kOne>(a, st)
            : exps == kTwo ? launch_distill<__nv_bfloat16, kTwo>(a, st)
                           : launch_distill<__nv_bfloat16, kSquare>(a, st);
    else
        e = exps == kOne   ? launch_distill<float, kOne>(a, st)
            : exps == kTwo ? launch_distill<float, kTwo>(a, st)
                           : launch_distill<float, kSquare>(a, st);
    return count_launch(e, 1);
}
