// hcw_distill.cu -- distillation from a teacher's top logits, loss and gradient in one
// pass over the student's logits (hcw_distill_loss).  Per row, with M the row's maximum:
//
//   p = softmax over the given slots of t / tau        (the teacher, K slots)
//   q = softmax(z / tau),  q1 = softmax(z)             (the student, V symbols)
//   loss = w [ a tau^2 sum_k p_k (log p_k - log q_{i_k}) + b (log sum exp(z) - z_y) ]
//   dz_j = w [ a tau (P q_j - sum_{k: i_k = j} p_k) + b (q1_j - [j = y]) ]
//
// (P = 1, or 0 for a row without slots).  Bound by memory: the logits are read once and
// the gradient is written once, 4 bytes a symbol in bf16.  A row stays in registers
// between the sums and the gradient: a cluster of up to 8 CTAs shares a long row (or the
// few rows of a short batch), each CTA summing its part against its own maximum and the
// parts being joined through distributed shared memory.  Short rows (V <= 1024) take a
// warp each.  The dense part of the gradient goes out first; then the symbols that the
// teacher or the label names are written again with their share taken off, each by the
// one thread that owns the symbol's first slot, so no atomics and no fixed-up rounding:
// every output is rounded once, from fp32.
//
// A row starts anywhere (V may be odd): its whole 16-byte vectors go to the threads in
// turn and the up to seven symbols on either side of them to the first threads of the
// row's first CTA.
#include "hcw.h"
#include "hcw_internal.h"
#include "hcw_ptx.cuh"

#include <math.h>

namespace hcw {

namespace {

constexpr int kDMaxK = 1024;          // slots of a row
constexpr int kDMaxV = 262144;        // 8 CTAs x 512 threads x 64 symbols
constexpr int kDThreads = 512;
constexpr int kDWarpV = 1024;         // a warp a row up to here,
constexpr int kDWarpK = 64;           // and up to this many slots
constexpr int kDWarps = 8;            // rows of a CTA of the warp kernel
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

template <bool TWO>
__device__ __forceinline__ Stat stat_join(const Stat& x, const Stat& y, float c) {
    Stat r;
    r.m = fmaxf(x.m, y.m);
    const float b = stat_base(r.m);
    const float dx = x.m == -INFINITY ? -INFINITY : x.m - b, dy = y.m == -INFINITY ? -INFINITY : y.m - b;
    // a part without symbols has no sum; one with NaN keeps it
    const float fx = ex2(dx * c), fy = ex2(dy * c);
    r.s = (x.m == -INFINITY ? x.s : x.s * fx) + (y.m == -INFINITY ? y.s : y.s * fy);
    if (TWO) {
        const float gx = ex2(dx * kLog2e), gy = ex2(dy * kLog2e);
        r.s1 = (x.m == -INFINITY ? x.s1 : x.s1 * gx) + (y.m == -INFINITY ? y.s1 : y.s1 * gy);
    } else {
        r.s1 = r.s;
    }
    return r;
}

template <bool TWO>
__device__ __forceinline__ Stat stat_warp(Stat v, float c) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Stat u;
        u.m = __shfl_xor_sync(0xffffffffu, v.m, o);
        u.s = __shfl_xor_sync(0xffffffffu, v.s, o);
        u.s1 = TWO ? __shfl_xor_sync(0xffffffffu, v.s1, o) : u.s;
        v = stat_join<TWO>(v, u, c);
    }
    return v;
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
// id[k] (-1), and after it p_own[k]: the slots' sum for the symbol where slot k is its first
// one, else -1.  `threads` threads of index `t` take part, `sync` orders them.  An index at
// or past V is reported and counts as empty.
struct Slots {
    float *p, *own, *zk;
    int* id;
};

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

// One warp: fills p and id from the row's slots; returns sum_k p_k log p_k, and in *any
// whether there is a slot with any probability.
__device__ __forceinline__ float slots_read(const DistillArgs& a, size_t row, const Slots& s,
                                            int lane, bool* any) {
    const int* idx = a.idx + row * a.K;
    const float* tl = a.teacher + row * a.K;
    const float c = a.inv_tau;
    float m = -INFINITY;
    for (int k = lane; k < a.K; k += 32) {
        int i = idx[k];
        if (i >= a.V) {
            atomicExch(&g_error_word, kErrInvalid);
            i = -1;
        }
        const float t = i >= 0 ? tl[k] * c : -INFINITY;
        s.id[k] = i;
        s.p[k] = t;
        m = fmaxf(m, t);
    }
    m = warp_max(m);
    const float b = stat_base(m);
    float sum = 0.f;
    for (int k = lane; k < a.K; k += 32) sum += s.id[k] >= 0 ? expf(s.p[k] - b) : 0.f;
    sum = warp_sum(sum);
    *any = sum != 0.f;   // NaN counts: it belongs in the result
    const float lse = *any ? b + logf(sum) : 0.f, inv = *any ? 1.f / sum : 0.f;
    float ent = 0.f;
    for (int k = lane; k < a.K; k += 32) {
        const float t = s.p[k];
        const float p = *any && s.id[k] >= 0 ? expf(t - b) * inv : 0.f;
        s.p[k] = p;
        if (p != 0.f) ent += p * (t - lse);
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

// ------------------------------------------------------------------ a warp a row
// NE symbols a lane, symbol lane + 32 e: coalesced whatever the row's alignment.
template <typename T, int NE, bool TWO>
__global__ void __launch_bounds__(32 * kDWarps) distill_warp_kernel(const DistillArgs a) {
    __shared__ float sp[kDWarps][kDWarpK], so[kDWarps][kDWarpK], sz[kDWarps][kDWarpK];
    __shared__ int si[kDWarps][kDWarpK];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    const long long row = (long long)blockIdx.x * kDWarps + warp;
    if (row >= a.T) return;
    const T* z = static_cast<const T*>(a.z) + (size_t)row * a.V;
    T* dz = a.dz ? static_cast<T*>(a.dz) + (size_t)row * a.V : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {   // whatever the row holds
        if (dz)
            for (int j = lane; j < a.V; j += 32) put(dz + j, 0.f);
        if (lane == 0 && a.loss) a.loss[row] = 0.f;
        return;
    }
    float v[NE];
#pragma unroll
    for (int e = 0; e < NE; ++e) v[e] = lane + 32 * e < a.V ? logit(z + lane + 32 * e) : -INFINITY;
    const Slots sl = {sp[warp], so[warp], sz[warp], si[warp]};
    bool any = false;
    float ent = 0.f;
    if (a.idx) {
        ent = slots_read(a, (size_t)row, sl, lane, &any);
        __syncwarp();
        for (int k = lane; k < a.K; k += 32) {
            sl.own[k] = slot_owned(sl, a.K, k);
            sl.zk[k] = sl.id[k] >= 0 ? logit(z + sl.id[k]) : 0.f;
        }
        __syncwarp();
    }
    int y = a.target ? a.target[row] : -1;
    if (y >= a.V) {
        if (lane == 0) atomicExch(&g_error_word, kErrInvalid);
        y = -1;
    }
    const float zy = y >= 0 ? logit(z + y) : 0.f;
    const float c = a.inv_tau * kLog2e;
    Stat st = {-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < NE; ++e) st.m = fmaxf(st.m, v[e]);
    st.m = warp_max(st.m);
    const float base = stat_base(st.m);
#pragma unroll
    for (int e = 0; e < NE; ++e) {
        st.s += ex2((v[e] - base) * c);
        if (TWO) st.s1 += ex2((v[e] - base) * kLog2e);
    }
    st.s = warp_sum(st.s);
    st.s1 = TWO ? warp_sum(st.s1) : st.s;
    if (st.s == 0.f) {   // no logit above -inf: nothing to learn from
        any = false;
        y = -1;
        st.s = st.s1 = 1.f;
    }
    // log-sums relative to the maximum, as the logits are: the row's own size cancels first
    const float ls = logf(st.s), ls1 = logf(st.s1);
    float l = 0.f;
    if (any)
        for (int k = lane; k < a.K; k += 32)
            if (sl.p[k] != 0.f) l -= sl.p[k] * ((sl.zk[k] - base) * a.inv_tau - ls);
    l = warp_sum(l) + (any ? ent : 0.f);
    if (lane == 0 && a.loss) a.loss[row] = w * (a.kl * l + (y >= 0 ? a.ce * (ls1 - (zy - base)) : 0.f));
    if (!dz) return;
    const float fq = any ? w * a.kl_tau / st.s : 0.f, f1 = y >= 0 ? w * a.ce / st.s1 : 0.f;
    auto dense = [&](float x) {
        const float e = ex2((x - base) * c);
        return TWO ? fq * e + f1 * ex2((x - base) * kLog2e) : (fq + f1) * e;
    };
#pragma unroll
    for (int e = 0; e < NE; ++e)
        if (lane + 32 * e < a.V) put(dz + lane + 32 * e, dense(v[e]));
    __syncwarp();   // the dense values are in place
    bool y_done = false;
    if (any)
        for (int k = lane; k < a.K; k += 32) {
            const float t = sl.own[k];
            if (t < 0.f) continue;
            const bool is_y = sl.id[k] == y;
            y_done |= is_y;
            put(dz + sl.id[k], dense(sl.zk[k]) - w * (a.kl_tau * t + (is_y ? a.ce : 0.f)));
        }
    y_done = __any_sync(0xffffffffu, y_done);
    if (y >= 0 && !y_done && lane == 0) put(dz + y, dense(zy) - w * a.ce);
}

// ------------------------------------------------------------------ a cluster a row
// NV 16-byte vectors a thread.  The cluster's CTAs take the row's vectors in equal runs.
template <typename T, int NV, bool TWO>
__global__ void __launch_bounds__(kDThreads) distill_row_kernel(const DistillArgs a, int C) {
    constexpr int VE = 16 / (int)sizeof(T);   // symbols of a vector
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ Stat warp_stat[kDThreads / 32];
    __shared__ Stat cta_stat;   // read by the cluster
    __shared__ float s_ent;
    __shared__ int s_any;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
    const int n_warps = (int)blockDim.x >> 5, nt = (int)blockDim.x;
    const int rank = (int)blockIdx.x % C;
    const long long row = blockIdx.x / C;
    Slots sl;
    sl.p = reinterpret_cast<float*>(dyn);
    sl.own = sl.p + a.K;
    sl.zk = sl.own + a.K;
    sl.id = reinterpret_cast<int*>(sl.zk + a.K);
    pdl_wait();
    pdl_trigger();
    const T* z = static_cast<const T*>(a.z) + (size_t)row * a.V;
    T* dz = a.dz ? static_cast<T*>(a.dz) + (size_t)row * a.V : nullptr;
    // symbols before the row's first whole vector, the vectors, this CTA's run of them
    const int skew = (int)(((size_t)row * a.V) % VE);
    int head = skew ? VE - skew : 0;
    if (head > a.V) head = a.V;
    const int n_vec = (a.V - head) / VE;
    const int per = (n_vec + C - 1) / C;
    const int v0 = rank * per < n_vec ? rank * per : n_vec;
    const int v1 = v0 + per < n_vec ? v0 + per : n_vec;
    const int tail0 = head + n_vec * VE;
    // and this thread's symbol beside the vectors
    int edge = -1;
    if (rank == 0 && tid < VE && tid < head) edge = tid;
    if (rank == 0 && tid >= VE && tid < 2 * VE && tail0 + tid - VE < a.V) edge = tail0 + tid - VE;
    const uint4* zv = reinterpret_cast<const uint4*>(z + head);
    uint4* dv = dz ? reinterpret_cast<uint4*>(dz + head) : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {   // whatever the row holds; the whole cluster leaves here
        if (dz) {
            for (int i = v0 + tid; i < v1; i += nt) dv[i] = make_uint4(0u, 0u, 0u, 0u);
            if (edge >= 0) put(dz + edge, 0.f);
        }
        if (rank == 0 && tid == 0 && a.loss) a.loss[row] = 0.f;
        return;
    }
    const uint32_t ninf = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    uint4 q[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = v0 + tid + i * nt;
        q[i] = j < v1 ? zv[j] : make_uint4(ninf, ninf, ninf, ninf);
    }
    const float ze = edge >= 0 ? logit(z + edge) : -INFINITY;
    int y = a.target ? a.target[row] : -1;
    if (y >= a.V) {
        if (tid == 0) atomicExch(&g_error_word, kErrInvalid);
        y = -1;
    }
    const float zy = y >= 0 ? logit(z + y) : 0.f;
    // the slots, while the row is on its way
    if (a.idx && warp == 0) {
        bool any;
        const float ent = slots_read(a, (size_t)row, sl, lane, &any);
        if (lane == 0) {
            s_ent = ent;
            s_any = any;
        }
    }
    if (!a.idx && tid == 0) s_any = 0;
    __syncthreads();
    if (a.idx)
        for (int k = tid; k < a.K; k += nt) {
            sl.own[k] = slot_owned(sl, a.K, k);
            sl.zk[k] = sl.id[k] >= 0 ? logit(z + sl.id[k]) : 0.f;
        }

    auto elem = [&](const uint4& u, int e) {
        const uint32_t ws[4] = {u.x, u.y, u.z, u.w};
        if (sizeof(T) == 4) return __uint_as_float(ws[e]);
        return __uint_as_float(e & 1 ? ws[e >> 1] & 0xFFFF0000u : ws[e >> 1] << 16);
    };
    const float c = a.inv_tau * kLog2e;
    Stat st = {ze, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) st.m = fmaxf(st.m, elem(q[i], e));
    {
        const float b = stat_base(st.m);
        st.s = ex2((ze - b) * c);
        if (TWO) st.s1 = ex2((ze - b) * kLog2e);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float x = elem(q[i], e) - b;
                st.s += ex2(x * c);
                if (TWO) st.s1 += ex2(x * kLog2e);
            }
    }
    st = stat_warp<TWO>(st, c);
    if (lane == 0) warp_stat[warp] = st;
    __syncthreads();
    if (warp == 0) {
        Stat u = {-INFINITY, 0.f, 0.f};
        if (lane < n_warps) u = warp_stat[lane];
        u = stat_warp<TWO>(u, c);
        if (lane == 0) cta_stat = u;
    }
    __syncwarp();
    if (C > 1) {
        cluster_sync_all();
        // every thread joins the CTAs' parts, in rank order
        st = Stat{-INFINITY, 0.f, 0.f};
        for (int r = 0; r < C; ++r) {
            const uint32_t at = mapa_shared(&cta_stat, (uint32_t)r);
            Stat u;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u.m) : "r"(at) : "memory");
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u.s) : "r"(at + 4) : "memory");
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u.s1) : "r"(at + 8) : "memory");
            st = stat_join<TWO>(st, u, c);
        }
        // no CTA leaves while another may still read its part
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    } else {
        __syncthreads();
        st = cta_stat;
    }
    const float base = stat_base(st.m);
    bool any = s_any != 0;
    if (st.s == 0.f) {   // no logit above -inf: nothing to learn from
        any = false;
        y = -1;
        st.s = st.s1 = 1.f;
    }
    if (rank == 0 && warp == 0 && a.loss) {
        // log-sums relative to the maximum, as the logits are: the row's own size cancels first
        const float ls = logf(st.s), ls1 = logf(st.s1);
        float l = 0.f;
        if (any)
            for (int k = lane; k < a.K; k += 32)
                if (sl.p[k] != 0.f) l -= sl.p[k] * ((sl.zk[k] - base) * a.inv_tau - ls);
        l = warp_sum(l) + (any ? s_ent : 0.f);
        if (lane == 0) a.loss[row] = w * (a.kl * l + (y >= 0 ? a.ce * (ls1 - (zy - base)) : 0.f));
    }
    if (dz) {
        const float fq = any ? w * a.kl_tau / st.s : 0.f, f1 = y >= 0 ? w * a.ce / st.s1 : 0.f;
        auto dense = [&](float x) {
            const float e = ex2((x - base) * c);
            return TWO ? fq * e + f1 * ex2((x - base) * kLog2e) : (fq + f1) * e;
        };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = v0 + tid + i * nt;
            if (j >= v1) continue;
            uint32_t o[4];
            if (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(dense(elem(q[i], e)));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[e] = pack_bf16x2(dense(elem(q[i], 2 * e)), dense(elem(q[i], 2 * e + 1)));
            }
            dv[j] = make_uint4(o[0], o[1], o[2], o[3]);
        }
        if (edge >= 0) put(dz + edge, dense(ze));
        __syncthreads();   // the CTA's dense values are in place
        // the named symbols of this CTA's part of the row
        auto mine = [&](int j) {
            if (j < head || j >= tail0) return rank == 0;
            const int v = (j - head) / VE;
            return v >= v0 && v < v1;
        };
        // (the label itself where no slot names it)
        bool y_named = false;
        if (any)
            for (int k = tid; k < a.K; k += nt) {
                const float t = sl.own[k];
                if (t < 0.f) continue;
                const bool is_y = sl.id[k] == y;
                y_named |= is_y;
                if (mine(sl.id[k]))
                    put(dz + sl.id[k], dense(sl.zk[k]) - w * (a.kl_tau * t + (is_y ? a.ce : 0.f)));
            }
        y_named = __syncthreads_or(y_named);
        if (y >= 0 && !y_named && tid == 0 && mine(y)) put(dz + y, dense(zy) - w * a.ce);
    }
    __syncwarp();
    if (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

int distill_sms() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1)
        return 148;
    return n;
}

template <typename T, int NV, bool TWO>
cudaError_t launch_distill_rows(const DistillArgs& a, int C, int threads, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.T * (unsigned)C);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)a.K * 16;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)C;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = C > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, distill_row_kernel<T, NV, TWO>, a, C);
}

template <typename T, bool TWO>
cudaError_t launch_distill(const DistillArgs& a, cudaStream_t st) {
    if (a.V <= kDWarpV && a.K <= kDWarpK) {
        const dim3 grid((unsigned)((a.T + kDWarps - 1) / kDWarps)), block(32 * kDWarps);
        if (a.V <= 256) return launch_pdl(distill_warp_kernel<T, 8, TWO>, grid, block, 0, st, a);
        return launch_pdl(distill_warp_kernel<T, 32, TWO>, grid, block, 0, st, a);
    }
    constexpr int VE = 16 / (int)sizeof(T);
    constexpr int kMost = 64 / VE;   // vectors a thread: 64 symbols
    // the fewest CTAs a row whose threads hold it, and more while the rows alone leave SMs
    // without a CTA and each thread has two vectors or more
    const long long n_vec = a.V / VE;
    int C = 1;
    while (C < 8 && n_vec > (long long)C * kDThreads * kMost) C *= 2;
    const int sms = distill_sms();
    while (C < 8 && (long long)a.T * C * 2 <= sms && n_vec > (long long)C * kDThreads * 2) C *= 2;
    const int per = (int)((n_vec + C - 1) / C);
    int threads = 128;
    while (threads < kDThreads && per > threads * 2) threads *= 2;
    const int nv = (per + threads - 1) / threads;
    if (nv <= 2) return launch_distill_rows<T, 2, TWO>(a, C, threads, st);
    if (nv <= 4) return launch_distill_rows<T, 4, TWO>(a, C, threads, st);
    if (nv <= 8 || kMost == 8) return launch_distill_rows<T, 8, TWO>(a, C, threads, st);
    return launch_distill_rows<T, kMost, TWO>(a, C, threads, st);
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
    const bool two = a.idx && a.target && temperature != 1.f;
    // without the teacher's part only the label's softmax is left
    if (!a.idx) a.inv_tau = 1.f;
    cudaError_t e;
    if (dtype == HCW_BF16)
        e = two ? launch_distill<__nv_bfloat16, true>(a, st)
                : launch_distill<__nv_bfloat16, false>(a, st);
    else
        e = two ? launch_distill<float, true>(a, st) : launch_distill<float, false>(a, st);
    return count_launch(e, 1);
}
