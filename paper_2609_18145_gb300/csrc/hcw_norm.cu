// hcw_norm.cu -- the norms after one block and before the next, fused with the
// block's gate and the residual scale (hcw_residual_norm_fwd / _bwd):
//
//   forward   v = N_post(f) (or f);  s = alpha r + gate v;  r_out = s;  x_out = N_pre(s)
//   backward  ds = dr_out + N_pre'(s)^T dx_out;  dr = alpha ds
//             df = N_post'(f)^T (gate ds)
//             dgate = sum ds v;  dpost_w = sum gate ds fhat;  dpost_b = sum gate ds
//             dpre_w = sum dx_out shat;  dpre_b = sum dx_out
//
// with N(v) = vhat w + b, vhat = (v - mean) / sqrt(var + eps) (LayerNorm) or
// v / sqrt(mean(v^2) + eps) (RMS), and the row gradient of either
//   N'(v)^T e = (e w - vhat mean(e w vhat) - [LayerNorm] mean(e w)) / sqrt(var + eps).
//
// Bound by memory: the forward reads two rows and writes two, the backward reads
// four and writes two; each row is read once and stays in registers through its
// two or three reductions.  W warps share a row (8 elements a thread and chunk: a
// 16-byte access in bf16), so that a thread's share of the parameter gradients
// stays in registers over all rows its CTA takes; the row sums go through
// shuffles and, between the warps of a row, shared memory.  The next row is
// loaded while a row is worked on.  Parameter gradients: each CTA writes one
// row of partial sums, a second kernel adds the rows in a fixed order, so the
// same inputs give the same bits.
//
// All statistics, sums and products are fp32; only r_out, x_out, dr and df are
// rounded to the storage type, once.  LayerNorm takes the mean first and sums the
// squares of the centred values (no cancellation under a large common offset).
#include "hcw.h"
#include "hcw_internal.h"

#include <math.h>

namespace hcw {

namespace {

constexpr int kNormThreads = 512;   // most threads of a CTA (16 warps on one row)
constexpr int kNormMaxD = 8192;
constexpr int kNormRed = 4;         // sums of one reduction round
constexpr int kNormPar = 4;         // parameter sums of a CTA: post_w, post_b, pre_w, pre_b

struct NormArgs {
    const void* r;        // forward: residual stream or null; backward: dr_out or null
    const void* f;        // branch output or null
    const void* s;        // backward: the stored stream
    const void* dx;       // backward: dx_out or null
    void* o0;             // r_out / dr, or null
    void* o1;             // x_out / df, or null
    const float* gate;    // [groups][d] or null (ones)
    const float* post_w;
    const float* post_b;
    const float* pre_w;
    const float* pre_b;
    float* cpart;         // backward: [grid][kNormPar][d], or null (no parameter gradients)
    float* gpart;         // backward: [groups * slices][d] sums of dgate, or null
    float alpha, eps;
    int T, d;
    int rows_per_gate;    // rows of a group (the last may be shorter)
    int groups, slices;   // an item is one of `slices` runs of rows of a group
    int post, pre;
    int W;                // warps a row
};

// A thread's 8 * NC elements of a row.  VEC (d a multiple of 8): chunk k is the 8 elements
// from 8 (l + 32 W k) on, l the thread's place in the row; else element j is l + 32 W j.
template <typename T, bool VEC, int NC>
struct RowRegs {
    static constexpr int kQ = 8 * NC * (int)sizeof(T) / 16;
    uint4 q[kQ];
    __device__ __forceinline__ static int col(int l, int nl, int j) {
        return VEC ? 8 * (l + nl * (j >> 3)) + (j & 7) : l + nl * j;
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kQ; ++i) q[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void load(const void* base, size_t row, int l, int nl, int d) {
        const T* p = static_cast<const T*>(base) + row * (size_t)d;
        if (VEC) {
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const int c = 8 * (l + nl * k);
#pragma unroll
                for (int i = 0; i < kQ / NC; ++i)
                    q[k * (kQ / NC) + i] = c < d ? reinterpret_cast<const uint4*>(p + c)[i]
                                                 : make_uint4(0u, 0u, 0u, 0u);
            }
        } else {
            uint32_t* w = reinterpret_cast<uint32_t*>(q);
            if (sizeof(T) == 4) {
#pragma unroll
                for (int j = 0; j < 8 * NC; ++j) {
                    const int c = l + nl * j;
                    w[j] = c < d ? reinterpret_cast<const uint32_t*>(p)[c] : 0u;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4 * NC; ++j) {
                    const int c0 = l + nl * 2 * j, c1 = c0 + nl;
                    const uint32_t a = c0 < d ? reinterpret_cast<const unsigned short*>(p)[c0] : 0u;
                    const uint32_t b = c1 < d ? reinterpret_cast<const unsigned short*>(p)[c1] : 0u;
                    w[j] = a | b << 16;
                }
            }
        }
    }
    __device__ __forceinline__ float get(int j) const {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(q);
        if (sizeof(T) == 4) return __uint_as_float(w[j]);
        return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16);
    }
    __device__ __forceinline__ static void store(void* base, size_t row, int l, int nl, int d,
                                                 const float (&v)[8 * NC]) {
        T* p = static_cast<T*>(base) + row * (size_t)d;
#pragma unroll
        for (int k = 0; k < NC; ++k) {
            if (VEC) {
                const int c = 8 * (l + nl * k);
                if (c >= d) continue;
                if (sizeof(T) == 4) {
                    reinterpret_cast<float4*>(p + c)[0] =
                        make_float4(v[8 * k], v[8 * k + 1], v[8 * k + 2], v[8 * k + 3]);
                    reinterpret_cast<float4*>(p + c)[1] =
                        make_float4(v[8 * k + 4], v[8 * k + 5], v[8 * k + 6], v[8 * k + 7]);
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const __nv_bfloat162 h =
                            __floats2bfloat162_rn(v[8 * k + 2 * i], v[8 * k + 2 * i + 1]);
                        w[i] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                    *reinterpret_cast<uint4*>(p + c) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = l + nl * (8 * k + i);
                    if (c >= d) continue;
                    if (sizeof(T) == 4)
                        reinterpret_cast<float*>(p)[c] = v[8 * k + i];
                    else
                        reinterpret_cast<__nv_bfloat16*>(p)[c] = __float2bfloat16_rn(v[8 * k + i]);
                }
            }
        }
    }
};

// The parameter vector at the thread's columns (null: `none` everywhere).
template <bool VEC, int NC>
__device__ __forceinline__ void load_par(float (&v)[8 * NC], const float* p, float none, int l,
                                         int nl, int d) {
#pragma unroll
    for (int j = 0; j < 8 * NC; ++j) {
        const int c = RowRegs<float, VEC, NC>::col(l, nl, j);
        v[j] = c < d ? (p ? p[c] : none) : 0.f;
    }
}

// Sums over a row of N values of each of its threads, on every one of them.  Between the
// warps of a row through red[parity][warp]: the parity alternates from round to round, so a
// round's values are read before the round after the next overwrites them (a barrier of the
// row's warps lies between).
struct RowSum {
    float (*red)[kNormThreads / 32][kNormRed];   // [2][warps of the CTA]
    int parity, W, warp;
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N]) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        if (W == 1) return;
        const int lane = threadIdx.x & 31, first = warp / W * W;
        float(*buf)[kNormRed] = red[parity];
        parity ^= 1;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) buf[warp][i] = v[i];
        asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / W), "r"(32 * W) : "memory");
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.f;
        for (int w = 0; w < W; ++w) {
            const float4 q = *reinterpret_cast<const float4*>(buf[first + w]);
            const float t[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += t[i];
        }
    }
};

// Rows [r0, r1) of an item.
__device__ __forceinline__ void item_rows(const NormArgs& a, int item, int& g, int& r0, int& r1) {
    g = item / a.slices;
    const int first = g * a.rows_per_gate;
    const int n = a.T - first < a.rows_per_gate ? a.T - first : a.rows_per_gate;
    const int len = (n + a.slices - 1) / a.slices;
    const int sl = item - g * a.slices;
    r0 = first + (sl * len < n ? sl * len : n);
    r1 = first + (sl * len < n - len ? sl * len + len : n);
}

// LN: some norm is a LayerNorm (means and centred squares in rounds of their own).
template <typename T, bool VEC, int NC, bool LN>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_kernel(const NormArgs a) {
    __shared__ __align__(16) float red[2][kNormThreads / 32][kNormRed];
    constexpr int E = 8 * NC;
    using Row = RowRegs<T, VEC, NC>;
    const int warp = threadIdx.x >> 5, W = a.W;
    const int nl = 32 * W, l = (int)threadIdx.x % nl;
    const int grp = warp / W, n_grp = (int)(blockDim.x >> 5) / W;
    const float inv_d = 1.f / (float)a.d;
    RowSum rs = {red, 0, W, warp};
    pdl_wait();
    pdl_trigger();
    const int items = a.groups * a.slices;
    float pw[E], pb[E];
    load_par<VEC, NC>(pw, a.pre_w, 1.f, l, nl, a.d);
    load_par<VEC, NC>(pb, LN ? a.pre_b : nullptr, 0.f, l, nl, a.d);
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        int g, r0, r1;
        item_rows(a, item, g, r0, r1);
        float gw[E], gb[E];   // gate * post_w, gate * post_b
        {
            float t[E];
            load_par<VEC, NC>(t, a.gate ? a.gate + (size_t)g * a.d : nullptr, 1.f, l, nl, a.d);
            load_par<VEC, NC>(gw, a.post_w, 1.f, l, nl, a.d);
            load_par<VEC, NC>(gb, LN ? a.post_b : nullptr, 0.f, l, nl, a.d);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                gw[j] *= t[j];
                gb[j] *= t[j];
            }
        }
        Row rr, fr;
        rr.clear();
        fr.clear();
        int row = r0 + grp;
        if (row < r1) {
            if (a.r) rr.load(a.r, row, l, nl, a.d);
            if (a.f) fr.load(a.f, row, l, nl, a.d);
        }
        for (; row < r1; row += n_grp) {
            const Row rc = rr, fc = fr;
            if (row + n_grp < r1) {
                if (a.r) rr.load(a.r, row + n_grp, l, nl, a.d);
                if (a.f) fr.load(a.f, row + n_grp, l, nl, a.d);
            }
            float s[E];
            if (a.f) {
                float mean = 0.f, rstd = 1.f;
                if (LN && a.post == HCW_NORM_LAYER) {
                    float t[1] = {0.f};
#pragma unroll
                    for (int j = 0; j < E; ++j) t[0] += fc.get(j);
                    rs.sum(t);
                    mean = t[0] * inv_d;
                }
                if (a.post != HCW_NORM_NONE) {
                    float t[1] = {0.f};
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float c = Row::col(l, nl, j) < a.d ? fc.get(j) - mean : 0.f;
                        t[0] += c * c;
                    }
                    rs.sum(t);
                    rstd = 1.f / sqrtf(t[0] * inv_d + a.eps);
                }
#pragma unroll
                for (int j = 0; j < E; ++j)
                    s[j] = a.alpha * rc.get(j) + ((fc.get(j) - mean) * rstd * gw[j] + gb[j]);
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) s[j] = a.alpha * rc.get(j);
            }
            if (a.o0) Row::store(a.o0, row, l, nl, a.d, s);
            if (a.o1) {
                float mean = 0.f;
                if (LN && a.pre == HCW_NORM_LAYER) {
                    float t[1] = {0.f};
#pragma unroll
                    for (int j = 0; j < E; ++j) t[0] += s[j];
                    rs.sum(t);
                    mean = t[0] * inv_d;
                }
                float t[1] = {0.f};
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    s[j] = Row::col(l, nl, j) < a.d ? s[j] - mean : 0.f;
                    t[0] += s[j] * s[j];
                }
                rs.sum(t);
                const float rstd = 1.f / sqrtf(t[0] * inv_d + a.eps);
#pragma unroll
                for (int j = 0; j < E; ++j) s[j] = s[j] * rstd * pw[j] + pb[j];
                Row::store(a.o1, row, l, nl, a.d, s);
            }
        }
    }
}

// Adds the row groups' values v of a CTA into group 0's, in group order, through `buf`
// ([n_grp - 1][E][32 W] floats).
template <int E>
__device__ __forceinline__ void group_add(float (&v)[E], float* buf, int grp, int n_grp, int l,
                                          int nl) {
    if (n_grp == 1) return;
    __syncthreads();
    if (grp > 0)
#pragma unroll
        for (int j = 0; j < E; ++j) buf[((size_t)(grp - 1) * E + j) * nl + l] = v[j];
    __syncthreads();
    if (grp == 0)
        for (int q = 0; q < n_grp - 1; ++q)
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] += buf[((size_t)q * E + j) * nl + l];
}

template <typename T, bool VEC, int NC, bool LN>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(const NormArgs a) {
    __shared__ __align__(16) float red[2][kNormThreads / 32][kNormRed];
    extern __shared__ __align__(16) float gbuf[];
    constexpr int E = 8 * NC;
    using Row = RowRegs<T, VEC, NC>;
    const int warp = threadIdx.x >> 5, W = a.W;
    const int nl = 32 * W, l = (int)threadIdx.x % nl;
    const int grp = warp / W, n_grp = (int)(blockDim.x >> 5) / W;
    const float inv_d = 1.f / (float)a.d;
    RowSum rs = {red, 0, W, warp};
    pdl_wait();
    pdl_trigger();
    const int items = a.groups * a.slices;
    float pw[E];
    load_par<VEC, NC>(pw, a.pre_w, 1.f, l, nl, a.d);
    // sums over all of the CTA's rows: gate ds fhat, gate ds, dx shat, dx
    float c_w[E], c_b[E], c_pw[E], c_pb[E];
#pragma unroll
    for (int j = 0; j < E; ++j) c_w[j] = c_b[j] = c_pw[j] = c_pb[j] = 0.f;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        int g, r0, r1;
        item_rows(a, item, g, r0, r1);
        const float* gate = a.gate ? a.gate + (size_t)g * a.d : nullptr;
        float gp[E];   // gate * post_w
        {
            float t[E];
            load_par<VEC, NC>(t, gate, 1.f, l, nl, a.d);
            load_par<VEC, NC>(gp, a.post_w, 1.f, l, nl, a.d);
#pragma unroll
            for (int j = 0; j < E; ++j) gp[j] *= t[j];
        }
        // sums over the item's rows: ds fhat, ds
        float i_w[E], i_b[E];
#pragma unroll
        for (int j = 0; j < E; ++j) i_w[j] = i_b[j] = 0.f;
        Row nr, nf, ns, nx;
        nr.clear();
        nf.clear();
        ns.clear();
        nx.clear();
        auto load = [&](int row) {
            if (a.r) nr.load(a.r, row, l, nl, a.d);
            if (a.f) nf.load(a.f, row, l, nl, a.d);
            if (a.dx) {
                ns.load(a.s, row, l, nl, a.d);
                nx.load(a.dx, row, l, nl, a.d);
            }
        };
        int row = r0 + grp;
        if (row < r1) load(row);
        for (; row < r1; row += n_grp) {
            const Row cr = nr, cf = nf, cs = ns, cx = nx;
            if (row + n_grp < r1) load(row + n_grp);
            float mean_s = 0.f, mean_f = 0.f;
            if (LN) {
                float t[2] = {0.f, 0.f};
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    t[0] += cs.get(j);
                    t[1] += cf.get(j);
                }
                rs.sum(t);
                mean_s = a.pre == HCW_NORM_LAYER ? t[0] * inv_d : 0.f;
                mean_f = a.post == HCW_NORM_LAYER ? t[1] * inv_d : 0.f;
            }
            // sums of (s - mean)^2, (f - mean)^2, e (s - mean), e  with e = dx pre_w
            float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const bool in = Row::col(l, nl, j) < a.d;
                const float sc = in ? cs.get(j) - mean_s : 0.f;
                const float fc = in ? cf.get(j) - mean_f : 0.f;
                const float e = cx.get(j) * pw[j];
                t[0] += sc * sc;
                t[1] += fc * fc;
                t[2] += e * sc;
                t[3] += e;
            }
            rs.sum(t);
            const float rs_s = 1.f / sqrtf(t[0] * inv_d + a.eps);
            const float rs_f = a.post != HCW_NORM_NONE ? 1.f / sqrtf(t[1] * inv_d + a.eps) : 1.f;
            const float m2 = t[2] * inv_d * rs_s;   // mean(e shat)
            const float m1 = LN && a.pre == HCW_NORM_LAYER ? t[3] * inv_d : 0.f;
            float ds[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                ds[j] = cr.get(j);
                if (a.dx) {
                    const float x = cx.get(j);
                    const float sh = (cs.get(j) - mean_s) * rs_s;
                    ds[j] += (x * pw[j] - sh * m2 - m1) * rs_s;
                    c_pw[j] += x * sh;
                    if (LN) c_pb[j] += x;
                }
            }
            if (a.f) {
                float u[2] = {0.f, 0.f};   // sums of h fhat, h  with h = gate ds post_w
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const float fh = (cf.get(j) - mean_f) * rs_f;
                    const float h = ds[j] * gp[j];   // 0 past the row's end
                    i_w[j] += ds[j] * fh;
                    if (LN) i_b[j] += ds[j];
                    u[0] += h * fh;
                    u[1] += h;
                }
                if (a.o1) {
                    if (a.post != HCW_NORM_NONE) rs.sum(u);
                    const float m4 = a.post != HCW_NORM_NONE ? u[0] * inv_d : 0.f;
                    const float m3 = LN && a.post == HCW_NORM_LAYER ? u[1] * inv_d : 0.f;
                    float o[E];
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const float fh = (cf.get(j) - mean_f) * rs_f;
                        o[j] = (ds[j] * gp[j] - fh * m4 - m3) * rs_f;
                    }
                    Row::store(a.o1, row, l, nl, a.d, o);
                }
            }
            if (a.o0) {
#pragma unroll
                for (int j = 0; j < E; ++j) ds[j] *= a.alpha;
                Row::store(a.o0, row, l, nl, a.d, ds);
            }
        }
        if (a.cpart || a.gpart) {
            group_add<E>(i_w, gbuf, grp, n_grp, l, nl);
            if (LN) group_add<E>(i_b, gbuf, grp, n_grp, l, nl);
            if (grp == 0) {
                float t[E], q[E];
                load_par<VEC, NC>(t, gate, 1.f, l, nl, a.d);
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    c_w[j] += t[j] * i_w[j];
                    if (LN) c_b[j] += t[j] * i_b[j];
                }
                if (a.gpart) {   // ds v = ds (fhat post_w + post_b)
                    load_par<VEC, NC>(t, a.post_w, 1.f, l, nl, a.d);
                    load_par<VEC, NC>(q, LN ? a.post_b : nullptr, 0.f, l, nl, a.d);
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const int c = Row::col(l, nl, j);
                        if (c < a.d)
                            a.gpart[(size_t)item * a.d + c] = i_w[j] * t[j] + (LN ? i_b[j] * q[j] : 0.f);
                    }
                }
            }
        }
    }
    if (a.cpart) {
        group_add<E>(c_pw, gbuf, grp, n_grp, l, nl);
        if (LN) group_add<E>(c_pb, gbuf, grp, n_grp, l, nl);
        if (grp == 0) {
            float* out = a.cpart + (size_t)blockIdx.x * kNormPar * a.d;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int c = Row::col(l, nl, j);
                if (c >= a.d) continue;
                out[c] = c_w[j];
                out[(size_t)2 * a.d + c] = c_pw[j];
                if (LN) {
                    out[(size_t)a.d + c] = c_b[j];
                    out[(size_t)3 * a.d + c] = c_pb[j];
                }
            }
        }
    }
}

// Column sums of the partial rows, 32 columns a block, 32 rows at a time, in a fixed order.
// Blocks [0, par * ncb): parameter vector par (out[par], if wanted) over the CTAs' rows;
// then one run of ncb blocks a group: dgate over the group's slices.
struct NormReduceArgs {
    const float* cpart;
    const float* gpart;
    float* out[kNormPar];
    float* dgate;
    int rows;        // rows of cpart
    int slices;      // rows of gpart a group
    int d, ncb;
};

__global__ void __launch_bounds__(1024) norm_reduce_kernel(const NormReduceArgs a) {
    __shared__ float sh[32][33];
    pdl_wait();
    pdl_trigger();
    const int which = (int)(blockIdx.x / a.ncb), cb = (int)(blockIdx.x - (unsigned)which * a.ncb);
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int c = cb * 32 + tx;
    const float* src;
    float* dst;
    size_t ld;
    int rows;
    if (which < kNormPar) {
        if (!a.out[which]) return;
        src = a.cpart + (size_t)which * a.d;
        ld = (size_t)kNormPar * a.d;
        dst = a.out[which];
        rows = a.rows;
    } else {
        const int g = which - kNormPar;
        src = a.gpart + (size_t)g * a.slices * a.d;
        ld = a.d;
        dst = a.dgate + (size_t)g * a.d;
        rows = a.slices;
    }
    float t = 0.f;
    if (c < a.d)
#pragma unroll 4
        for (int r = ty; r < rows; r += 32) t += src[(size_t)r * ld + c];
    sh[ty][tx] = t;
    __syncthreads();
    t = sh[tx][ty];   // row tx of column ty
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    const int co = cb * 32 + ty;
    if (tx == 0 && co < a.d) dst[co] = t;
}

// Warps a row and CTA size for a width.
struct NormPlan {
    int W, threads, nc, grid, slices, groups;
};

int norm_sms() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1)
        return 148;
    return n;
}

int norm_groups(int T, int rows_per_gate) {
    return rows_per_gate > 0 ? (int)(((long long)T + rows_per_gate - 1) / rows_per_gate) : 1;
}

NormPlan norm_plan(int T, int d, int rows_per_gate, int ctas_per_sm) {
    NormPlan p;
    p.nc = d <= 4096 ? 1 : 2;
    p.W = 1;
    while (p.W * 256 * p.nc < d) p.W *= 2;
    p.threads = p.W <= 8 ? 256 : 32 * p.W;
    const int n_grp = p.threads / 32 / p.W;
    p.groups = norm_groups(T, rows_per_gate);
    const int rows = rows_per_gate > 0 && rows_per_gate < T ? rows_per_gate : T;
    const int most = norm_sms() * ctas_per_sm;
    // enough runs of rows for every CTA, each with a row for every row group
    p.slices = p.groups > 0 ? (most + p.groups - 1) / p.groups : 1;
    const int runs = (rows + n_grp - 1) / n_grp;
    if (p.slices > runs) p.slices = runs;
    if (p.slices < 1) p.slices = 1;
    const long long items = (long long)p.groups * p.slices;
    p.grid = (int)(items < most ? items : most);
    return p;
}

template <typename T, bool VEC, int NC, bool LN>
cudaError_t launch_norm(bool bwd, const NormPlan& p, const NormArgs& a, cudaStream_t st) {
    if (!bwd)
        return launch_pdl(norm_fwd_kernel<T, VEC, NC, LN>, dim3(p.grid), dim3(p.threads), 0, st, a);
    const int n_grp = p.threads / 32 / p.W;
    const size_t smem = (size_t)(n_grp - 1) * 8 * NC * 32 * p.W * sizeof(float);
    return launch_pdl(norm_bwd_kernel<T, VEC, NC, LN>, dim3(p.grid), dim3(p.threads), smem, st, a);
}

template <typename T>
cudaError_t launch_norm_any(bool bwd, const NormPlan& p, const NormArgs& a, cudaStream_t st) {
    const bool ln = a.post == HCW_NORM_LAYER || a.pre == HCW_NORM_LAYER;
    const bool vec = a.d % 8 == 0;   // every row starts 16-byte aligned
    if (p.nc == 1)
        return vec ? (ln ? launch_norm<T, true, 1, true>(bwd, p, a, st)
                         : launch_norm<T, true, 1, false>(bwd, p, a, st))
                   : (ln ? launch_norm<T, false, 1, true>(bwd, p, a, st)
                         : launch_norm<T, false, 1, false>(bwd, p, a, st));
    return vec ? (ln ? launch_norm<T, true, 2, true>(bwd, p, a, st)
                     : launch_norm<T, true, 2, false>(bwd, p, a, st))
               : (ln ? launch_norm<T, false, 2, true>(bwd, p, a, st)
                     : launch_norm<T, false, 2, false>(bwd, p, a, st));
}

constexpr int kNormBwdCtas = 2;   // backward CTAs per SM (kNormThreads / 2 threads each)
constexpr int kNormFwdCtas = 4;

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

bool norm_kind(int k) { return k == HCW_NORM_NONE || k == HCW_NORM_RMS || k == HCW_NORM_LAYER; }

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Span {
    const void* p;
    size_t n;
};

bool meet(const Span& a, const Span& b) {
    if (!a.p || !b.p || !a.n || !b.n) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x < y + b.n && y < x + a.n;
}

// Sizes, alignment and overlaps: no output on an input or on another output.
int norm_check(int T, int d, int dtype, int post, int pre, int rows_per_gate, float alpha,
               float eps, const Span* in, int n_in, const Span* out, int n_out) {
    if (T < 0 || d < 1 || rows_per_gate < 0 || !norm_kind(post) || !norm_kind(pre) ||
        !(eps >= 0.f) || !isfinite(eps) || !isfinite(alpha) ||
        (dtype != HCW_BF16 && dtype != HCW_F32))
        return HCW_ERR_INVALID_ARG;
    if (d > kNormMaxD) return HCW_ERR_UNSUPPORTED;
    for (int i = 0; i < n_in; ++i)
        if (!aligned(in[i].p)) return HCW_ERR_ALIGNMENT;
    for (int i = 0; i < n_out; ++i)
        if (!aligned(out[i].p)) return HCW_ERR_ALIGNMENT;
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (meet(out[i], in[j])) return HCW_ERR_ALIASING;
        for (int j = i + 1; j < n_out; ++j)
            if (meet(out[i], out[j])) return HCW_ERR_ALIASING;
    }
    return HCW_OK;
}

// The backward's partial sums: the CTAs' parameter rows, then dgate's rows.
struct NormWs {
    size_t gpart, bytes;
};
NormWs norm_ws(const NormPlan& p, int d) {
    NormWs w;
    w.gpart = round256((size_t)p.grid * kNormPar * d * sizeof(float));
    w.bytes = w.gpart +
              (p.slices > 1 ? round256((size_t)p.groups * p.slices * d * sizeof(float)) : 0);
    return w;
}

}  // namespace

}  // namespace hcw

using namespace hcw;

extern "C" {

int hcw_residual_norm_fwd(const void* r, const void* f, const float* gate, int rows_per_gate,
                          float alpha, int post, const float* post_w, const float* post_b, int pre,
                          const float* pre_w, const float* pre_b, float eps, int T, int d,
                          int dtype, void* r_out, void* x_out, void* stream) {
    const size_t row = (size_t)(T > 0 ? T : 0) * (d > 0 ? d : 0) * (dtype == HCW_F32 ? 4 : 2);
    const size_t vec = (size_t)(d > 0 ? d : 0) * 4;
    const size_t gates = T > 0 ? (size_t)norm_groups(T, rows_per_gate > 0 ? rows_per_gate : 0) : 0;
    const Span in[] = {{r, row}, {f, row}, {gate, gates * vec}, {post_w, vec}, {post_b, vec},
                       {pre_w, vec}, {pre_b, vec}};
    const Span out[] = {{r_out, row}, {x_out, row}};
    const int rc = norm_check(T, d, dtype, post, pre, rows_per_gate, alpha, eps, in, 7, out, 2);
    if (rc) return rc;
    if (x_out && pre == HCW_NORM_NONE) return HCW_ERR_INVALID_ARG;
    if (T == 0) return HCW_OK;
    if ((!r && !f) || (!r_out && !x_out)) return HCW_ERR_INVALID_ARG;
    const NormPlan p = norm_plan(T, d, rows_per_gate, kNormFwdCtas);
    NormArgs a = {};
    a.r = r;
    a.f = f;
    a.o0 = r_out;
    a.o1 = x_out;
    a.gate = gate;
    a.post_w = post == HCW_NORM_NONE ? nullptr : post_w;
    a.post_b = post == HCW_NORM_LAYER ? post_b : nullptr;
    a.pre_w = pre_w;
    a.pre_b = pre == HCW_NORM_LAYER ? pre_b : nullptr;
    a.alpha = alpha;
    a.eps = eps;
    a.T = T;
    a.d = d;
    a.rows_per_gate = rows_per_gate > 0 && rows_per_gate < T ? rows_per_gate : T;
    a.groups = p.groups;
    a.slices = p.slices;
    a.post = f ? post : HCW_NORM_NONE;
    a.pre = x_out ? pre : HCW_NORM_NONE;
    a.W = p.W;
    const cudaStream_t st = (cudaStream_t)stream;
    return count_launch(dtype == HCW_BF16 ? launch_norm_any<__nv_bfloat16>(false, p, a, st)
                                          : launch_norm_any<float>(false, p, a, st), 1);
}

size_t hcw_residual_norm_bwd_workspace_bytes(int T, int d, int rows_per_gate) {
    if (T < 1 || d < 1 || d > kNormMaxD || rows_per_gate < 0) return 0;
    return norm_ws(norm_plan(T, d, rows_per_gate, kNormBwdCtas), d).bytes;
}

int hcw_residual_norm_bwd(const void* dr_out, const void* dx_out, const void* s, const void* f,
                          const float* gate, int rows_per_gate, float alpha, int post,
                          const float* post_w, const float* post_b, int pre, const float* pre_w,
                          float eps, int T, int d, int dtype, void* dr, void* df, float* dgate,
                          float* dpost_w, float* dpost_b, float* dpre_w, float* dpre_b,
                          void* workspace, size_t ws_bytes, void* stream) {
    const size_t row = (size_t)(T > 0 ? T : 0) * (d > 0 ? d : 0) * (dtype == HCW_F32 ? 4 : 2);
    const size_t vec = (size_t)(d > 0 ? d : 0) * 4;
    // a call without rows still writes one gate's gradient when all rows share it
    const size_t gates =
        T > 0 ? (size_t)norm_groups(T, rows_per_gate > 0 ? rows_per_gate : 0) : rows_per_gate ? 0 : 1;
    const Span in[] = {{dr_out, row}, {dx_out, row}, {s, row}, {f, row}, {gate, gates * vec},
                       {post_w, vec}, {post_b, vec}, {pre_w, vec}};
    const Span out[] = {{dr, row}, {df, row}, {dgate, gates * vec}, {dpost_w, vec},
                        {dpost_b, vec}, {dpre_w, vec}, {dpre_b, vec},
                        {workspace, workspace ? ws_bytes : 0}};
    const int rc = norm_check(T, d, dtype, post, pre, rows_per_gate, alpha, eps, in, 8, out, 8);
    if (rc) return rc;
    const bool has_pre = pre != HCW_NORM_NONE, has_post = post != HCW_NORM_NONE;
    if ((dpost_w && !has_post) || (dpost_b && post != HCW_NORM_LAYER) || (dpre_w && !has_pre) ||
        (dpre_b && pre != HCW_NORM_LAYER))
        return HCW_ERR_INVALID_ARG;
    const bool params = dpost_w || dpost_b || dpre_w || dpre_b;
    if (T > 0 && !dr && !df && !dgate && !params) return HCW_ERR_INVALID_ARG;
    const bool branch = df || dgate || dpost_w || dpost_b;
    if (T > 0 && ((!dr_out && !dx_out) || (dx_out && (!s || !has_pre)) ||
                  ((dpre_w || dpre_b) && !dx_out) || (branch && !f)))
        return HCW_ERR_INVALID_ARG;
    const cudaStream_t st = (cudaStream_t)stream;
    NormPlan p = norm_plan(T, d, rows_per_gate, kNormBwdCtas);
    NormWs w = {};
    const bool ws_needed = T > 0 && (params || (dgate && p.slices > 1));
    if (ws_needed) {
        w = norm_ws(p, d);
        if (!workspace || ws_bytes < w.bytes) return HCW_ERR_WORKSPACE;
    }
    float* part = static_cast<float*>(workspace);
    float* gpart = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + w.gpart);
    if (T > 0) {
        NormArgs a = {};
        a.r = dr_out;
        a.f = branch ? f : nullptr;
        a.s = s;
        a.dx = dx_out;
        a.o0 = dr;
        a.o1 = df;
        a.gate = gate;
        a.post_w = has_post ? post_w : nullptr;
        a.post_b = post == HCW_NORM_LAYER ? post_b : nullptr;
        a.pre_w = pre_w;
        a.cpart = params ? part : nullptr;
        a.gpart = dgate ? (p.slices > 1 ? gpart : dgate) : nullptr;
        a.alpha = alpha;
        a.eps = eps;
        a.T = T;
        a.d = d;
        a.rows_per_gate = rows_per_gate > 0 && rows_per_gate < T ? rows_per_gate : T;
        a.groups = p.groups;
        a.slices = p.slices;
        a.post = branch ? post : HCW_NORM_NONE;
        a.pre = dx_out ? pre : HCW_NORM_NONE;
        a.W = p.W;
        const int e = count_launch(dtype == HCW_BF16
                                       ? launch_norm_any<__nv_bfloat16>(true, p, a, st)
                                       : launch_norm_any<float>(true, p, a, st), 1);
        if (e) return e;
    }
    // without rows the sums are zero: the same kernel over no partial rows
    const bool gate_sum = dgate && gates > 0 && (T == 0 || p.slices > 1);
    if (!params && !gate_sum) return HCW_OK;
    NormReduceArgs q = {};
    q.cpart = part;
    q.gpart = gpart;
    q.out[0] = dpost_w;
    q.out[1] = dpost_b;
    q.out[2] = dpre_w;
    q.out[3] = dpre_b;
    q.dgate = dgate;
    q.rows = T > 0 ? p.grid : 0;
    q.slices = T > 0 ? p.slices : 0;
    q.d = d;
    q.ncb = (d + 31) / 32;
    const unsigned blocks =
        (unsigned)q.ncb * (unsigned)(kNormPar + (gate_sum ? (T > 0 ? p.groups : 1) : 0));
    return count_launch(launch_pdl(norm_reduce_kernel, dim3(blocks), dim3(1024), 0, st, q), 1);
}

}  // extern "C"
