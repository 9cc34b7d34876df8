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
// Bound by memory: the forward reads two rows and writes two, the backward reads four and
// writes two.  Runs of consecutive rows are always on their way into a ring in shared memory
// (bulk copies: consecutive rows are one piece, whatever their width and alignment), so the
// reductions of one row never hold up the loads of the next.  A row belongs to `nl`
// threads (16 columns each, in the backward 8 up to 4096 columns: up to 512 and 256 columns no
// two warps share a row), whose columns stay the same from row to row: a thread's share of the
// parameter gradients stays in registers over all rows of its CTA, the parameters in shared
// memory.  The sums of a row go through
// shuffles that halve the number of values at each step and, between the warps of a row,
// through shared memory behind a barrier of those warps.  The arithmetic is in packed pairs (two
// fp32 operations an instruction).  Parameter gradients: each CTA writes one row of partial
// sums, a second kernel adds the rows in a fixed order, so the same inputs give the same
// bits.
//
// All statistics, sums and products are fp32; only r_out, x_out, dr and df are
// rounded to the storage type, once.  LayerNorm takes the mean first and sums the
// squares of the centred values (no cancellation under a large common offset).
#include "hcw.h"
#include "hcw_internal.h"
#include "hcw_ptx.cuh"

#include <math.h>
#include <mutex>

namespace hcw {

namespace {

constexpr int kNormThreads = 512;   // most threads of a CTA
constexpr int kNormMaxD = 8192;
constexpr int kNormPar = 4;         // parameter sums of a CTA: post_w, post_b, pre_w, pre_b
constexpr int kNormRed = 8;         // values of one reduction round
constexpr int kNormCols = 16;       // columns a thread, in parts of 8:
constexpr int kNormPart = 4;        // pairs of a part
// A thread's 16 (8) floats in shared memory are 64 (32) bytes, its 16-byte pieces in an order
// of its own (piece c at c ^ (l / 2 & 3), c ^ (l / 4 & 1)), so that 8 neighbours' accesses to
// one piece fall into different banks.
constexpr int kNormMaxBufs = 8;
constexpr size_t kNormSmem = 232448 - 2048;   // dynamic, beside NormShared
constexpr unsigned long long kNormTimeoutNs = 2000000000ull;

struct NormArgs {
    // the tensors of a ring buffer: forward r, f; backward dr_out, f, s, dx_out (null: not there)
    const void* in[4];
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
    int ln;               // a LayerNorm among them
    int nl;               // threads a row
    int rows;             // rows of a buffer
    int bufs;
    int piece;            // bytes of a tensor in a buffer
    uint32_t starve;      // self-test: thread 0 gives up after so many fetches (0: never)
};

struct __align__(16) NormShared {
    float red[2][kNormThreads / 32][kNormRed];
    float zero[4];
    uint64_t full[kNormMaxBufs], empty[kNormMaxBufs];
    int abort;
};

// Rows [r0, r1) of an item.
__device__ __forceinline__ void item_rows(const NormArgs& a, int item, int& g, int& r0, int& r1) {
    g = item / a.slices;
    const int first = g * a.rows_per_gate;
    // (unsigned: up to slices - 1 more than the rows, of which there may be 2^31 - 1)
    const unsigned n = a.T - first < a.rows_per_gate ? a.T - first : a.rows_per_gate;
    const unsigned len = (n + a.slices - 1) / a.slices;
    const unsigned at = (unsigned)(item - g * a.slices) * len;
    r0 = first + (int)(at < n ? at : n);
    r1 = first + (int)(at < n - len ? at + len : n);
}

// `step` on from i, or to the end
__device__ __forceinline__ int norm_next(int i, int step, int end) {
    return step < end - i ? i + step : end;
}

// The ring's source: thread 0 walks the same items and rows as the CTA works through, up
// to `bufs` buffers ahead.
struct NormFeed {
    int item, row, r1;     // next rows to fetch
    int b;                 // buffer they go to
    uint32_t round;        // how often the ring has been gone through
    size_t at;             // where they start in a tensor, in elements
    uint32_t fetches;
    __device__ __forceinline__ void start(const NormArgs& a) {
        item = blockIdx.x;
        b = 0;
        round = fetches = 0;
        row = r1 = 0;
        if (item < a.groups * a.slices) {
            int g;
            item_rows(a, item, g, row, r1);
        }
        settle(a);
        at = (size_t)row * a.d;
    }
    // on to an item with rows left
    __device__ __forceinline__ void settle(const NormArgs& a) {
        const int items = a.groups * a.slices;
        while (item < items && row >= r1) {
            item = norm_next(item, (int)gridDim.x, items);
            int g;
            if (item < items) item_rows(a, item, g, row, r1);
        }
    }
    // Fetches the next rows into the next buffer, which must be free.  Where it gives up the
    // buffer stays empty, and who waits for it sees `abort`.
    template <typename T, int NIN>
    __device__ __forceinline__ void fetch(const NormArgs& a, uint8_t* ring, NormShared* sh) {
        if (item >= a.groups * a.slices) return;
        if (a.starve && fetches++ >= a.starve) {   // as if the wait below had run out
            atomicExch(&g_error_word, kErrTimeout);
            *(volatile int*)&sh->abort = 1;
            return;
        }
        if (round && !mbar_wait(&sh->empty[b], (round & 1) ^ 1, &sh->abort, kNormTimeoutNs))
            return;
        const int n = r1 - row < a.rows ? r1 - row : a.rows;
        // the 16-byte pieces the rows touch, those wholly inside the tensor in one copy and
        // the last few bytes of the tensor element by element
        const size_t end = (size_t)a.T * a.d * sizeof(T);
        const size_t from = at * sizeof(T) & ~(size_t)15;
        at += (size_t)n * a.d;
        size_t to = (at * sizeof(T) + 15) & ~(size_t)15;
        const bool cut = to > end;
        if (cut) to = end & ~(size_t)15;
        const uint32_t bytes = to > from ? (uint32_t)(to - from) : 0;
        uint8_t* dst = ring + (size_t)b * NIN * a.piece;
        uint32_t total = 0;
#pragma unroll 1
        for (int i = 0; i < NIN; ++i) {
            if (!a.in[i]) continue;
            total += bytes;
            if (cut)
                for (size_t q = from + bytes; q < end; q += sizeof(T))
                    *reinterpret_cast<T*>(dst + (size_t)i * a.piece + (q - from)) =
                        *reinterpret_cast<const T*>(static_cast<const uint8_t*>(a.in[i]) + q);
        }
        mbar_arrive_expect_tx(&sh->full[b], total);
        if (bytes)
#pragma unroll 1
            for (int i = 0; i < NIN; ++i)
                if (a.in[i])
                    asm volatile(
                        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes "
                        "[%0], [%1], %2, [%3];" ::"r"(smem_u32(dst + (size_t)i * a.piece)),
                        "l"(static_cast<const uint8_t*>(a.in[i]) + from), "r"(bytes),
                        "r"(smem_u32(&sh->full[b]))
                        : "memory");
        row += n;
        if (row >= r1) {
            settle(a);
            at = (size_t)row * a.d;
        }
        if (++b == a.bufs) {
            b = 0;
            ++round;
        }
    }
    // Every copy has landed before the CTA leaves, also after giving up.
    __device__ __forceinline__ void drain(const NormArgs& a, NormShared* sh) const {
        for (int i = 0; i < a.bufs; ++i)
            if (round || i < b)
                mbar_wait_drain(&sh->full[i], (i < b ? round : round - 1) & 1, kNormTimeoutNs);
    }
};

// A warp's wait for the rows of buffer b.  false: the warp has given up.  It then takes its part in every later step all the same, without waiting,
// storing or handing buffers back: the other warps of its rows, which may find buffers that
// are full already, meet it at the barrier of each sum, and an item's end is every warp's.
__device__ __forceinline__ bool norm_rows_landed(NormShared& sh, int b, uint32_t round) {
    return __all_sync(0xffffffffu, mbar_wait(&sh.full[b], round & 1, &sh.abort, kNormTimeoutNs));
}

// Shared memory by its 32-bit address.
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 q;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(at));
    return q;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t q;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(q) : "r"(at));
    return q;
}
__device__ __forceinline__ uint32_t lds16(uint32_t at) {
    unsigned short q;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(q) : "r"(at));
    return q;
}

// A thread's E columns of a row, as pairs: VW neighbours at a time, nl threads apart.
template <typename T, int VW, int E>
struct Cols {
    static constexpr int H = E / 2, N = E / VW;   // pairs, runs of neighbours
    static constexpr int B = VW * (int)sizeof(T);   // bytes of a run
    int l, nl, d;
    uint32_t in;             // bit i: run i lies inside the row
    uint32_t zero;           // 16 bytes of zeros in shared memory, read in place of the others
    int at0, gap;            // bytes from a row's start to run 0, and from run to run
    __device__ __forceinline__ Cols(int l_, int nl_, int d_, const void* zero_)
        : l(l_), nl(nl_), d(d_), in(0), zero(smem_u32(zero_)), at0(B * l_), gap(B * nl_) {
#pragma unroll
        for (int i = 0; i < N; ++i) in |= (uint32_t)(col(VW * i) < d) << i;
    }
    __device__ __forceinline__ int col(int j) const { return VW * (l + nl * (j / VW)) + j % VW; }
    __device__ __forceinline__ bool has(int run) const { return in >> run & 1; }
    __device__ __forceinline__ uint32_t run(uint32_t row, int i) const {
        return has(i) ? row + at0 + i * gap : zero;
    }
    // Part k (8 columns) of a row in shared memory, zeros past its end.
    __device__ __forceinline__ void load8(uint64_t (&v)[kNormPart], uint32_t row, int k) const {
        if (sizeof(T) == 2 && VW == 8) {
            const uint4 q = lds128(run(row, k));
            v[0] = bf16x2_to_f32x2(q.x);
            v[1] = bf16x2_to_f32x2(q.y);
            v[2] = bf16x2_to_f32x2(q.z);
            v[3] = bf16x2_to_f32x2(q.w);
        } else if (sizeof(T) == 2 && VW == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = bf16x2_to_f32x2(lds32(run(row, 4 * k + j)));
        } else if (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t x = lds16(run(row, 8 * k + 2 * j)), y = lds16(run(row, 8 * k + 2 * j + 1));
                v[j] = f32x2_pack(__uint_as_float(x << 16), __uint_as_float(y << 16));
            }
        } else if (VW == 4) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint4 q = lds128(run(row, 2 * k + j));
                v[2 * j] = f32x2_pack(__uint_as_float(q.x), __uint_as_float(q.y));
                v[2 * j + 1] = f32x2_pack(__uint_as_float(q.z), __uint_as_float(q.w));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = f32x2_pack(__uint_as_float(lds32(run(row, 8 * k + 2 * j))),
                                  __uint_as_float(lds32(run(row, 8 * k + 2 * j + 1))));
        }
    }
    // Part k of a row of bf16 as it is stored.
    __device__ __forceinline__ void raw8(uint32_t (&v)[kNormPart], uint32_t row, int k) const {
        if (VW == 8) {
            const uint4 q = lds128(run(row, k));
            v[0] = q.x;
            v[1] = q.y;
            v[2] = q.z;
            v[3] = q.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = VW == 2 ? lds32(run(row, 4 * k + j))
                               : lds16(run(row, 8 * k + 2 * j)) |
                                     lds16(run(row, 8 * k + 2 * j + 1)) << 16;
        }
    }
    __device__ __forceinline__ void load(uint64_t (&v)[H], uint32_t row) const {
#pragma unroll
        for (int k = 0; k < H / kNormPart; ++k) {
            uint64_t q[kNormPart];
            load8(q, row, k);
#pragma unroll
            for (int j = 0; j < kNormPart; ++j) v[k * kNormPart + j] = q[j];
        }
    }
    // Part k of row `row` of a global tensor.
    __device__ __forceinline__ void store8(void* base, size_t row, int k,
                                           const uint64_t (&v)[kNormPart]) const {
        T* p = static_cast<T*>(base) + row * (size_t)d;
        auto pack = [&](int i) {
            const float2 f = f32x2_unpack(v[i]);
            return pack_bf16x2(f.x, f.y);
        };
        if (sizeof(T) == 2 && VW == 8) {
            if (has(k))
                *reinterpret_cast<uint4*>(p + col(8 * k)) =
                    make_uint4(pack(0), pack(1), pack(2), pack(3));
        } else if (sizeof(T) == 2 && VW == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (has(4 * k + j)) *reinterpret_cast<uint32_t*>(p + col(8 * k + 2 * j)) = pack(j);
        } else if (VW == 4) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 x = f32x2_unpack(v[2 * j]), y = f32x2_unpack(v[2 * j + 1]);
                if (has(2 * k + j))
                    *reinterpret_cast<float4*>(p + col(8 * k + 4 * j)) = make_float4(x.x, x.y, y.x, y.y);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = f32x2_unpack(v[j]);
                const int i = 8 * k + 2 * j;
                if (sizeof(T) == 2) {
                    __nv_bfloat16* h = reinterpret_cast<__nv_bfloat16*>(p);
                    if (has(i)) h[col(i)] = __float2bfloat16_rn(f.x);
                    if (has(i + 1)) h[col(i + 1)] = __float2bfloat16_rn(f.y);
                } else {
                    float* h = reinterpret_cast<float*>(p);
                    if (has(i)) h[col(i)] = f.x;
                    if (has(i + 1)) h[col(i + 1)] = f.y;
                }
            }
        }
    }
    __device__ __forceinline__ void store(void* base, size_t row, const uint64_t (&v)[H]) const {
#pragma unroll
        for (int k = 0; k < H / kNormPart; ++k) {
            uint64_t q[kNormPart];
#pragma unroll
            for (int j = 0; j < kNormPart; ++j) q[j] = v[k * kNormPart + j];
            store8(base, row, k, q);
        }
    }
    // Address of a thread's own E floats of a vector in shared memory (`i`: its place).
    static constexpr int OWN = E * (int)sizeof(float);
    __device__ __forceinline__ static uint32_t own(const void* vec, int i) {
        return smem_u32(vec) + (uint32_t)(i * OWN + (E == 16 ? (i >> 1 & 3) << 4 : (i >> 2 & 1) << 4));
    }
    __device__ __forceinline__ static uint32_t piece(uint32_t own, int c) {
        return own ^ (uint32_t)(c << 4);
    }
    // The product of a parameter vector (null: `none`) and, if given, another into its own
    // floats, zeros past the row's end.
    __device__ __forceinline__ void fill(uint32_t to, const float* p, const float* q,
                                         float none) const {
        float v[E], w[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int c = col(j);
            v[j] = c < d ? (p ? p[c] : none) : 0.f;
            w[j] = c < d && q ? q[c] : 1.f;
        }
#pragma unroll
        for (int c = 0; c < E / 4; ++c)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(piece(to, c)),
                         "f"(v[4 * c] * w[4 * c]), "f"(v[4 * c + 1] * w[4 * c + 1]),
                         "f"(v[4 * c + 2] * w[4 * c + 2]), "f"(v[4 * c + 3] * w[4 * c + 3])
                         : "memory");
    }
    // part k of own floats
    __device__ __forceinline__ static void fetch8(uint64_t (&v)[kNormPart], uint32_t own, int k) {
#pragma unroll
        for (int j = 0; j < kNormPart / 2; ++j)
            asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];"
                         : "=l"(v[2 * j]), "=l"(v[2 * j + 1])
                         : "r"(piece(own, k * (kNormPart / 2) + j))
                         : "memory");
    }
    __device__ __forceinline__ static void put8(uint32_t own, int k, const uint64_t (&v)[kNormPart]) {
#pragma unroll
        for (int j = 0; j < kNormPart / 2; ++j)
            asm volatile("st.shared.v2.u64 [%0], {%1, %2};" ::"r"(
                             piece(own, k * (kNormPart / 2) + j)),
                         "l"(v[2 * j]), "l"(v[2 * j + 1])
                         : "memory");
    }
    // part k of v - m (past the row's end v stays 0)
    __device__ __forceinline__ void centre8(uint64_t (&v)[kNormPart], float m, int k) const {
#pragma unroll
        for (int j = 0; j < kNormPart; ++j) {
            const int i = 8 * k + 2 * j;
            v[j] = f32x2_add(v[j], f32x2_pack(has(i / VW) ? -m : 0.f, has((i + 1) / VW) ? -m : 0.f));
        }
    }
};

template <int H>
__device__ __forceinline__ void pairs_zero(uint64_t (&v)[H]) {
#pragma unroll
    for (int j = 0; j < H; ++j) v[j] = 0;
}
__device__ __forceinline__ float pair_sum(uint64_t v) {
    const float2 f = f32x2_unpack(v);
    return f.x + f.y;
}
__device__ __forceinline__ uint64_t both(float x) { return f32x2_pack(x, x); }

// Sums of N <= 8 values over the nl threads of a row, on every one of them.
struct RowSum {
    NormShared* sh;
    int nl, warp, lane;
    int parity, W, first;   // warps of the row and the first of them
    __device__ __forceinline__ RowSum(NormShared* sh_, int nl_, int warp_, int lane_)
        : sh(sh_), nl(nl_), warp(warp_), lane(lane_), parity(0), W(nl_ >> 5), first(0) {
        if (W > 1) first = warp / W * W;
    }
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N]) {
        if (nl < 32) {   // several rows in a warp
            for (int o = nl >> 1; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
            return;
        }
        // each step sends half of the values away and takes in the partner's other half;
        // value i ends on the lanes whose upper bits spell it
        constexpr int M = N <= 1 ? 1 : N <= 2 ? 2 : N <= 4 ? 4 : 8;
        float t[M];
#pragma unroll
        for (int i = 0; i < M; ++i) t[i] = i < N ? v[i] : 0.f;
        int o = 16;
#pragma unroll
        for (int m = M >> 1; m > 0; m >>= 1, o >>= 1) {
            const bool up = lane & o;
#pragma unroll
            for (int i = 0; i < m; ++i) {
                const float give = up ? t[i] : t[i + m];
                const float keep = up ? t[i + m] : t[i];
                t[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        }
#pragma unroll
        for (int k = 16 / M; k > 0; k >>= 1) t[0] += __shfl_xor_sync(0xffffffffu, t[0], k);
        // lanes i * (32 / M) .. hold value i
        if (nl == 32) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, t[0], i * (32 / M));
            return;
        }
        // Between the row's warps.  The parity alternates from round to round: a round's
        // values are read before the round after the next overwrites them, a barrier of the
        // row's warps lies between.
        float(*buf)[kNormRed] = sh->red[parity];
        parity ^= 1;
        if ((lane & (32 / M - 1)) == 0) buf[warp][lane / (32 / M)] = t[0];
        asm volatile("bar.sync %0, %1;" ::"r"(1 + first), "r"(nl) : "memory");
        // lane l adds value l % M of every (32 / M)-th warp
        float x = 0.f;
#pragma unroll
        for (int k = 0; k * (32 / M) < kNormThreads / 32; ++k) {
            const int w = lane / M + k * (32 / M);
            if (w < W) x += buf[first + w][lane % M];
        }
#pragma unroll
        for (int k = M; k < 32; k <<= 1) x += __shfl_xor_sync(0xffffffffu, x, k);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, x, i);
    }
};

// LN: some norm is a LayerNorm (means, centred values and biases).  R: rows a row group works
// on at once.  bf16, us and TB/s: 32768 x 4096 RMS 188, 5.7, LayerNorms 182, 5.9; 16384 x 512
// LayerNorms 17, 4.0 (108 rows an SM: a start and an end of about 5 us).
template <typename T, int VW, bool LN, int R>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_kernel(const NormArgs a) {
    extern __shared__ __align__(128) uint8_t norm_smem[];
    __shared__ NormShared sh;
    constexpr int E = kNormCols, H = E / 2, Q = kNormPart;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nt = (int)blockDim.x, nl = a.nl, d = a.d;
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.bufs; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], nt >> 5);
        }
        sh.abort = 0;
        sh.zero[0] = sh.zero[1] = sh.zero[2] = sh.zero[3] = 0.f;
        fence_mbar_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    NormFeed feed;
    if (threadIdx.x == 0) {
        feed.start(a);
        for (int i = 0; i < a.bufs; ++i) feed.fetch<T, 2>(a, norm_smem, &sh);
    }
    const int grp = (int)threadIdx.x / nl, n_grp = nt / nl;
    const float inv_d = 1.f / (float)d;
    const bool has_r = a.in[0], has_f = a.in[1];
    const int first = grp * d * (int)sizeof(T), step = n_grp * d * (int)sizeof(T);
    const int items = a.groups * a.slices;
    RowSum rs(&sh, nl, warp, lane);
    const Cols<T, VW, E> C((int)threadIdx.x % nl, nl, d, sh.zero);
    const uint64_t alpha = both(a.alpha);
    // parameters: pre_w, gate * post_w, pre_b, gate * post_b
    const uint8_t* const par = norm_smem + (size_t)a.bufs * 2 * a.piece;
    const uint32_t pw = C.own(par, C.l), gw = pw + C.OWN * nl, pb = gw + C.OWN * nl,
                   gb = pb + C.OWN * nl;
    int b = 0;
    uint32_t round = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < items; item = norm_next(item, (int)gridDim.x, items)) {
        int g, r0, r1;
        item_rows(a, item, g, r0, r1);
        const float* gate = a.gate ? a.gate + (size_t)g * d : nullptr;
        const bool fresh = item == (int)blockIdx.x;
        if (!fresh) __syncthreads();   // the item before has been worked through
        // a vector a row group: their loads wait side by side
        for (int k = n_grp - 1 - grp; k < (fresh ? 4 : 2); k += n_grp) {
            if (k == 0) C.fill(gw, a.post_w, gate, 1.f);
            if (LN && k == 1) C.fill(gb, a.post_b, a.post_b ? gate : nullptr, 0.f);
            if (k == 2) C.fill(pw, a.pre_w, nullptr, 1.f);
            if (LN && k == 3) C.fill(pb, a.pre_b, nullptr, 0.f);
        }
        __syncthreads();
        for (int row0 = r0; row0 < r1; row0 = norm_next(row0, a.rows, r1)) {
            ok = ok && norm_rows_landed(sh, b, round);
            // a group's rows past the buffer's n hold what was there before: they are worked
            // on and not stored
            const int n = !ok ? 0 : r1 - row0 < a.rows ? r1 - row0 : a.rows;
            const uint32_t buf = smem_u32(norm_smem) + b * 2 * a.piece +
                                 ((uint32_t)row0 * (uint32_t)d * (uint32_t)sizeof(T) & 15) + first;
            uint64_t v[R][H];
            float q[R];
            // mean out of v (a LayerNorm), then 1 / sqrt(mean square + eps) into q
            auto statistics = [&](bool layer) {
                if (LN && layer) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        uint64_t t = v[r][0];
#pragma unroll
                        for (int j = 1; j < H; ++j) t = f32x2_add(t, v[r][j]);
                        q[r] = pair_sum(t);
                    }
                    rs.sum(q);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int k = 0; k < H / Q; ++k) {
                            uint64_t x[Q];
#pragma unroll
                            for (int j = 0; j < Q; ++j) x[j] = v[r][k * Q + j];
                            C.centre8(x, q[r] * inv_d, k);
#pragma unroll
                            for (int j = 0; j < Q; ++j) v[r][k * Q + j] = x[j];
                        }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    uint64_t t = 0;
#pragma unroll
                    for (int j = 0; j < H; ++j) t = f32x2_fma(v[r][j], v[r][j], t);
                    q[r] = pair_sum(t);
                }
                rs.sum(q);
#pragma unroll
                for (int r = 0; r < R; ++r) q[r] = rsqrtf(q[r] * inv_d + a.eps);
            };
#pragma unroll
            for (int r = 0; r < R; ++r) {
                q[r] = 1.f;
                if (has_f)
                    C.load(v[r], buf + a.piece + r * step);
                else
                    pairs_zero(v[r]);
            }
            if (has_f && a.post != HCW_NORM_NONE) statistics(a.post == HCW_NORM_LAYER);
#pragma unroll
            for (int k = 0; k < H / Q; ++k) {
                uint64_t w[Q], wb[Q];
                C.fetch8(w, gw, k);
                if (LN) C.fetch8(wb, gb, k);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    uint64_t x[Q];
                    if (has_r)
                        C.load8(x, buf + r * step, k);
                    else
                        pairs_zero(x);
                    const uint64_t qq = both(q[r]);
#pragma unroll
                    for (int j = 0; j < Q; ++j) {
                        const int i = k * Q + j;
                        uint64_t t = f32x2_mul(x[j], alpha);
                        if (LN) t = f32x2_add(t, wb[j]);
                        v[r][i] = f32x2_fma(f32x2_mul(v[r][i], qq), w[j], t);
                    }
                }
            }
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(&sh.empty[b]);   // the buffer has been read
            if (a.o0)
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (grp + n_grp * r < n) C.store(a.o0, row0 + grp + n_grp * r, v[r]);
            if (a.o1) {
                statistics(a.pre == HCW_NORM_LAYER);
#pragma unroll
                for (int k = 0; k < H / Q; ++k) {
                    uint64_t w[Q], wb[Q];
                    C.fetch8(w, pw, k);
                    if (LN) C.fetch8(wb, pb, k);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const uint64_t qq = both(q[r]);
                        uint64_t x[Q];
#pragma unroll
                        for (int j = 0; j < Q; ++j) {
                            x[j] = f32x2_mul(v[r][k * Q + j], qq);
                            x[j] = LN ? f32x2_fma(x[j], w[j], wb[j]) : f32x2_mul(x[j], w[j]);
                        }
                        if (grp + n_grp * r < n) C.store8(a.o1, row0 + grp + n_grp * r, k, x);
                    }
                }
            }
            if (ok && threadIdx.x == 0) feed.fetch<T, 2>(a, norm_smem, &sh);
            __syncwarp();
            if (++b == a.bufs) {
                b = 0;
                ++round;
            }
        }
    }
    if (threadIdx.x == 0) feed.drain(a, &sh);
}

// The sums of the row groups' values v, in group order, column by column: emit(c, sum) on
// the thread that has column c.  Through `buf` ([n_grp][nl * E] floats, one after the
// other by column).
template <typename C, int H, typename F>
__device__ __forceinline__ void group_sum(const C& cols, const uint64_t (&v)[H], float* buf, int grp,
                                          int n_grp, F emit) {
    const int ld = cols.nl * 2 * H;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < H; ++j) {
        const float2 f = f32x2_unpack(v[j]);
        buf[grp * ld + cols.col(2 * j)] = f.x;
        buf[grp * ld + cols.col(2 * j + 1)] = f.y;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < cols.d; c += blockDim.x) {
        float t = buf[c];
#pragma unroll 4
        for (int g = 1; g < n_grp; ++g) t += buf[g * ld + c];
        emit(c, t);
    }
}

// E columns a thread, R rows a row group works on at once: 8 and 2 where a row then fits the
// CTA, which reads the parameters once for two rows, adds up both rows' sums in one go and has
// two rows' work between waits; 16 and 1 for wider rows.
// SM: with LayerNorms, the sums of dx and ds in shared memory (16 columns' sums have no room in
// the registers; without SM they are there all the same, for rows whose ring leaves no room
// either).
// bf16, with the second launch, us and TB/s: 32768 x 4096 RMS 324, 5.0, LayerNorms 432, 3.7;
// 65536 x 1024 RMS 148, 5.4; 16384 x 512 RMS 27, 3.7, LayerNorms 34, 3.0: bound by waiting, at
// the barriers of the sums, two in sequence (LayerNorms: three), and for shared memory, with the
// 16 warps that the registers allow; about half of the issue slots are used (0.45 to 0.51 a cycle).
template <typename T, int VW, bool LN, bool SM, int E, int R>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(const NormArgs a) {
    extern __shared__ __align__(128) uint8_t norm_smem[];
    __shared__ NormShared sh;
    constexpr int H = E / 2, Q = kNormPart;   // pairs in all, and at a time
    // bf16 rows are read from shared memory once and kept as they are, where the sums leave
    // room in the registers: f, and without LayerNorms s and dx
    constexpr bool KF = sizeof(T) == 2 && E == 8, KX = KF && !LN;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nt = (int)blockDim.x, nl = a.nl, d = a.d;
    // parameters: pre_w, gate * post_w; the sums of dx and ds (SM); the row groups' sums on
    // their way together (through the sums of ds, which are in registers by then)
    const uint8_t* const par = norm_smem + (size_t)a.bufs * 4 * a.piece;
    const uint32_t pw = Cols<T, VW, E>::own(par, (int)threadIdx.x % nl), gp = pw + Cols<T, VW, E>::OWN * nl;
    const uint32_t c_b = Cols<T, VW, E>::own(par + 2 * Cols<T, VW, E>::OWN * nl, threadIdx.x),
                   i_b = c_b + Cols<T, VW, E>::OWN * nt;
    float* const gbuf = reinterpret_cast<float*>(
        norm_smem + (size_t)a.bufs * 4 * a.piece + Cols<T, VW, E>::OWN * (2 * nl + (SM ? nt : 0)));
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.bufs; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], nt >> 5);
        }
        sh.abort = 0;
        sh.zero[0] = sh.zero[1] = sh.zero[2] = sh.zero[3] = 0.f;
        fence_mbar_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    NormFeed feed;
    if (threadIdx.x == 0) {
        feed.start(a);
        for (int i = 0; i < a.bufs; ++i) feed.fetch<T, 4>(a, norm_smem, &sh);
    }
    const int l = (int)threadIdx.x % nl, grp = (int)threadIdx.x / nl, n_grp = nt / nl;
    const float inv_d = 1.f / (float)d;
    const bool has_dr = a.in[0], has_f = a.in[1], has_dx = a.in[3];
    const int first = grp * d * (int)sizeof(T), step = n_grp * d * (int)sizeof(T);
    const int items = a.groups * a.slices;
    RowSum rs(&sh, nl, warp, lane);
    const Cols<T, VW, E> C(l, nl, d, sh.zero);
    // sums over all of the CTA's rows: dx shat, dx
    uint64_t c_w[H];
    pairs_zero(c_w);
    const uint64_t none[Q] = {};
    uint64_t c_r[LN && !SM ? H : 1] = {}, i_r[LN && !SM ? H : 1];   // dx and ds without SM
    if (SM)
#pragma unroll
        for (int k = 0; k < H / Q; ++k) C.put8(c_b, k, none);
    auto own_sums = [&](uint64_t (&v)[H], uint32_t own) {
#pragma unroll
        for (int k = 0; k < H / Q; ++k) {
            uint64_t q[Q];
            C.fetch8(q, own, k);
#pragma unroll
            for (int j = 0; j < Q; ++j) v[k * Q + j] = q[j];
        }
    };
    float* const crow = a.cpart ? a.cpart + (size_t)blockIdx.x * kNormPar * d : nullptr;
    int b = 0;
    uint32_t round = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < items; item = norm_next(item, (int)gridDim.x, items)) {
        int g, r0, r1;
        item_rows(a, item, g, r0, r1);
        const float* gate = a.gate ? a.gate + (size_t)g * d : nullptr;
        const bool fresh = item == (int)blockIdx.x;
        if (!fresh) __syncthreads();   // the item before has been worked through
        for (int k = n_grp - 1 - grp; k < (fresh ? 2 : 1); k += n_grp) {
            if (k == 0) C.fill(gp, a.post_w, gate, 1.f);
            if (k == 1) C.fill(pw, a.pre_w, nullptr, 1.f);
        }
        __syncthreads();
        // sums over the item's rows: ds fhat, ds
        uint64_t i_w[H];
        pairs_zero(i_w);
        if (SM)
#pragma unroll
            for (int k = 0; k < H / Q; ++k) C.put8(i_b, k, none);
        if constexpr (LN && !SM) pairs_zero(i_r);
        for (int row0 = r0; row0 < r1; row0 = norm_next(row0, a.rows, r1)) {
            ok = ok && norm_rows_landed(sh, b, round);
            const int n = !ok ? 0 : r1 - row0 < a.rows ? r1 - row0 : a.rows;
            const uint32_t buf = smem_u32(norm_smem) + b * 4 * a.piece +
                                 ((uint32_t)row0 * (uint32_t)d * (uint32_t)sizeof(T) & 15) + first;
            // 8 columns at a time, in passes over the rows: the sums over the rows take the
            // registers.  A row past the buffer's n reads zeros and has zero factors.
            uint32_t mr[R], mf_[R], mx[R];   // columns to read: dr, f, s and dx
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool in = grp + n_grp * r < n;
                mr[r] = in && has_dr ? C.in : 0u;
                mf_[r] = in && has_f ? C.in : 0u;
                mx[r] = in && has_dx ? C.in : 0u;
            }
            const uint32_t f_row = buf + a.piece, s_row = buf + 2 * a.piece, x_row = buf + 3 * a.piece;
            uint32_t kf[KF ? R : 1][Q], ks[KX ? R : 1][Q], kx[KX ? R : 1][Q];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                Cols<T, VW, E> c = C;
                c.in = mf_[r];
                if constexpr (KF) c.raw8(kf[r], f_row + r * step, 0);
                c.in = mx[r];
                if constexpr (KX) {
                    c.raw8(ks[r], s_row + r * step, 0);
                    c.raw8(kx[r], x_row + r * step, 0);
                }
            }
            // part k of row r
            auto kept = [&](uint64_t (&v)[Q], const uint32_t (&raw)[Q]) {
#pragma unroll
                for (int j = 0; j < Q; ++j) v[j] = bf16x2_to_f32x2(raw[j]);
            };
            auto part = [&](uint64_t (&v)[Q], uint32_t row, uint32_t mask, int r, int k) {
                Cols<T, VW, E> c = C;
                c.in = mask;
                c.load8(v, row + r * step, k);
            };
            auto part_s = [&](uint64_t (&v)[Q], int r, int k) {
                if constexpr (KX) kept(v, ks[r]);
                else part(v, s_row, mx[r], r, k);
            };
            auto part_x = [&](uint64_t (&v)[Q], int r, int k) {
                if constexpr (KX) kept(v, kx[r]);
                else part(v, x_row, mx[r], r, k);
            };
            auto part_f = [&](uint64_t (&v)[Q], int r, int k) {
                if constexpr (KF) kept(v, kf[r]);
                else part(v, f_row, mf_[r], r, k);
            };
            float ms[R] = {}, mf[R] = {};
            if (LN) {
                float t[2 * R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    uint64_t x = 0, y = 0;
#pragma unroll
                    for (int k = 0; k < H / Q; ++k) {
                        uint64_t v[Q];
                        part_s(v, r, k);
#pragma unroll
                        for (int j = 0; j < Q; ++j) x = f32x2_add(x, v[j]);
                        part_f(v, r, k);
#pragma unroll
                        for (int j = 0; j < Q; ++j) y = f32x2_add(y, v[j]);
                    }
                    t[2 * r] = pair_sum(x);
                    t[2 * r + 1] = pair_sum(y);
                }
                rs.sum(t);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    ms[r] = a.pre == HCW_NORM_LAYER ? t[2 * r] * inv_d : 0.f;
                    mf[r] = a.post == HCW_NORM_LAYER ? t[2 * r + 1] * inv_d : 0.f;
                }
            }
            // s or f, centred where its norm is a LayerNorm
            auto centred_s = [&](uint64_t (&v)[Q], int r, int k) {
                part_s(v, r, k);
                if (LN) C.centre8(v, ms[r], k);
            };
            auto centred_f = [&](uint64_t (&v)[Q], int r, int k) {
                part_f(v, r, k);
                if (LN) C.centre8(v, mf[r], k);
            };
            // sums of s^2, e s, f^2, e  with e = dx pre_w
            constexpr int NS = LN ? 4 : 3;
            float t[NS * R];
            {
                uint64_t ss[R] = {}, es[R] = {}, ff[R] = {}, e1[R] = {};
#pragma unroll
                for (int k = 0; k < H / Q; ++k) {
                    uint64_t w[Q];
                    C.fetch8(w, pw, k);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        uint64_t v[Q], x[Q];
                        centred_s(v, r, k);
                        part_x(x, r, k);
#pragma unroll
                        for (int j = 0; j < Q; ++j) {
                            const uint64_t e = f32x2_mul(x[j], w[j]);
                            ss[r] = f32x2_fma(v[j], v[j], ss[r]);
                            es[r] = f32x2_fma(e, v[j], es[r]);
                            if (LN) e1[r] = f32x2_add(e1[r], e);
                        }
                        centred_f(v, r, k);
#pragma unroll
                        for (int j = 0; j < Q; ++j) ff[r] = f32x2_fma(v[j], v[j], ff[r]);
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    t[NS * r] = pair_sum(ss[r]);
                    t[NS * r + 1] = pair_sum(es[r]);
                    t[NS * r + 2] = pair_sum(ff[r]);
                    if (LN) t[NS * r + NS - 1] = pair_sum(e1[r]);
                }
            }
            rs.sum(t);
            float rstd[R], qf[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                rstd[r] = mx[r] ? rsqrtf(t[NS * r] * inv_d + a.eps) : 0.f;
                qf[r] = a.post != HCW_NORM_NONE && mf_[r] ? rsqrtf(t[NS * r + 2] * inv_d + a.eps) : 1.f;
            }
            uint64_t ds[R][H], hf[R] = {}, h1[R] = {};   // sums of h fhat, h  with h = gate ds post_w
#pragma unroll
            for (int k = 0; k < H / Q; ++k) {
                uint64_t w[Q];
                C.fetch8(w, pw, k);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint64_t rr = both(rstd[r]);
                    const uint64_t nm2 = both(-t[NS * r + 1] * inv_d * rstd[r]);   // mean(e shat)
                    const uint64_t nm1 =
                        both(LN && a.pre == HCW_NORM_LAYER ? -t[NS * r + NS - 1] * inv_d : 0.f);
                    uint64_t v[Q], x[Q], g_[Q];
                    Cols<T, VW, E> c = C;
                    c.in = mr[r];
                    c.load8(g_, buf + r * step, k);
                    centred_s(v, r, k);
                    part_x(x, r, k);
#pragma unroll
                    for (int j = 0; j < Q; ++j) {
                        const int i = k * Q + j;
                        const uint64_t h = f32x2_mul(v[j], rr);
                        uint64_t e = f32x2_fma(h, nm2, f32x2_mul(x[j], w[j]));
                        if (LN) e = f32x2_add(e, nm1);
                        c_w[i] = f32x2_fma(x[j], h, c_w[i]);
                        ds[r][i] = f32x2_fma(e, rr, g_[j]);
                    }
                    if constexpr (LN && !SM)
#pragma unroll
                        for (int j = 0; j < Q; ++j) {
                            c_r[k * Q + j] = f32x2_add(c_r[k * Q + j], x[j]);
                            i_r[k * Q + j] = f32x2_add(i_r[k * Q + j], ds[r][k * Q + j]);
                        }
                    if (SM) {
                        uint64_t u[Q];
                        C.fetch8(u, c_b, k);
#pragma unroll
                        for (int j = 0; j < Q; ++j) u[j] = f32x2_add(u[j], x[j]);
                        C.put8(c_b, k, u);
                        C.fetch8(u, i_b, k);
#pragma unroll
                        for (int j = 0; j < Q; ++j) u[j] = f32x2_add(u[j], ds[r][k * Q + j]);
                        C.put8(i_b, k, u);
                    }
                }
            }
            auto read = [&]() {   // the buffer has been read
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(&sh.empty[b]);
            };
            if (KF) read();
#pragma unroll
            for (int k = 0; k < H / Q; ++k) {
                uint64_t w[Q];
                C.fetch8(w, gp, k);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint64_t qq = both(qf[r]);
                    uint64_t v[Q];
                    centred_f(v, r, k);
#pragma unroll
                    for (int j = 0; j < Q; ++j) {
                        const int i = k * Q + j;
                        const uint64_t fh = f32x2_mul(v[j], qq);
                        const uint64_t h = f32x2_mul(ds[r][i], w[j]);   // 0 past the row's end
                        i_w[i] = f32x2_fma(ds[r][i], fh, i_w[i]);
                        hf[r] = f32x2_fma(h, fh, hf[r]);
                        if (LN) h1[r] = f32x2_add(h1[r], h);
                    }
                }
            }
            if (a.o1) {
                constexpr int NU = LN ? 2 : 1;
                float u[NU * R] = {};
                if (a.post != HCW_NORM_NONE) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        u[NU * r] = pair_sum(hf[r]);
                        if (LN) u[NU * r + NU - 1] = pair_sum(h1[r]);
                    }
                    rs.sum(u);
                }
#pragma unroll
                for (int k = 0; k < H / Q; ++k) {
                    uint64_t w[Q];
                    C.fetch8(w, gp, k);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const uint64_t qq = both(qf[r]);
                        // fhat mean(h fhat) = f qf mean
                        const uint64_t n4 = both(-u[NU * r] * inv_d * qf[r]);
                        const uint64_t n3 = both(
                            LN && a.post == HCW_NORM_LAYER ? -u[NU * r + NU - 1] * inv_d : 0.f);
                        uint64_t v[Q];
                        centred_f(v, r, k);
#pragma unroll
                        for (int j = 0; j < Q; ++j) {
                            uint64_t o = f32x2_fma(v[j], n4, f32x2_mul(ds[r][k * Q + j], w[j]));
                            if (LN) o = f32x2_add(o, n3);
                            v[j] = f32x2_mul(o, qq);
                        }
                        if (grp + n_grp * r < n) C.store8(a.o1, row0 + grp + n_grp * r, k, v);
                    }
                }
            }
            if (!KF) read();
            if (a.o0) {
                const uint64_t alpha = both(a.alpha);
#pragma unroll
                for (int k = 0; k < H / Q; ++k)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        uint64_t v[Q];
#pragma unroll
                        for (int j = 0; j < Q; ++j) v[j] = f32x2_mul(ds[r][k * Q + j], alpha);
                        if (grp + n_grp * r < n) C.store8(a.o0, row0 + grp + n_grp * r, k, v);
                    }
            }
            if (ok && threadIdx.x == 0) feed.fetch<T, 4>(a, norm_smem, &sh);
            __syncwarp();
            if (++b == a.bufs) {
                b = 0;
                ++round;
            }
        }
        if (a.cpart || a.gpart) {
            // the CTA's sums of gate ds fhat and gate ds build up in its partial row; dgate's of
            // ds v = ds (fhat post_w + post_b) are the item's alone
            float* const grow = a.gpart ? a.gpart + (size_t)item * d : nullptr;
            uint64_t b_[H];
            if (SM) own_sums(b_, i_b);
            group_sum(C, i_w, gbuf, grp, n_grp, [&](int c, float v) {
                if (crow) crow[c] = (fresh ? 0.f : crow[c]) + (gate ? gate[c] : 1.f) * v;
                if (grow) grow[c] = v * (a.post_w ? a.post_w[c] : 1.f);
            });
            if (LN) {
                if constexpr (LN && !SM)
#pragma unroll
                    for (int j = 0; j < H; ++j) b_[j] = i_r[j];
                group_sum(C, b_, gbuf, grp, n_grp, [&](int c, float v) {
                    if (crow) crow[d + c] = (fresh ? 0.f : crow[d + c]) + (gate ? gate[c] : 1.f) * v;
                    if (grow && a.post_b) grow[c] += v * a.post_b[c];
                });
            }
        }
    }
    if (crow) {
        uint64_t b_[H];
        if (SM) own_sums(b_, c_b);
        group_sum(C, c_w, gbuf, grp, n_grp, [&](int c, float v) { crow[(size_t)2 * d + c] = v; });
        if (LN) {
            if constexpr (LN && !SM)
#pragma unroll
                for (int j = 0; j < H; ++j) b_[j] = c_r[j];
            group_sum(C, b_, gbuf, grp, n_grp, [&](int c, float v) { crow[(size_t)3 * d + c] = v; });
        }
    }
    if (threadIdx.x == 0) feed.drain(a, &sh);
}

// Column sums of the partial rows, in a fixed order, by blocks of 1024 threads: 32 columns and 32
// rows at a time, or up to 32 rows by more columns.  Blocks [0, kNormPar * ncb): parameter vector
// (out[], if wanted) over the CTAs' rows; then a run of ncg blocks a group: dgate over the
// group's slices.
struct NormReduceArgs {
    const float* cpart;
    const float* gpart;
    float* out[kNormPar];
    float* dgate;
    int rows;        // rows of cpart
    int slices;      // rows of gpart a group
    int d;
    int ncb, ncg;    // column blocks of a vector
    int c_log2, g_log2;   // columns of a block
};
constexpr int kReduceThreads = 1024;   // 1 << 10

__global__ void __launch_bounds__(kReduceThreads) norm_reduce_kernel(const NormReduceArgs a) {
    __shared__ float sh[32 * 33];
    pdl_wait();
    pdl_trigger();
    const bool par = (int)blockIdx.x < kNormPar * a.ncb;
    const int b = par ? blockIdx.x : (int)blockIdx.x - kNormPar * a.ncb, nc = par ? a.ncb : a.ncg;
    const int which = b / nc, cb = b - which * nc;
    const int log2 = par ? a.c_log2 : a.g_log2, tx = threadIdx.x & ((1 << log2) - 1);
    const int ty = threadIdx.x >> log2, step = kReduceThreads >> log2;
    const int c = (cb << log2) + tx;
    const float* src;
    float* dst;
    size_t ld;
    int rows;
    if (par) {
        if (!a.out[which]) return;
        src = a.cpart + (size_t)which * a.d;
        ld = (size_t)kNormPar * a.d;
        dst = a.out[which];
        rows = a.rows;
    } else {
        src = a.gpart + (size_t)which * a.slices * a.d;
        ld = a.d;
        dst = a.dgate + (size_t)which * a.d;
        rows = a.slices;
    }
    float t = 0.f;
    if (c < a.d)
#pragma unroll 4
        for (int r = ty; r < rows; r += step) t += src[(size_t)r * ld + c];
    if (log2 == 5) {
        sh[ty * 33 + tx] = t;
        __syncthreads();
        t = sh[tx * 33 + ty];   // row tx of column ty
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        const int co = (cb << 5) + ty;
        if (tx == 0 && co < a.d) dst[co] = t;
        return;
    }
    if (step > 1) {
        sh[threadIdx.x] = t;
        __syncthreads();
        if (ty) return;
        for (int k = 1; k < step; ++k) t += sh[(k << log2) + tx];
    }
    if (c < a.d) dst[c] = t;
}

// Columns (their log2) of a block that adds so many rows: 8 rows a thread at most up to 32 rows.
// (4099 x 777 fp32, 8 slices of 17 groups: the backward 29.0 us with 32 columns, 27.2 so.)
int reduce_cols(int rows) { return rows > 32 ? 5 : rows > 16 ? 8 : rows > 8 ? 9 : 10; }

// Threads a row and a CTA, buffers and items for a call.
struct NormPlan {
    bool ln, sm;
    int cols;   // columns a thread
    int nl, threads, grid, slices, groups;
    int rows, bufs, piece;
    size_t smem;
};

int norm_groups(int T, int rows_per_gate) {
    return rows_per_gate > 0 ? (int)(((long long)T + rows_per_gate - 1) / rows_per_gate) : 1;
}

constexpr int kNormPerCta = 8;   // items a CTA takes of groups that are cut, at most

// rows a row group works on at once in the forward, and in the backward with 8 columns a thread
constexpr int kNormRows = 2;

// elem: bytes of an element, ln: a LayerNorm (grid, slices and groups depend on neither).
NormPlan norm_plan(bool bwd, bool ln, int T, int d, int elem, int rows_per_gate) {
    NormPlan p;
    p.ln = ln;
    p.cols = bwd && d <= kNormThreads * kNormCols / 2 ? kNormCols / 2 : kNormCols;
    const int sms = device_sms(), E = p.cols;
    // a power of two up to a warp, whole warps above
    p.nl = 8;
    while (p.nl < 32 && p.nl * E < d) p.nl *= 2;
    if (p.nl * E < d) p.nl = (d + 32 * E - 1) / (32 * E) * 32;
    // one CTA an SM, row groups of 512 threads in all; fewer where the rows do not go round,
    // but whole warps
    int n_grp = p.nl < kNormThreads ? kNormThreads / p.nl : 1;
    const int least = p.nl < 32 ? 32 / p.nl : 1, share = (int)(((long long)T + sms - 1) / sms);
    while (n_grp / 2 >= least && n_grp / 2 >= share) n_grp /= 2;
    p.threads = n_grp * p.nl;
    const int n_in = bwd ? 4 : 2;
    int r = bwd && E == kNormCols ? 1 : kNormRows;
    const size_t vec = (size_t)E * sizeof(float) * p.nl;
    size_t fixed = !bwd ? (ln ? 4 : 2) * vec : (2 + (ln && E == kNormCols ? 2 : 1) * n_grp) * vec;
    auto piece = [&](int rows) { return (int)(((size_t)rows * d * elem + 32 + 127) / 128 * 128); };
    p.sm = bwd && ln && E == kNormCols;
    if (p.sm && fixed + (size_t)n_in * piece(n_grp) > kNormSmem) {
        p.sm = false;
        fixed = (2 + n_grp) * vec;
    }
    const size_t room = kNormSmem - fixed;
    // One row a group where the ring would have but one buffer of two rows and other groups
    // fill its waits (forward of 16384 x 2048 fp32, LayerNorms, 4 groups: 102 -> 89 us; of
    // 16384 x 8192 bf16, one group: 290 -> 323), or not one buffer.  (The backward's second
    // row is then past the buffer's rows.)
    while (r > 1 && (size_t)n_in * piece(n_grp * r) * (bwd || n_grp == 1 ? 1 : 2) > room) r /= 2;
    p.rows = n_grp * r;
    p.piece = piece(p.rows);
    p.bufs = (int)(room / ((size_t)n_in * p.piece));
    if (p.bufs > 4) p.bufs = 4;
    if (p.bufs < 1) p.bufs = 1;
    p.smem = (size_t)p.bufs * n_in * p.piece + fixed;
    p.groups = norm_groups(T, rows_per_gate);
    const int rows = rows_per_gate > 0 && rows_per_gate < T ? rows_per_gate : T;
    const int most = sms;
    // Runs of rows of a group: as many as make the busiest CTA's work least, in row groups'
    // steps and 4 steps a run; for each number of runs a CTA takes, the shortest runs.
    p.slices = 1;
    if (p.groups > 0) {
        long long best = -1;
        const int runs = rows > 0 ? (int)(((long long)rows + n_grp - 1) / n_grp) : 1;
        for (int per = 1; per <= kNormPerCta; ++per) {
            long long k = (long long)most * per / p.groups;
            k = k < 1 ? 1 : k < runs ? k : runs;
            const long long busiest = (p.groups * k + most - 1) / most;
            const long long len = ((rows + k - 1) / k + n_grp - 1) / n_grp;
            if (best < 0 || busiest * (len + 4) < best) {
                best = busiest * (len + 4);
                p.slices = (int)k;
            }
            if (k == runs) break;
        }
    }
    const long long items = (long long)p.groups * p.slices;
    p.grid = (int)(items < most ? items : most);
    return p;
}

template <typename T, int VW, bool LN>
cudaError_t launch_norm(bool bwd, const NormPlan& p, const NormArgs& a, cudaStream_t st) {
    auto kern = !bwd                    ? (p.rows * p.nl > p.threads ? norm_fwd_kernel<T, VW, LN, kNormRows>
                                                                     : norm_fwd_kernel<T, VW, LN, 1>)
                : p.cols == kNormCols ? norm_bwd_kernel<T, VW, LN, LN, kNormCols, 1>
                                      : norm_bwd_kernel<T, VW, LN, false, kNormCols / 2, kNormRows>;
    int which = !bwd ? (p.rows * p.nl > p.threads ? 0 : 4) : p.cols == kNormCols ? 1 : 2;
    // (a row of bf16 always leaves the sums room: 192 KB in all at 8192 columns)
    if constexpr (LN && sizeof(T) == 4)
        if (which == 1 && !p.sm) {
            kern = norm_bwd_kernel<T, VW, LN, false, kNormCols, 1>;
            which = 3;
        }
    static std::once_flag once[64][5];
    static cudaError_t set_err[64][5];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::call_once(once[dev][which], [&] {
        set_err[dev][which] = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)kNormSmem);
    });
    if (set_err[dev][which] != cudaSuccess) return set_err[dev][which];
    return launch_pdl(kern, dim3((unsigned)p.grid), dim3((unsigned)p.threads), p.smem, st, a);
}

template <typename T, int VW>
cudaError_t launch_norm_vw(bool bwd, const NormPlan& p, const NormArgs& a, cudaStream_t st) {
    const bool ln = a.ln;
    return ln ? launch_norm<T, VW, true>(bwd, p, a, st) : launch_norm<T, VW, false>(bwd, p, a, st);
}

// The widest access every row's start allows.
cudaError_t launch_norm_any(bool bwd, int dtype, const NormPlan& p, const NormArgs& a,
                            cudaStream_t st) {
    if (dtype == HCW_F32)
        return a.d % 4 == 0 ? launch_norm_vw<float, 4>(bwd, p, a, st)
                            : launch_norm_vw<float, 1>(bwd, p, a, st);
    return a.d % 8 == 0   ? launch_norm_vw<__nv_bfloat16, 8>(bwd, p, a, st)
           : a.d % 2 == 0 ? launch_norm_vw<__nv_bfloat16, 2>(bwd, p, a, st)
                          : launch_norm_vw<__nv_bfloat16, 1>(bwd, p, a, st);
}

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

std::atomic<int> g_starve{0};

void norm_geometry(NormArgs& a, const NormPlan& p) {
    a.starve = (uint32_t)g_starve.load(std::memory_order_relaxed);
    a.ln = p.ln;
    a.nl = p.nl;
    a.rows = p.rows;
    a.bufs = p.bufs;
    a.piece = p.piece;
}

// The backward's partial sums (of a size that does not depend on the type: the plan's grid
// and slices do not): the CTAs' parameter rows, then dgate's rows.
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

// The most of that for up to T rows (a workspace for the longest batch does for every shorter
// one, whose groups may be cut where the longest's are not): a partial row a CTA, of which
// there are no more than SMs or than items, and no more items than the groups have rows; and a
// row for every item of groups that are cut, of which each CTA takes kNormPerCta.
size_t norm_ws_up_to(int T, int d, int rows_per_gate) {
    const int rows = rows_per_gate > 0 && rows_per_gate < T ? rows_per_gate : T;
    const long long all = (long long)norm_groups(T, rows_per_gate) * rows, sms = device_sms();
    const long long ctas = all < sms ? all : sms, most = sms * kNormPerCta;
    return round256((size_t)ctas * kNormPar * d * sizeof(float)) +
           (rows > 1 ? round256((size_t)(all < most ? all : most) * d * sizeof(float)) : 0);
}

}  // namespace

cudaError_t norm_error_word_read_clear(int* word) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(word, g_error_word, sizeof(int));
    if (e == cudaSuccess && *word) e = cudaMemcpyToSymbol(g_error_word, &zero, sizeof(int));
    return e;
}

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
    // without a branch there is nothing that its gate and its norm's parameters apply to
    if (!f) {
        post = HCW_NORM_NONE;
        gate = nullptr;
    }
    const NormPlan p = norm_plan(false, post == HCW_NORM_LAYER || pre == HCW_NORM_LAYER, T, d,
                                 dtype == HCW_F32 ? 4 : 2, rows_per_gate);
    NormArgs a = {};
    a.in[0] = r;
    a.in[1] = f;
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
    a.post = post;
    a.pre = x_out ? pre : HCW_NORM_NONE;
    norm_geometry(a, p);
    return count_launch(launch_norm_any(false, dtype, p, a, (cudaStream_t)stream), 1);
}

int hcw_selftest_norm_starve(int fetches) { return g_starve.exchange(fetches > 0 ? fetches : 0); }

size_t hcw_residual_norm_bwd_workspace_bytes(int T, int d, int rows_per_gate) {
    if (T < 1 || d < 1 || d > kNormMaxD || rows_per_gate < 0) return 0;
    return norm_ws_up_to(T, d, rows_per_gate);
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
    NormPlan p = norm_plan(true, post == HCW_NORM_LAYER || pre == HCW_NORM_LAYER, T, d,
                           dtype == HCW_F32 ? 4 : 2, rows_per_gate);
    NormWs w = {};
    const bool ws_needed = T > 0 && (params || (dgate && p.slices > 1));
    if (ws_needed) {
        w = norm_ws(p, d);
        if (!workspace || ws_bytes < norm_ws_up_to(T, d, rows_per_gate) || ws_bytes < w.bytes)
            return HCW_ERR_WORKSPACE;
    }
    float* part = static_cast<float*>(workspace);
    float* gpart = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + w.gpart);
    if (T > 0) {
        NormArgs a = {};
        a.in[0] = dr_out;
        a.in[1] = branch ? f : nullptr;
        a.in[2] = dx_out ? s : nullptr;
        a.in[3] = dx_out;
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
        norm_geometry(a, p);
        const int e = count_launch(launch_norm_any(true, dtype, p, a, st), 1);
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
    q.c_log2 = reduce_cols(q.rows);
    q.g_log2 = reduce_cols(q.slices);
    q.ncb = (d + (1 << q.c_log2) - 1) >> q.c_log2;
    q.ncg = (d + (1 << q.g_log2) - 1) >> q.g_log2;
    const unsigned blocks = (unsigned)q.ncb * kNormPar +
                            (unsigned)q.ncg * (gate_sum ? (unsigned)(T > 0 ? p.groups : 1) : 0u);
    return count_launch(
        launch_pdl(norm_reduce_kernel, dim3(blocks), dim3(kReduceThreads), 0, st, q), 1);
}

}  // extern "C"
