// hcw_embed.cu -- the lookup of symbols (hcw_embed_fwd) and its gradient (hcw_embed_bwd):
//
//   x_t = scale E[id_t]                         (zeros for a negative id)
//   dE_v (+)= scale sum over {t: id_t = v} of dx_t
//
// Both are bound by memory: the lookup reads and writes T rows, the gradient reads T rows and
// writes V (or, added to what is there, reads and writes the rows that are named).
//
// Text names a few symbols thousands of times and most of them never, so the gradient goes by the
// sorted tokens: the positions in the order of their symbols, cut into chunks of equal length.  A CTA
// takes a chunk for a block of columns, each of its 8 warps adds an eighth of the rows, and the warps'
// sums of a symbol that lies in several of them are joined in shared memory.  A symbol whose positions
// lie in one chunk is written there; one that reaches over a chunk's end leaves a partial sum in the
// workspace at each, and a last launch adds these in the order of the chunks.  No atomics on
// numbers: the order of every sum depends on the ids and the sizes alone.
//
// The sort is one launch.  Each CTA, or some CTAs together, own a range of symbols and go through all
// ids: they count those of smaller symbols, where their own begin in the sorted order, and their own
// by symbol.  The rows of symbols that do not occur are zeroed on the way, by bulk copies.
#include "hcw.h"
#include "hcw_internal.h"
#include "hcw_ptx.cuh"

#include <algorithm>
#include <mutex>

namespace hcw {

namespace {

constexpr int kErrInvalid = 1;            // HCW_ERR_INVALID_ARG in the error word
constexpr int kSortWarps = 32;
constexpr int kSortThreads = 32 * kSortWarps;
constexpr int kDigits = 256;              // values of a sorting pass's digit
constexpr int kMaxRange = 65536;          // symbols of a CTA: two passes, 8 KB of flags
constexpr int kMaxV = 1 << 23;
constexpr int kMaxD = 1 << 20;
constexpr int kSumWarps = 8;
constexpr int kZeroBytes = 4096;          // of a bulk copy of zeros at most
constexpr int kLongRow = 512;             // bytes of a row that a warp zeroes on its own

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A row's elements as a warp takes them, 16 bytes a lane in loads of W bytes: 16 where the rows lie
// on 16 bytes, else as much as all of them lie on (4, or 2 for bf16 rows of odd width).
template <int W>
struct Raw;
template <>
struct Raw<16> {
    using type = uint4;
};
template <>
struct Raw<4> {
    using type = uint32_t;
};
template <>
struct Raw<2> {
    using type = unsigned short;
};
template <typename T, int W>
struct Cols {
    static constexpr int E = 16 / sizeof(T);   // elements of a lane, of 32 E
    static constexpr int P = W / sizeof(T);    // neighbours among them
    static constexpr int L = E / P;            // loads
    static __device__ __forceinline__ int at(int lane, int e) { return (lane + 32 * (e / P)) * P + e % P; }
};

// A lane's elements of a row on their way, as they lie there.  `left`: elements of the row from the
// block's first one, a multiple of P; what would lie behind them is the last P again (loads under a
// condition waited one for another: gradient of 65536 tokens, 32000 x 1023 fp32, 259 us, without 101).
template <typename T, int W>
struct Row {
    using C = Cols<T, W>;
    typename Raw<W>::type q[C::L];
    __device__ __forceinline__ void load(const T* p, int lane, int left) {
#pragma unroll
        for (int l = 0; l < C::L; ++l)
            q[l] = *reinterpret_cast<const typename Raw<W>::type*>(p + min((lane + 32 * l) * C::P, left - C::P));
    }
    __device__ __forceinline__ void get(float (&v)[C::E]) const {
        if constexpr (W == 16) {
            const uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
#pragma unroll
            for (int e = 0; e < C::E; ++e) v[e] = part(w[e * sizeof(T) / 4], e);
        } else {
#pragma unroll
            for (int e = 0; e < C::E; ++e) v[e] = part(q[e / C::P], e);
        }
    }
    // element e of the row in the word that holds it
    __device__ __forceinline__ static float part(uint32_t w, int e) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w);
        return __uint_as_float(W != 2 && (e & 1) ? w & 0xffff0000u : w << 16);
    }
};

// P neighbours of a row of type O: 16 bytes at a time at most.
template <int P>
__device__ __forceinline__ void get_piece(const float* p, float* v) {
    if constexpr (P >= 4) {
#pragma unroll
        for (int i = 0; i < P / 4; ++i) {
            const float4 q = reinterpret_cast<const float4*>(p)[i];
            v[4 * i] = q.x;
            v[4 * i + 1] = q.y;
            v[4 * i + 2] = q.z;
            v[4 * i + 3] = q.w;
        }
    } else if constexpr (P == 2) {
        const float2 q = *reinterpret_cast<const float2*>(p);
        v[0] = q.x;
        v[1] = q.y;
    } else {
        v[0] = p[0];
    }
}
template <int P>
__device__ __forceinline__ void get_piece(const __nv_bfloat16* p, float* v) {
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = to_f32(p[i]);
}
template <int P>
__device__ __forceinline__ void put_piece(float* p, const float* v) {
    if constexpr (P >= 4) {
#pragma unroll
        for (int i = 0; i < P / 4; ++i)
            reinterpret_cast<float4*>(p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else if constexpr (P == 2) {
        *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
    } else {
        p[0] = v[0];
    }
}
template <int P>
__device__ __forceinline__ void put_piece(__nv_bfloat16* p, const float* v) {
    if constexpr (P == 8)
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                  pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    else if constexpr (P == 4)
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    else if constexpr (P == 2)
        *reinterpret_cast<uint32_t*>(p) = pack_bf16x2(v[0], v[1]);
    else
        put(p, v[0]);
}
// The lane's elements of an output row (of type O, rounded here).
template <typename C, typename O>
__device__ __forceinline__ void store_row(O* p, int lane, int left, const float (&v)[C::E]) {
#pragma unroll
    for (int l = 0; l < C::L; ++l) {
        const int j = (lane + 32 * l) * C::P;
        if (j < left) put_piece<C::P>(p + j, v + l * C::P);
    }
}
template <typename C, typename O>
__device__ __forceinline__ void load_out(const O* p, int lane, int left, float (&v)[C::E]) {
#pragma unroll
    for (int l = 0; l < C::L; ++l) get_piece<C::P>(p + min((lane + 32 * l) * C::P, left - C::P), v + l * C::P);
}

// ------------------------------------------------------------------ lookup
// A warp takes R rows, 32 E columns of them: all R rows' loads on their way at once, as nothing but
// memory bounds it (65536 of 131072 x 2048 bf16: 56 us, 6.2 TB/s of rows read and written; 64 of
// 32000 x 512, where the wait for a row after its id counts: 1.2 us).
template <typename T, int W, int R>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const int* ids, const T* table, long long T_,
                                                        int V, int d, float scale, T* x) {
    using C = Cols<T, W>;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const long long row0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * R;
    const int col = blockIdx.y * (32 * C::E);
    int id[R];
#pragma unroll
    for (int r = 0; r < R; ++r) id[r] = row0 + r < T_ ? ids[row0 + r] : -1;
    Row<T, W> q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (id[r] >= V) {
            if (lane == 0) atomicExch(&g_error_word, kErrInvalid);
            id[r] = -1;
        }
        q[r].load(table + (size_t)max(id[r], 0) * d + col, lane, d - col);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (row0 + r >= T_) break;
        float v[C::E];
        q[r].get(v);
#pragma unroll
        for (int e = 0; e < C::E; ++e) v[e] = id[r] >= 0 ? v[e] * scale : 0.f;
        store_row<C>(x + (size_t)(row0 + r) * d + col, lane, d - col, v);
    }
}

// ------------------------------------------------------------------ the sorted tokens
struct SortArgs {
    const int* ids;
    int T, V, range;          // symbols of a CTA, or of several that share them
    int* key[3];              // [T] symbols and [T] positions: two for the passes, and the sorted ones
    int* pos[3];
    int* count;               // tokens that name a symbol
    void* dE;                 // null: no zeros
    size_t row_bytes;
};

// The ids i .. i + 3, i a multiple of four; -1 from `end` on.
__device__ __forceinline__ void ids_at(const int* ids, long long i, long long end, int (&id)[4]) {
    if (i + 3 < end && (reinterpret_cast<uintptr_t>(ids) & 15) == 0) {
        const int4 q = *reinterpret_cast<const int4*>(ids + i);
        id[0] = q.x;
        id[1] = q.y;
        id[2] = q.z;
        id[3] = q.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) id[e] = i + e < end ? ids[i + e] : -1;
    }
}

// Exclusive prefix of v over the block's threads; the total in *total.
__device__ __forceinline__ int block_prefix(int v, int* scratch, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
    }
    __syncthreads();   // scratch's last use
    if (lane == 31) scratch[warp] = s;
    __syncthreads();
    int w = scratch[lane];   // every warp: the warps' sums, added up
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += u;
    }
    *total = __shfl_sync(0xffffffffu, w, 31);
    const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return (warp ? before : 0) + s - v;
}

// Starts bytes of zeros at p, on 16-byte boundaries both.
__device__ __forceinline__ void bulk_zeros(char* p, size_t bytes, const uint4* source) {
    for (size_t at = 0; at < bytes; at += kZeroBytes)
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(p + at),
                     "r"(smem_u32(source)),
                     "r"((uint32_t)(bytes - at < kZeroBytes ? bytes - at : kZeroBytes))
                     : "memory");
}

// `warps` warps, this one being the w-th: start the zeros of the rows of [z0, z1) that are not named
// (flags from symbol lo on).  Rows of whole 32-byte sectors by bulk copies, a row a lane
// (1000 tokens, 131072 x 16 fp32: 14 us, by plain stores 27; 2^20 x 16: 25 against 130).  Others of
// kLongRow bytes or more by plain stores, a row a warp (4099 tokens, 32003 x 777 fp32: 39 us, by bulk
// copies between 16-byte boundaries 41, when the sums took 9 more than now); shorter ones by bulk copies
// again, 8 rows a lane with those next to one another as one piece (1000 tokens, 131072 x 9 fp32: 19 us,
// by plain stores 27; 2^20 x 9: 27 against 125; from 131072 x 201 on plain stores win, 30 against 34).
__device__ __forceinline__ void start_zeros(const SortArgs& a, int z0, int z1, int lo,
                                            const uint32_t* named, const uint4* source, int w, int warps) {
    const auto is_named = [&](int v) { return named[(v - lo) >> 5] >> ((v - lo) & 31) & 1; };
    const int lane = threadIdx.x & 31;
    char* const rows = static_cast<char*>(a.dE);
    if (a.row_bytes % 32 == 0) {
        for (int v = z0 + 32 * w + lane; v < z1; v += 32 * warps)
            if (!is_named(v)) bulk_zeros(rows + (size_t)v * a.row_bytes, a.row_bytes, source);
    } else if (a.row_bytes >= kLongRow) {
        for (int v = z0 + w; v < z1; v += warps) {
            if (is_named(v)) continue;
            char* const p = rows + (size_t)v * a.row_bytes;
            char* const end = p + a.row_bytes;
            char* const in = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(p) + 15) & ~(uintptr_t)15);
            char* const out = reinterpret_cast<char*>(reinterpret_cast<uintptr_t>(end) & ~(uintptr_t)15);
            if (p + 2 * lane < in) *reinterpret_cast<short*>(p + 2 * lane) = 0;
            for (char* q = in + 16 * lane; q < out; q += 512) *reinterpret_cast<uint4*>(q) = make_uint4(0, 0, 0, 0);
            if (out + 2 * lane < end) *reinterpret_cast<short*>(out + 2 * lane) = 0;
        }
    } else {
        for (int v0 = z0 + 8 * (32 * w + lane); v0 < z1; v0 += 8 * 32 * warps) {
            const int v1 = min(v0 + 8, z1);
            for (int v = v0; v < v1; ++v) {
                if (is_named(v)) continue;
                char* p = rows + (size_t)v * a.row_bytes;
                while (v + 1 < v1 && !is_named(v + 1)) ++v;
                char* const end = rows + (size_t)(v + 1) * a.row_bytes;
                for (; p < end && (reinterpret_cast<uintptr_t>(p) & 15); p += 2) *reinterpret_cast<short*>(p) = 0;
                const size_t whole = (size_t)(end - p) & ~(size_t)15;
                bulk_zeros(p, whole, source);
                for (p += whole; p < end; p += 2) *reinterpret_cast<short*>(p) = 0;
            }
        }
    }
    bulk_commit();
}

// A warp goes through the tokens [w0, w1), four a lane at a time: counts those of the range's symbols.
// Returns how many of the lane's have a smaller symbol.
__device__ __forceinline__ int count_tokens(const SortArgs& a, long long w0, long long w1, int lo, int hi,
                                            int* tally) {
    const int lane = threadIdx.x & 31;
    int below = 0;
    for (long long i0 = w0; i0 < w1; i0 += 512) {
        int id[4][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) ids_at(a.ids, i0 + 128 * q + 4 * lane, w1, id[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = id[q][e];
                below += v >= 0 && v < lo;
                if (v >= lo && v < hi) atomicAdd(&tally[v - lo], 1);
                if (v >= a.V) atomicExch(&g_error_word, kErrInvalid);
            }
    }
    return below;
}

// A warp goes through them again, 32 at a time, and puts each where the range's tallies say.
__device__ __forceinline__ void place_tokens(const SortArgs& a, long long w0, long long w1, int lo, int hi,
                                             int* tally) {
    const int lane = threadIdx.x & 31;
    for (long long i0 = w0; i0 < w1; i0 += 512) {
        int id[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) id[q] = i0 + 32 * q + lane < w1 ? a.ids[i0 + 32 * q + lane] : -1;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const bool in = id[q] >= lo && id[q] < hi;
            if (!__any_sync(0xffffffffu, in)) continue;
            const uint32_t same = __match_any_sync(0xffffffffu, in ? id[q] : -1);
            const int rank = __popc(same & ((1u << lane) - 1));
            const int to = in ? tally[id[q] - lo] + rank : 0;
            __syncwarp();
            if (in && rank == 0) tally[id[q] - lo] += __popc(same);
            __syncwarp();
            if (in) {
                a.key[2][to] = id[q];
                a.pos[2][to] = (int)(i0 + 32 * q + lane);
            }
        }
    }
}

// Where a range's counts fit into shared memory.  A range has kSplit CTAs, each with the runs of
// kOwn warps (a frequent symbol's tokens would keep one CTA busy long after the others).  Each counts, for
// every symbol of the range, the tokens before its runs, in each of them and after them: so it knows
// where those of each run go, and the run's warp puts them there, 32 at a time.  All ids pass through
// every CTA, from L2: 64 KB for 16384 tokens, which take 8.7 us under the profiler with 201 symbols, most
// of them launch, barriers and loads that wait for one another, and with 32000 and the zeros of 65 MB 15.5.
constexpr int kSplit = 8, kOwn = kSortWarps / kSplit, kTallies = kOwn + 2;

__global__ void __launch_bounds__(kSortThreads) embed_place_kernel(const SortArgs a) {
    extern __shared__ int counts[];                 // [kTallies][range]: before, own .., after
    __shared__ int scratch[kSortWarps];
    __shared__ __align__(16) uint4 source[kZeroBytes / 16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, range = a.range;
    uint32_t* const named = reinterpret_cast<uint32_t*>(counts + kTallies * range);
    if (threadIdx.x < kZeroBytes / 16) source[threadIdx.x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();   // before the barriers that come first, for the bulk copies that read them
    for (int i = threadIdx.x; i < kTallies * range; i += kSortThreads) counts[i] = 0;
    pdl_wait();
    pdl_trigger();
    const int lo = blockIdx.x / kSplit * range, hi = min(a.V, lo + range);
    const int part = blockIdx.x % kSplit, own = warp - part * kOwn;
    int* const tally = counts + (own < 0 ? 0 : own < kOwn ? 1 + own : kOwn + 1) * range;
    __syncthreads();
    // each warp goes through a run of ids, four a lane at a time
    const int run = ((a.T + kSortThreads - 1) / kSortThreads * 32 + 127) / 128 * 128;   // of a warp
    const long long w0 = (long long)warp * run, w1 = min((long long)a.T, w0 + run);
    const int below = count_tokens(a, w0, w1, lo, hi, tally);
    int base, all;
    (void)block_prefix(below, scratch, &base);   // (and the counts are complete)
    const int per = (range + kSortThreads - 1) / kSortThreads;
    const int v0 = min((int)threadIdx.x * per, range), v1 = min(v0 + per, range);
    int total = 0;
    for (int v = v0; v < v1; ++v)
#pragma unroll
        for (int k = 0; k < kTallies; ++k) total += counts[k * range + v];
    for (int i = threadIdx.x; i < (range + 31) / 32 * 32; i += kSortThreads) {
        int any = 0;
#pragma unroll
        for (int k = 0; k < kTallies; ++k) any |= i < range ? counts[k * range + i] : 0;
        const uint32_t word = __ballot_sync(0xffffffffu, any != 0);
        if (lane == 0) named[i >> 5] = word;
    }
    int at = base + block_prefix(total, scratch, &all);
    for (int v = v0; v < v1; ++v) {
#pragma unroll
        for (int k = 0; k < kTallies; ++k) {   // the first place of the symbol's tokens in each part
            const int c = counts[k * range + v];
            counts[k * range + v] = at;
            at += c;
        }
    }
    if (threadIdx.x == 0 && hi == a.V && part == 0) *a.count = base + all;
    __syncthreads();
    if (own >= 0 && own < kOwn) {
        place_tokens(a, w0, w1, lo, hi, tally);
    } else if (a.dE) {
        // the other warps: zeros; the CTAs of a range share its rows
        const int share = (range + kSplit - 1) / kSplit;
        const int z0 = min(lo + part * share, hi), z1 = min(z0 + share, hi);
        start_zeros(a, z0, z1, lo, named, source, own < 0 ? warp : warp - kOwn, kSortWarps - kOwn);
        bulk_wait<0>();
    }
}

// The same for many tokens, where what takes the time is that each of 152 CTAs goes through all of them
// (65536: 22 us, 262144: 68).  A cluster of kCluster CTAs has a range, each of its CTAs a part of the
// tokens; they count those of kRuns runs of neighbours each and read each other's sums.  The gradient of
// 65536 tokens, 32000 x 1024 bf16: 71 us, without clusters 75; 500 x 128: 27 and 36; 262144 tokens, 201 x
// 512: 97 and 133.  Few tokens wait longer for the cluster than for the counts (4096 tokens, 201 x 512: 13.2
// and 12.4; 16384 the same).  Of 8 CTAs fewer clusters run at once, which the zeros feel (16384
// tokens, 32000 x 512: 34, of 4 29).
constexpr int kCluster = 4, kRuns = 16;

__device__ __forceinline__ int from_cta(const int* p, int rank) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(p, rank)) : "memory");
    return v;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kSortThreads)
    embed_place_cluster_kernel(const SortArgs a) {
    extern __shared__ int counts[];                 // [kRuns][range], then the sums, [range] each:
    __shared__ int scratch[kSortWarps];
    __shared__ int below_here;
    __shared__ __align__(16) uint4 source[kZeroBytes / 16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, range = a.range;
    int* const here = counts + kRuns * range;       // of this CTA's tokens
    int* const all = here + range;                  // of all tokens
    int* const before = all + range;                // of those of the CTAs before this one
    uint32_t* const named = reinterpret_cast<uint32_t*>(before + range);
    if (threadIdx.x < kZeroBytes / 16) source[threadIdx.x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();   // before the barriers that come first, for the bulk copies that read them
    for (int i = threadIdx.x; i < kRuns * range; i += kSortThreads) counts[i] = 0;
    pdl_wait();
    pdl_trigger();
    const int part = (int)cluster_ctarank();
    const int lo = blockIdx.x / kCluster * range, hi = min(a.V, lo + range);
    __syncthreads();
    // a warp's share of the tokens (a multiple of four), of which a run has several
    const long long share = ((a.T + kCluster * kSortWarps - 1) / (kCluster * kSortWarps) + 3) & ~3;
    constexpr int kShares = kSortWarps / kRuns;
    const long long first = part * kSortWarps * share;
    const int below = count_tokens(a, first + warp * share, min((long long)a.T, first + (warp + 1) * share), lo,
                                   hi, counts + warp / kShares * range);
    int base, sum;
    (void)block_prefix(below, scratch, &base);   // (and the counts are complete)
    if (threadIdx.x == 0) below_here = base;
    for (int v = threadIdx.x; v < range; v += kSortThreads) {
        int n = 0;
#pragma unroll
        for (int k = 0; k < kRuns; ++k) n += counts[k * range + v];
        here[v] = n;
    }
    cluster_sync_all();
    base = lane < kCluster ? from_cta(&below_here, lane) : 0;
    for (int v = threadIdx.x; v < range; v += kSortThreads) {
        int n = 0, ahead = 0;
#pragma unroll
        for (int q = 0; q < kCluster; ++q) {
            const int c = from_cta(here + v, q);
            n += c;
            ahead += q < part ? c : 0;
        }
        all[v] = n;
        before[v] = ahead;
    }
    // (the others' sums have been read; a CTA leaves once its own have been)
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) base += __shfl_xor_sync(0xffffffffu, base, o);
    __syncthreads();
    for (int i = threadIdx.x; i < (range + 31) / 32 * 32; i += kSortThreads) {
        const uint32_t word = __ballot_sync(0xffffffffu, i < range && all[i] != 0);
        if (lane == 0) named[i >> 5] = word;
    }
    const int per = (range + kSortThreads - 1) / kSortThreads;
    const int v0 = min((int)threadIdx.x * per, range), v1 = min(v0 + per, range);
    int total = 0;
    for (int v = v0; v < v1; ++v) total += all[v];
    int at = base + block_prefix(total, scratch, &sum);
    for (int v = v0; v < v1; ++v) {
        int to = at + before[v];
#pragma unroll
        for (int k = 0; k < kRuns; ++k) {   // the first place of the symbol's tokens in each run
            const int c = counts[k * range + v];
            counts[k * range + v] = to;
            to += c;
        }
        at += all[v];
    }
    if (threadIdx.x == 0 && hi == a.V && part == 0) *a.count = base + sum;
    __syncthreads();
    if (warp < kRuns) {
        const long long w0 = first + warp * kShares * share;
        place_tokens(a, w0, min((long long)a.T, w0 + kShares * share), lo, hi, counts + warp * range);
    } else if (a.dE) {
        // the other warps: zeros; the CTAs of a cluster share the range's rows
        const int rows = (range + kCluster - 1) / kCluster;
        const int z0 = min(lo + part * rows, hi), z1 = min(z0 + rows, hi);
        start_zeros(a, z0, z1, lo, named, source, warp - kRuns, kSortWarps - kRuns);
        bulk_wait<0>();
    }
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// For larger vocabularies: a CTA a range, which collects its own in their order and sorts them, 8 bits
// of the symbol in each of two passes, each warp counting and placing a run of them.  The first range has
// most of a text's tokens, and its CTA is the last one: 65536 tokens of 262144 symbols take 147 us, whatever
// the width (2048 columns bf16: 405 us for the whole gradient, of 357 for its bytes; 512: 184 of 89).
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const SortArgs a) {
    __shared__ __align__(16) int hist[kDigits * kSortWarps];
    __shared__ uint32_t named[kMaxRange / 32];
    __shared__ int scratch[kSortWarps];
    __shared__ __align__(16) uint4 source[kZeroBytes / 16];
    if (threadIdx.x < kZeroBytes / 16) source[threadIdx.x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();   // before the barriers that come first, for the bulk copies that read them
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int lo = blockIdx.x * a.range, hi = min(a.V, lo + a.range);
    for (int i = threadIdx.x; i < (a.range + 31) / 32; i += kSortThreads) named[i] = 0;
    __syncthreads();
    // each warp goes through a run of ids, four a lane at a time
    const int run = ((a.T + kSortThreads - 1) / kSortThreads * 32 + 127) / 128 * 128;   // of a warp
    const long long w0 = (long long)warp * run, w1 = min((long long)a.T, w0 + run);
    int below = 0, mine = 0;
    for (long long i0 = w0; i0 < w1; i0 += 512) {
        int id[4][4];
#pragma unroll
        for (int q = 0; q < 4; ++q) ids_at(a.ids, i0 + 128 * q + 4 * lane, w1, id[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = id[q][e];
                below += v >= 0 && v < lo;
                if (v >= lo && v < hi) {
                    ++mine;
                    // (a frequent symbol is looked for before it is marked again)
                    const uint32_t bit = 1u << ((v - lo) & 31);
                    if (!(*(volatile uint32_t*)&named[(v - lo) >> 5] & bit)) atomicOr(&named[(v - lo) >> 5], bit);
                }
                if (v >= a.V) atomicExch(&g_error_word, kErrInvalid);
            }
    }
    int m, base;
    (void)block_prefix(below, scratch, &base);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    int at = block_prefix(lane == 0 ? mine : 0, scratch, &m);
    at = __shfl_sync(0xffffffffu, at, 0);
    if (threadIdx.x == 0 && hi == a.V) *a.count = base + m;
    // (the prefixes above were behind a barrier: the flags are complete)
    if (a.dE) start_zeros(a, lo, hi, lo, named, source, warp, kSortWarps);
    // its own, in order
    if (m > 0) {
        int *key = a.key[0] + base, *pos = a.pos[0] + base;
        int *key_to = a.key[1] + base, *pos_to = a.pos[1] + base;
        for (long long i0 = w0; i0 < w1; i0 += 512) {
            int id[4][4];
#pragma unroll
            for (int q = 0; q < 4; ++q) ids_at(a.ids, i0 + 128 * q + 4 * lane, w1, id[q]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bool in[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) in[e] = id[q][e] >= lo && id[q][e] < hi;
                if (!__any_sync(0xffffffffu, in[0] || in[1] || in[2] || in[3])) continue;
                uint32_t have[4];
                int before = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    have[e] = __ballot_sync(0xffffffffu, in[e]);
                    before += __popc(have[e] & ((1u << lane) - 1));
                }
                int k = at + before;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (in[e]) {
                        key[k] = id[q][e];
                        pos[k] = (int)(i0 + 128 * q + 4 * lane + e);
                        ++k;
                    }
                    at += __popc(have[e]);
                }
            }
        }
        const int own = ((m + kSortThreads - 1) / kSortThreads) * 32;   // of a warp
        const int m0 = min(m, warp * own), m1 = min(m, m0 + own);
        for (int shift = 0; shift < 16; shift += 8) {
            const bool last = shift == 8;
            // (8 counters a thread, two vectors)
            static_assert(kDigits * kSortWarps == 8 * kSortThreads, "a thread's counters");
            int4* const my = reinterpret_cast<int4*>(hist) + 2 * threadIdx.x;
            my[0] = my[1] = make_int4(0, 0, 0, 0);
            __syncthreads();   // and the list is there
            for (int i = m0 + lane; i < m1; i += 32)
                atomicAdd(&hist[(((key[i] - lo) >> shift) & (kDigits - 1)) * kSortWarps + warp], 1);
            __syncthreads();
            // places: by digit, then by warp
            const int4 c = my[0], e = my[1];
            int all, p = block_prefix(c.x + c.y + c.z + c.w + e.x + e.y + e.z + e.w, scratch, &all);
            const int q = p + c.x + c.y + c.z + c.w;
            my[0] = make_int4(p, p + c.x, p + c.x + c.y, p + c.x + c.y + c.z);
            my[1] = make_int4(q, q + e.x, q + e.x + e.y, q + e.x + e.y + e.z);
            __syncthreads();
            for (int i0 = m0; i0 < m1; i0 += 32) {
                const int i = i0 + lane;
                const bool on = i < m1;
                const int k = on ? key[i] : 0, t = on ? pos[i] : 0;
                const int d = on ? ((k - lo) >> shift) & (kDigits - 1) : kDigits;
                const uint32_t same = __match_any_sync(0xffffffffu, d);
                const int rank = __popc(same & ((1u << lane) - 1));
                const int place = on ? hist[d * kSortWarps + warp] + rank : 0;
                __syncwarp();
                if (on && rank == 0) hist[d * kSortWarps + warp] += __popc(same);
                __syncwarp();
                if (on) {
                    (last ? a.key[2] + base : key_to)[place] = k;
                    (last ? a.pos[2] + base : pos_to)[place] = t;
                }
            }
            __syncthreads();
            int* t = key;
            key = key_to;
            key_to = t;
            t = pos;
            pos = pos_to;
            pos_to = t;
        }
    }
    bulk_wait<0>();   // the zeros
}

// ------------------------------------------------------------------ the sums
struct SumArgs {
    const int* key;       // the sorted tokens: symbols and positions
    const int* pos;
    const int* count;
    const void* dx;
    void* dE;
    float* part;          // [chunks][2][d]: of the run that came in from before, and of the one that goes on
    int d, T;
    int chunk_log2;       // tokens of a chunk
    int tiles;            // blocks of columns
    float scale;
    int add;
};

// Writes a symbol's sum: scale sum, or that on top of what is there, rounded once.
template <typename C, typename O>
__device__ __forceinline__ void write_sum(const SumArgs& a, int symbol, int col, int lane,
                                          const float (&s)[C::E]) {
    O* row = static_cast<O*>(a.dE) + (size_t)symbol * a.d + col;
    const int left = a.d - col;
    float v[C::E];
    if (a.add) {
        load_out<C>(row, lane, left, v);
#pragma unroll
        for (int e = 0; e < C::E; ++e) v[e] = fmaf(a.scale, s[e], v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < C::E; ++e) v[e] = a.scale * s[e];
    }
    store_row<C>(row, lane, left, v);
}

// A CTA adds the rows of one chunk, 32 E columns of them, each warp an eighth: at most 32 rows, in an
// order that the lanes hold, 8 of them on their way at once in registers (65536 tokens, 32000 x 1024
// bf16: 75 us for the whole gradient; with chunks of 64 tokens throughout 7 more).
template <typename T, typename O, int W>
__global__ void __launch_bounds__(32 * kSumWarps) embed_sum_kernel(const SumArgs a) {
    using C = Cols<T, W>;
    constexpr int E = C::E;
    __shared__ __align__(16) float head[kSumWarps][32 * E], tail[kSumWarps][32 * E];
    __shared__ int state[kSumWarps], head_symbol[kSumWarps];
    constexpr int kRows = W == 2 ? 4 : 8;   // on their way at once
    // of a warp: has a run that came in from before it, which goes on behind it; another one that does
    constexpr int kFrom = 1, kThrough = 2, kOn = 4;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int chunk = blockIdx.x / a.tiles, col = blockIdx.x % a.tiles * (32 * E);
    const long long chunk0 = (long long)chunk << a.chunk_log2;
    const int share = 1 << (a.chunk_log2 - 3);   // a warp's, 32 at most
    const long long first = chunk0 + warp * share;
    // everything that depends on the place alone (behind the count the lists hold nothing of use)
    const int count = *a.count;
    const int at = (int)min(first + lane, (long long)a.T - 1);
    int key = a.key[at];
    const int pos = a.pos[at];
    const int before = first > 0 && first - 1 < a.T ? a.key[first - 1] : -1;
    const int behind = first + share < a.T ? a.key[first + share] : -1;
    if (chunk0 >= count) return;
    const int n = (int)max(0ll, min((long long)share, count - first));
    const T* dx = static_cast<const T*>(a.dx) + col;
    const int left = a.d - col;
    if (n > 0) {
        if (lane >= n) key = -1;
        const int after = first + n < count ? behind : -1;
        float s[E];
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] = 0.f;
        const int first_symbol = __shfl_sync(0xffffffffu, key, 0);
        bool from_before = first > 0 && first_symbol == before;
        int flags = 0;
        // the lanes whose symbol is another one behind them
        int next = __shfl_down_sync(0xffffffffu, key, 1);
        if (lane + 1 >= n) next = after;
        const uint32_t last = __ballot_sync(0xffffffffu, lane < n && (next != key || lane + 1 == n));
        for (int r0 = 0; r0 < n; r0 += kRows) {
            Row<T, W> q[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {   // (past the chunk's last row that one again)
                const int t = __shfl_sync(0xffffffffu, pos, min(r0 + r, n - 1));
                q[r].load(dx + (size_t)t * a.d, lane, left);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                if (r0 + r >= n) break;
                float v[E];
                q[r].get(v);
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] += v[e];
                if (!(last >> (r0 + r) & 1)) continue;
                const int symbol = __shfl_sync(0xffffffffu, key, r0 + r);
                const bool goes_on = r0 + r + 1 == n && after == symbol;
                if (from_before || goes_on) {
                    float* const to = from_before ? head[warp] : tail[warp];
                    flags |= from_before ? (goes_on ? kFrom | kThrough : kFrom) : kOn;
#pragma unroll
                    for (int e = 0; e < E; ++e) to[C::at(lane, e)] = s[e];
                } else {
                    write_sum<C, O>(a, symbol, col, lane, s);
                }
                from_before = false;
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] = 0.f;
            }
        }
        if (lane == 0) {
            state[warp] = flags;
            head_symbol[warp] = first_symbol;
        }
    } else if (lane == 0) {
        state[warp] = 0;
    }
    __syncthreads();
    // a thread a column: the runs over several warps, or over an end of the chunk
    const int c = threadIdx.x;
    if (c >= 32 * E || c >= left) return;
    float* const part = a.part + (size_t)chunk * 2 * a.d + col + c;
    float s = 0.f;
    bool open = state[0] & kFrom, came = open;   // a run is under way, and was before the chunk
    for (int w = 0; w < kSumWarps; ++w) {
        const int f = state[w];
        if (f & kFrom) {
            s += head[w][c];
            if (!(f & kThrough)) {
                if (came) {
                    part[0] = s;
                } else {
                    O* const to = static_cast<O*>(a.dE) + (size_t)head_symbol[w] * a.d + col + c;
                    put(to, a.add ? fmaf(a.scale, s, to_f32(*to)) : a.scale * s);
                }
                open = came = false;
            }
        }
        if (f & kOn) {
            s = tail[w][c];
            open = true;
        }
    }
    if (open) part[came ? 0 : a.d] = s;
}

// A run over several chunks: TEAM warps of the chunk it starts in add the parts, in order, each warp eight
// or its share of them, eight on their way at once (no chunk's CTA can do it, as none knows when the
// others are done).  Eight warps where the symbols' runs fill a chunk on average (the gradient of 16384
// tokens, 201 x 512 bf16: 16.9 us, with one warp 18.1; 262144 tokens 133, with one 148); one where most chunks
// have none to join (65536 tokens, 131072 x 2048: 243, with eight 248).
template <typename T, typename O, int W, int TEAM>
__global__ void __launch_bounds__(32 * kSumWarps) embed_join_kernel(const SumArgs a) {
    static_assert(TEAM == 1 || TEAM == kSumWarps, "a warp or a CTA for a run");
    using C = Cols<T, W>;
    constexpr int E = C::E;
    __shared__ float sums[TEAM][32 * E];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part_of = TEAM > 1 ? warp : 0;
    const long long item = TEAM > 1 ? (long long)blockIdx.x : (long long)blockIdx.x * kSumWarps + warp;
    const int chunk = (int)(item / a.tiles), col = (int)(item % a.tiles) * (32 * E);
    const int count = *a.count;
    const int size = 1 << a.chunk_log2;
    const long long first = (long long)chunk << a.chunk_log2;
    if (first + size >= a.T) return;   // no chunk behind it
    const int symbol = a.key[first + size - 1], behind = a.key[first + size], start = a.key[first],
              before = first > 0 ? a.key[first - 1] : -1;
    // the symbols around the ends of the 32 chunks from the from-th behind it on (behind the count the list
    // holds nothing of use); the first ones at once with those above, where they are needed as a rule
    int k[2];
    const auto ends = [&](int from) {
        const long long end = min(first + (long long)size * (from + lane + 2), (long long)a.T - 1);
        k[0] = a.key[end - 1];
        k[1] = a.key[end];
    };
    if (TEAM > 1) ends(0);
    if (first + size >= count || behind != symbol) return;
    if (first > 0 && start == symbol && before == symbol) return;   // started before
    if (TEAM == 1) ends(0);
    // the chunks behind it that the run reaches into
    int more = 0;
    for (;;) {
        const bool on = first + (long long)size * (more + lane + 2) < count && k[0] == symbol && k[1] == symbol;
        const uint32_t stop = __ballot_sync(0xffffffffu, !on);
        if (stop) {
            more += __ffs(stop);
            break;
        }
        more += 32;
        ends(more);
    }
    const int left = a.d - col;
    const float* part = a.part + ((size_t)chunk * 2 * a.d + col);
    float s[E];
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = 0.f;
    if (part_of == 0) load_out<C>(part + a.d, lane, left, s);
    const int share = TEAM > 1 ? max(8, (more + TEAM - 1) / TEAM) : more;
    const int j1 = min(more, (part_of + 1) * share);
    for (int j0 = part_of * share; j0 < j1; j0 += 8) {
        float v[8][E];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            load_out<C>(part + (size_t)(min(j0 + j, j1 - 1) + 1) * 2 * a.d, lane, left, v[j]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j0 + j < j1) {
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] += v[j][e];
            }
    }
    if (TEAM > 1 && more > 8) {   // (the same for the whole CTA)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[part_of][lane + 32 * e] = s[e];
        __syncthreads();
        if (part_of == 0) {
            for (int w = 1; w < TEAM; ++w)
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] += sums[w][lane + 32 * e];
        }
    }
    if (part_of == 0) write_sum<C, O>(a, symbol, col, lane, s);
}

// ------------------------------------------------------------------ host
size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// Tokens of a chunk: 64 to 256, as few as leave every SM eight CTAs at most, where that can be.
constexpr int kChunkMin = 6, kChunkMax = 8;
int chunk_log2_of(int T, int tiles, int sms) {
    int l = kChunkMin;
    while (l < kChunkMax && ((long long)T * tiles >> l) >= 8ll * sms) ++l;
    return l;
}

// Bytes of `tallies` counts for each symbol of a range, and of the flags.
constexpr size_t kPlaceSmem = 200 * 1024;   // of counts at most
size_t place_bytes(int range, int tallies) { return ((size_t)tallies * range + (range + 31) / 32) * 4; }
struct BwdPlan {
    int tiles, chunk_log2, chunks;
    size_t key[3], pos[3], count, part, bytes;
};

// The workspace's parts.  Chunks grow with T, so that a shorter batch's parts may be more of
// them: the room for the parts is that of any batch up to T.
BwdPlan bwd_plan(int T, int d, int elems) {
    BwdPlan p;
    p.tiles = (d + 32 * elems - 1) / (32 * elems);
    const int sms = device_sms();
    p.chunk_log2 = chunk_log2_of(T, p.tiles, sms);
    p.chunks = (int)(((long long)T + (1 << p.chunk_log2) - 1) >> p.chunk_log2);
    const size_t list = up((size_t)T * 4);
    size_t at = 0;
    for (int i = 0; i < 3; ++i) {
        p.key[i] = at;
        at += list;
        p.pos[i] = at;
        at += list;
    }
    p.count = at;
    at += 256;
    p.part = at;
    p.bytes = at + (size_t)p.chunks * 2 * d * 4;
    return p;
}

// At least what any batch of up to T tokens of width d takes, whatever its type: with chunks of
// 2^l tokens there are at most those of the longest batch that takes them.
size_t bwd_ws_bytes(int T, int d) {
    size_t most = 0;
    const int sms = device_sms();
    for (int elems = 4; elems <= 8; elems += 4) {
        const int tiles = (d + 32 * elems - 1) / (32 * elems);
        long long parts = 0;
        for (int l = kChunkMin; l <= kChunkMax; ++l) {
            // the longest batch with chunks of 2^l: one token fewer than takes the next size
            const long long next = ((8ll * sms << l) + tiles - 1) / tiles;
            const long long longest = l == kChunkMax || next > T ? T : next - 1;
            if (longest > 0) parts = std::max(parts, (longest + (1 << l) - 1) >> l);
        }
        most = std::max(most, (size_t)parts * 2 * d * 4);
    }
    return 6 * up((size_t)T * 4) + 256 + most;
}

template <typename T, int W>
cudaError_t fwd(const int* ids, const void* table, int tokens, int V, int d, float scale, void* x,
                cudaStream_t st) {
    constexpr int kCols = 32 * Cols<T, W>::E;
    const int tiles = (d + kCols - 1) / kCols;
    const T* t = static_cast<const T*>(table);
    // four rows a warp once that leaves 16 warps an SM
    if ((long long)tokens * tiles >= 64ll * device_sms()) {
        const dim3 grid((unsigned)(((long long)tokens + 31) / 32), tiles);
        return launch_pdl(embed_fwd_kernel<T, W, 4>, grid, dim3(256), 0, st, ids, t,
                          (long long)tokens, V, d, scale, static_cast<T*>(x));
    }
    const dim3 grid((unsigned)(((long long)tokens + 7) / 8), tiles);
    return launch_pdl(embed_fwd_kernel<T, W, 1>, grid, dim3(256), 0, st, ids, t,
                      (long long)tokens, V, d, scale, static_cast<T*>(x));
}

// Orders the tokens, and zeros the rows that none names.  More of them than a CTA's warps ask for at once:
// by clusters, as many as run at the same time, while their counts fit into shared memory (about 100000
// symbols); else without, while those do (about 160000 symbols: 16384 tokens of 32000 take 5 us less so than
// collected and sorted).
constexpr int kManyTokens = kSortWarps * 512;
cudaError_t launch_sort(SortArgs& a, cudaStream_t st) {
    static std::once_flag once[64];
    static cudaError_t set_err[64];
    static int clusters[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::call_once(once[dev], [&] {
        cudaError_t& err = set_err[dev];
        err = cudaFuncSetAttribute(embed_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                   (int)kPlaceSmem);
        if (err == cudaSuccess)
            err = cudaFuncSetAttribute(embed_place_cluster_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)kPlaceSmem);
        if (err != cudaSuccess) return;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(kCluster);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = kPlaceSmem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kCluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        err = cudaOccupancyMaxActiveClusters(&clusters[dev], embed_place_cluster_kernel, &cfg);
        if (err == cudaSuccess && clusters[dev] < 1) err = cudaErrorInvalidConfiguration;
    });
    if (set_err[dev] != cudaSuccess) return set_err[dev];
    const long long sms = device_sms();
    const auto launch = [&](void (*kern)(const SortArgs), int ctas_of_range, size_t smem) {
        const unsigned ranges = (unsigned)((a.V + a.range - 1) / a.range);
        return launch_pdl(kern, dim3(ranges * ctas_of_range), dim3(kSortThreads), smem, st, a);
    };
    a.range = (a.V + clusters[dev] - 1) / clusters[dev];
    if (a.T > kManyTokens && place_bytes(a.range, kRuns + 3) <= kPlaceSmem)
        return launch(embed_place_cluster_kernel, kCluster, place_bytes(a.range, kRuns + 3));
    a.range = (int)((a.V * (long long)kSplit + sms - 1) / sms);
    if (place_bytes(a.range, kTallies) <= kPlaceSmem)
        return launch(embed_place_kernel, kSplit, place_bytes(a.range, kTallies));
    a.range = (int)((a.V + sms - 1) / sms);
    return launch(embed_sort_kernel, 1, 0);
}

template <typename T, typename O, int W>
cudaError_t bwd(SortArgs& so, SumArgs& su, int tokens, char* ws, cudaStream_t st, int* launches) {
    const BwdPlan p = bwd_plan(tokens, su.d, Cols<T, W>::E);
    for (int i = 0; i < 3; ++i) {
        so.key[i] = reinterpret_cast<int*>(ws + p.key[i]);
        so.pos[i] = reinterpret_cast<int*>(ws + p.pos[i]);
    }
    so.count = reinterpret_cast<int*>(ws + p.count);
    su.key = so.key[2];
    su.pos = so.pos[2];
    su.count = so.count;
    su.part = reinterpret_cast<float*>(ws + p.part);
    su.chunk_log2 = p.chunk_log2;
    su.tiles = p.tiles;
    cudaError_t e = launch_sort(so, st);
    if (e != cudaSuccess) return e;
    ++*launches;
    const long long items = (long long)p.chunks * p.tiles;
    e = launch_pdl(embed_sum_kernel<T, O, W>, dim3((unsigned)items), dim3(32 * kSumWarps), 0, st, su);
    if (e != cudaSuccess) return e;
    ++*launches;
    if (p.chunks == 1) return cudaSuccess;   // no run over a chunk's end
    if ((long long)so.V << p.chunk_log2 <= tokens)
        e = launch_pdl(embed_join_kernel<T, O, W, kSumWarps>, dim3((unsigned)items), dim3(32 * kSumWarps), 0,
                       st, su);
    else
        e = launch_pdl(embed_join_kernel<T, O, W, 1>, dim3((unsigned)((items + kSumWarps - 1) / kSumWarps)),
                       dim3(32 * kSumWarps), 0, st, su);
    if (e != cudaSuccess) return e;
    ++*launches;
    return cudaSuccess;
}

template <typename T, typename O>
cudaError_t bwd_by_width(SortArgs& so, SumArgs& su, int tokens, char* ws, cudaStream_t st, int* launches) {
    const size_t row = (size_t)su.d * sizeof(T);
    if (row % 16 == 0) return bwd<T, O, 16>(so, su, tokens, ws, st, launches);
    if constexpr (sizeof(T) == 2)
        if (row % 4) return bwd<T, O, 2>(so, su, tokens, ws, st, launches);
    return bwd<T, O, 4>(so, su, tokens, ws, st, launches);
}

int check_sizes(int T, int V, int d, int dtype) {
    if (T < 0 || V < 1 || d < 1 || (dtype != HCW_BF16 && dtype != HCW_F32)) return HCW_ERR_INVALID_ARG;
    if (V > kMaxV || d > kMaxD || T > 1 << 28) return HCW_ERR_UNSUPPORTED;
    return HCW_OK;
}

}  // namespace

cudaError_t embed_error_word_read_clear(int* word) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(word, g_error_word, sizeof(int));
    if (e == cudaSuccess && *word) e = cudaMemcpyToSymbol(g_error_word, &zero, sizeof(int));
    return e;
}

}  // namespace hcw

using namespace hcw;

extern "C" int hcw_embed_fwd(const int* ids, const void* E, int T, int V, int d, int dtype, float scale,
                             void* x, void* stream) {
    const int rc = check_sizes(T, V, d, dtype);
    if (rc) return rc;
    if (!(scale - scale == 0.f)) return HCW_ERR_INVALID_ARG;   // infinite or NaN
    if (!on_4_bytes(ids) || !on_16_bytes(E) || !on_16_bytes(x)) return HCW_ERR_ALIGNMENT;
    const size_t es = dtype == HCW_F32 ? 4 : 2, xb = (size_t)T * d * es;
    if (spans_meet(x, xb, ids, (size_t)T * 4) || spans_meet(x, xb, E, (size_t)V * d * es))
        return HCW_ERR_ALIASING;
    if (T == 0) return HCW_OK;
    if (!ids || !E || !x) return HCW_ERR_INVALID_ARG;
    const cudaStream_t st = (cudaStream_t)stream;
    const int bytes = (int)(d * es % 16 == 0 ? 16 : d * es % 4 == 0 ? 4 : 2);
    cudaError_t e;
    if (dtype == HCW_BF16)
        e = bytes == 16  ? fwd<__nv_bfloat16, 16>(ids, E, T, V, d, scale, x, st)
            : bytes == 4 ? fwd<__nv_bfloat16, 4>(ids, E, T, V, d, scale, x, st)
                         : fwd<__nv_bfloat16, 2>(ids, E, T, V, d, scale, x, st);
    else
        e = bytes == 16 ? fwd<float, 16>(ids, E, T, V, d, scale, x, st)
                        : fwd<float, 4>(ids, E, T, V, d, scale, x, st);
    return count_launch(e, 1);
}

extern "C" size_t hcw_embed_bwd_workspace_bytes(int T, int V, int d) {
    if (check_sizes(T, V, d, HCW_BF16) || T == 0) return 0;
    return bwd_ws_bytes(T, d);
}

extern "C" int hcw_embed_bwd(const int* ids, const void* dx, int T, int V, int d, int dtype, float scale,
                             int accumulate, int de_dtype, void* dE, void* workspace,
                             size_t ws_bytes, void* stream) {
    const int rc = check_sizes(T, V, d, dtype);
    if (rc) return rc;
    if (!(scale - scale == 0.f) || (accumulate != 0 && accumulate != 1) ||
        (de_dtype != HCW_BF16 && de_dtype != HCW_F32))
        return HCW_ERR_INVALID_ARG;
    if (!on_4_bytes(ids) || !on_16_bytes(dx) || !on_16_bytes(dE) || !on_16_bytes(workspace))
        return HCW_ERR_ALIGNMENT;
    if (!dE || (T > 0 && (!ids || !dx))) return HCW_ERR_INVALID_ARG;
    const size_t es = dtype == HCW_F32 ? 4 : 2, oes = de_dtype == HCW_F32 ? 4 : 2;
    const size_t ob = (size_t)V * d * oes, need = T > 0 ? bwd_ws_bytes(T, d) : 0;
    if (need && (!workspace || ws_bytes < need)) return HCW_ERR_WORKSPACE;
    const BwdPlan plan = bwd_plan(T, d, dtype == HCW_BF16 ? 8 : 4);
    // (`need` is that of any batch up to T, so no less than this one's parts take)
    if (T > 0 && plan.bytes > ws_bytes) return HCW_ERR_WORKSPACE;
    const struct {
        const void* p;
        size_t n;
    } in[] = {{ids, (size_t)T * 4}, {dx, (size_t)T * d * es}};
    for (const auto& q : in)
        if (spans_meet(dE, ob, q.p, q.n) || spans_meet(workspace, need, q.p, q.n)) return HCW_ERR_ALIASING;
    if (spans_meet(dE, ob, workspace, need)) return HCW_ERR_ALIASING;
    const cudaStream_t st = (cudaStream_t)stream;
    if (T == 0) {
        if (accumulate) return HCW_OK;
        return cudaMemsetAsync(dE, 0, ob, st) == cudaSuccess ? HCW_OK : HCW_ERR_CUDA;
    }
    if ((V + device_sms() - 1) / device_sms() > kMaxRange || (long long)plan.chunks * plan.tiles > 0x7fffffff)
        return HCW_ERR_UNSUPPORTED;
    SortArgs so = {};
    so.ids = ids;
    so.T = T;
    so.V = V;
    so.dE = accumulate ? nullptr : dE;
    so.row_bytes = (size_t)d * oes;
    SumArgs su = {};
    su.dx = dx;
    su.dE = dE;
    su.d = d;
    su.T = T;
    su.scale = scale;
    su.add = accumulate;
    int launches = 0;
    cudaError_t e;
    char* ws = static_cast<char*>(workspace);
    if (dtype == HCW_BF16)
        e = de_dtype == HCW_BF16 ? bwd_by_width<__nv_bfloat16, __nv_bfloat16>(so, su, T, ws, st, &launches)
                                 : bwd_by_width<__nv_bfloat16, float>(so, su, T, ws, st, &launches);
    else
        e = de_dtype == HCW_BF16 ? bwd_by_width<float, __nv_bfloat16>(so, su, T, ws, st, &launches)
                                 : bwd_by_width<float, float>(so, su, T, ws, st, &launches);
    return count_launch(e, launches);
}
