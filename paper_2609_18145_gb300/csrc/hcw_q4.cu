// hcw_q4.cu -- products of a few tokens with weights of 4 bits and a scale for each group of
// them (hcw_q4_matmul), and the weights' way there (hcw_q4_quantize, hcw_q4_pack):
//
//   y_to = sum over k of x_tk s_{o, k / group} q_ok (+ b_o),   q in -8 .. 7
//
// Bound by memory: half a byte a weight (and two bytes a group), read once for all tokens of a call.
// The warp-level MMA does the products, 16 rows of weights against 8 tokens: at the memory's rate an
// SM meets 46 weights a cycle, which is too many for a multiply-add each and all tokens.
//
// Packed weights: pieces of 16 rows x 128 k, a row of pieces for every 16 rows.  A piece is two
// blocks of 64 k, 512 bytes each, in which a lane's 16 bytes are its operand words of four MMAs, then
// the scales (for rows g and g + 8 a word for each group).  The k of an MMA may be any 16, as long as
// both operands agree: lane (g, t) = (lane / 4, lane % 4) has rows g and g + 8 and, in MMAs 0 and 1 of
// a block, k = 8 t + 0 .. 7, in 2 and 3 those 32 further, so that its activations are two vectors of
// 16 bytes.  Codes are stored as q + 8, two of them 16 bits apart.  A bf16 number whose bits are a code
// in the lowest four is code 2^-133, in the next four 16 times that (the numbers below and just
// above the normal ones' limit are evenly spaced): one multiply-add of two bf16 numbers brings it to
// (q + 8) 2^-6 and takes 8 2^-6 off, exactly, so that four pairs of codes take one shift, four masks
// and four multiply-adds.  The products of a group are added in fp32 by the MMAs and then multiplied by
// its scale, in fp32; the factor 2^6 comes last.
#include "hcw.h"
#include "hcw_internal.h"

#include <math.h>

#include <algorithm>
#include <mutex>

namespace hcw {

namespace {

constexpr int kQMaxN = 1 << 24, kQMaxK = 1 << 20, kQMaxT = 1 << 19;

__host__ __device__ __forceinline__ size_t tiles_of(int N) { return ((size_t)N + 15) / 16; }
__host__ __device__ __forceinline__ size_t pieces_of(int K) { return ((size_t)K + 127) / 128; }
__host__ __device__ __forceinline__ size_t groups_of(int K, int group) {
    return ((size_t)K + group - 1) / group;
}
// Bytes of a piece: the codes, then for each pair of rows a word for each group.
__host__ __device__ __forceinline__ constexpr int piece_bytes(int group) {
    return 1024 + 128 / group * 32;
}

// ------------------------------------------------------------------ weights
__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// A warp a group: s = max |w| / 7 in bf16, q = w / s rounded to the nearest (ties to even), in
// -8 .. 7.
template <typename T>
__global__ void __launch_bounds__(256) q4_quantize_kernel(const T* W, int N, int K, int group,
                                                          signed char* codes,
                                                          __nv_bfloat16* scales) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, G = (int)groups_of(K, group);
    const long long at = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (at >= (long long)N * G) return;
    const long long row = at / G;
    const int g = (int)(at % G), k0 = g * group, n = min(group, K - k0);
    const T* w = W + row * K + k0;
    float v[4], m = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = lane + 32 * e < n ? value(w + lane + 32 * e) : 0.f;
        m = fmaxf(m, fabsf(v[e]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const __nv_bfloat16 s16 = __float2bfloat16_rn(m / 7.f);
    const float s = __bfloat162float(s16);
    if (lane == 0) scales[at] = s16;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (lane + 32 * e >= n) continue;
        const float q = s > 0.f ? rintf(v[e] / s) : 0.f;
        codes[row * K + k0 + lane + 32 * e] = (signed char)fminf(fmaxf(q, -8.f), 7.f);
    }
}

// A thread a word of the packed weights: eight codes of rows g and g + 8, or two scales.
__global__ void __launch_bounds__(256) q4_pack_kernel(const signed char* codes,
                                                      const unsigned short* scales, int N, int K,
                                                      int group, uint32_t* packed) {
    pdl_wait();
    pdl_trigger();
    const int words = piece_bytes(group) / 4, G = (int)groups_of(K, group);
    const long long pieces = (long long)pieces_of(K), all = (long long)tiles_of(N) * pieces * words;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all;
         i += (long long)gridDim.x * 256) {
        const int at = (int)(i % words);
        const long long piece = i / words, row0 = piece / pieces * 16, k0 = piece % pieces * 128;
        uint32_t w = 0;
        if (at < 256) {
            const int s = at & 3, lane = at >> 2 & 31, g = lane >> 2, t = lane & 3;
            const long long k = k0 + 64 * (at >> 7) + 32 * (s >> 1) + 8 * t + 4 * (s & 1);
#pragma unroll
            for (int p = 0; p < 4; ++p)       // a0 .. a3: rows g, g + 8, g, g + 8
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const long long r = row0 + g + 8 * (p & 1), kk = k + 2 * (p >> 1) + h;
                    const int q = r < N && kk < K ? codes[r * K + kk] : 0;
                    w |= (uint32_t)((q + 8) & 15) << (4 * p + 16 * h);
                }
        } else {
            const int per = 128 / group, g = (at - 256) / per;
            const long long gr = k0 / group + (at - 256) % per;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const long long r = row0 + g + 8 * h;
                if (r < N && gr < G) w |= (uint32_t)scales[r * G + gr] << (16 * h);
            }
        }
        packed[i] = w;
    }
}

// ------------------------------------------------------------------ product
struct Q4Args {
    const __nv_bfloat16* x;
    const char* packed;
    const float* bias;
    void* y;
    int T, N, K;
    int pieces, f32;
    int team;       // warps that share the k range
};

// D = A B + D of m16n8k16: 16 rows of weights, 8 tokens; FIRST: D = A B.
template <bool FIRST>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (FIRST)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
            "{%8,%9}, {%10,%10,%10,%10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
            "{%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// a b + c on two bf16 numbers, subnormal ones included.
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

// The four operand words of one MMA from a word of codes, times 2^-6.
__device__ __forceinline__ void expand(uint32_t w, uint32_t (&a)[4]) {
    constexpr uint32_t kLow = 0x7f007f00u;    // 2^127
    constexpr uint32_t kHigh = 0x7d007d00u;   // 2^123
    constexpr uint32_t kOff = 0xbe00be00u;    // -8 2^-6
    const uint32_t v = w >> 8;
    a[0] = fma_bf16x2(w & 0x000f000fu, kLow, kOff);
    a[1] = fma_bf16x2(w & 0x00f000f0u, kHigh, kOff);
    a[2] = fma_bf16x2(v & 0x000f000fu, kLow, kOff);
    a[3] = fma_bf16x2(v & 0x00f000f0u, kHigh, kOff);
}

constexpr int kQWarps = 16;           // warps of a CTA at most
constexpr int kQChunk = 4096;         // k of the activations in shared memory
constexpr int kQSmem = 232448;        // shared memory of an SM

// Floats of a warp's sums over RT row tiles: 8 tokens of 16 rows each, a token 20 floats from the next,
// so that the writes do not meet in a bank.
__host__ __device__ constexpr int part_floats(int rt, int nt) { return rt * nt * 160; }
// Bytes from one token's activations to the next's in shared memory: 64 beside the row, so that the 16
// byte reads of neighbouring tokens fall into different banks.
__host__ __device__ constexpr int x_stride(int pieces) { return pieces * 256 + 64; }

__device__ __forceinline__ uint32_t shared_at(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async_or_zero(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A team of 1 to 16 warps contracts RT row tiles at a time, its warps taking every team-th piece of
// the k range; a team of several has one set of tiles and adds up in shared memory.  The weights come
// through a ring of each warp's own, by asynchronous copies, D pieces of its RT tiles ahead; the
// activations are in shared memory, kQChunk of the k range at a time.  Tiles and tokens past the last
// ones are computed as something, and not written.
//
// Where there are many row tiles a warp has two of them to itself: no sums to join, and the activations'
// way from shared memory serves both.  131072 x 4096, groups of 128: one token 52 us (5.4 TB/s), 8 54, 16
// 65; bound by the issue of instructions, nine for every eight weights of a lane, and with 16 tokens
// by the MMA too (46 % of its cycles).  A k range shared by 8 warps took 74 and 94 us: joining the
// sums and reading the activations again and again cost as much as the products.
template <int RT, int NT, int GROUP, int D>
__global__ void __launch_bounds__(32 * kQWarps, 1) q4_kernel(const Q4Args a) {
    constexpr int GM = GROUP / 16;                 // MMAs of a group
    constexpr int SW = 128 / GROUP;                // words of scales of a pair of rows
    constexpr int PB = piece_bytes(GROUP), UB = RT * PB, PF = part_floats(RT, NT);
    static_assert(D * UB >= PF * 4, "a warp's sums take its ring's place");
    extern __shared__ __align__(16) uint8_t q_smem[];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int warps = blockDim.x >> 5, teams = warps / a.team;
    const int team = warp / a.team, part = warp % a.team;
    uint8_t* const ring = q_smem + warp * (D * UB);
    uint8_t* const xs = q_smem + warps * (D * UB);
    const int tiles = (int)tiles_of(a.N), tok0 = blockIdx.y * (NT * 8);
    const int rows = min(a.T - tok0, NT * 8);
    const int sets = (tiles + RT - 1) / RT;        // of RT tiles
    const int set0 = blockIdx.x * teams + team, step = gridDim.x * teams;
    const size_t row_bytes = (size_t)a.pieces * PB;
    constexpr int kPer = kQChunk / 128;            // pieces of a chunk of activations
    const int stride = x_stride(min(a.pieces, kPer));
    const auto activations = [&](int p0) {
        const int vecs = (min(a.pieces, p0 + kPer) - p0) * 16;   // of a token
        for (int i = threadIdx.x; i < rows * vecs; i += blockDim.x) {
            const int row = i / vecs, v = i % vecs, k = p0 * 128 + v * 8;
            copy_async_or_zero(shared_at(xs + row * stride + v * 16),
                               a.x + (size_t)(tok0 + row) * a.K + (k < a.K ? k : 0), k < a.K);
        }
        copies_commit();
    };
    activations(0);
    // the next copy: a piece of a set, and the lane's first 16 bytes of it in each of the set's tiles
    // (a team, of which there is none where RT is 2, may have more warps than a tile has pieces: the others
    // copy nothing)
    int next_set = RT > 1 || part < a.pieces ? set0 : sets, next_piece = part;
    const char* from[RT];
    const auto aim = [&]() {
#pragma unroll
        for (int r = 0; r < RT; ++r)
            from[r] = a.packed + min(next_set * RT + r, tiles - 1) * row_bytes + next_piece * PB + 16 * lane;
    };
    const uint32_t ring_at = shared_at(ring) + 16 * lane;
    const int ahead = a.team * PB;
    const auto issue = [&](int place) {
        if (next_set < sets) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                copy_async(ring_at + place + r * PB, from[r]);
                copy_async(ring_at + place + r * PB + 512, from[r] + 512);
                if (lane < 2 * SW) copy_async(ring_at + place + r * PB + 1024, from[r] + 1024);
                from[r] += ahead;
            }
            next_piece += a.team;
            if (next_piece >= a.pieces) {
                next_piece = part;
                next_set += step;
                aim();
            }
        }
        copies_commit();
    };
    aim();
#pragma unroll
    for (int u = 0; u < D; ++u) issue(u * UB);
    copies_wait<D>();
    __syncthreads();
    const uint8_t* xat[NT];   // the lane's tokens
#pragma unroll
    for (int n = 0; n < NT; ++n) xat[n] = xs + min(8 * n + g, rows - 1) * stride + 16 * t;
    const auto write = [&](int tile, int row, int n, float s) {
        const long long o = (long long)tile * 16 + row;
        if (tok0 + n >= a.T || o >= a.N) return;
        s *= 64.f;
        if (a.bias) s += a.bias[o];
        const size_t at = (size_t)(tok0 + n) * a.N + o;
        if (a.f32)
            static_cast<float*>(a.y)[at] = s;
        else
            static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(s);
    };
    int at_place = 0;
    // (the CTA's teams go through as many rounds: each meets the others where activations change)
    for (int set = set0, round = 0; set - team < sets; set += step, ++round) {
        float sum[RT][NT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) sum[r][n][c] = 0.f;
        int p = part;
        for (int p0 = 0; p0 < a.pieces; p0 += kPer) {
            if (a.pieces > kPer && (round || p0)) {
                __syncthreads();   // the chunk before has been read
                activations(p0);
                copies_wait<0>();
                __syncthreads();
            }
            const int p1 = set < sets ? min(a.pieces, p0 + kPer) : 0;
            for (; p < p1; p += a.team) {
                copies_wait<D - 1>();
                __syncwarp();
                const uint8_t* place = ring + at_place;
                uint4 w[RT][2];
                uint32_t sc[RT][SW];
#pragma unroll
                for (int r = 0; r < RT; ++r) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        w[r][b] = *reinterpret_cast<const uint4*>(place + r * PB + 512 * b + 16 * lane);
#pragma unroll
                    for (int j = 0; j < SW; ++j)
                        sc[r][j] = *reinterpret_cast<const uint32_t*>(place + r * PB + 1024 + 4 * SW * g + 4 * j);
                }
                __syncwarp();   // the place has been read
                issue(at_place);
                at_place = at_place + UB == D * UB ? 0 : at_place + UB;
                float acc[RT][NT][4];
                uint4 xv[NT];
#pragma unroll
                for (int m = 0; m < 8; ++m) {
                    if (!(m & 1)) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            xv[n] = *reinterpret_cast<const uint4*>(xat[n] + (p - p0) * 256 + 32 * m);
                    }
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const uint4& q = w[r][m >> 2];
                        uint32_t av[4];
                        expand((m & 3) == 0 ? q.x : (m & 3) == 1 ? q.y : (m & 3) == 2 ? q.z : q.w, av);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint4& v = xv[n];
                            if (m % GM == 0)
                                mma<true>(acc[r][n], av, m & 1 ? v.z : v.x, m & 1 ? v.w : v.y);
                            else
                                mma<false>(acc[r][n], av, m & 1 ? v.z : v.x, m & 1 ? v.w : v.y);
                            if (m % GM == GM - 1) {
                                const uint32_t s = sc[r][m / GM];
                                const float s0 = __uint_as_float(s << 16), s1 = __uint_as_float(s & 0xffff0000u);
                                sum[r][n][0] = fmaf(s0, acc[r][n][0], sum[r][n][0]);
                                sum[r][n][1] = fmaf(s0, acc[r][n][1], sum[r][n][1]);
                                sum[r][n][2] = fmaf(s1, acc[r][n][2], sum[r][n][2]);
                                sum[r][n][3] = fmaf(s1, acc[r][n][3], sum[r][n][3]);
                            }
                        }
                    }
                }
            }
        }
        if (a.team == 1) {
            if (set < sets) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            write(set * RT + r, g + 8 * (c >> 1), 8 * n + 2 * t + (c & 1), sum[r][n][c]);
            }
            continue;
        }
        // the team's only round: its rings are empty, its parts are added in the warps' order
        copies_wait<0>();
        __syncwarp();
        float* const to = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    to[(r * NT + n) * 160 + (2 * t + (c & 1)) * 20 + g + 8 * (c >> 1)] = sum[r][n][c];
        __syncthreads();
        if (set < sets) {
            const float* const parts = reinterpret_cast<const float*>(q_smem + team * a.team * (D * UB));
            for (int i = part * 32 + lane; i < RT * NT * 128; i += a.team * 32) {
                const int row = i & 15, n = i >> 4 & (NT * 8 - 1), r = i / (NT * 128);
                const float* f = parts + (r * NT + (n >> 3)) * 160 + (n & 7) * 20 + row;
                float s = 0.f;
#pragma unroll 4
                for (int w = 0; w < a.team; ++w) s += f[w * (D * UB / 4)];
                write(set * RT + r, row, n, s);
            }
        }
        break;
    }
    copies_wait<0>();
}

template <int RT, int NT, int GROUP, int D>
cudaError_t launch_q4(const Q4Args& a, int teams, cudaStream_t st) {
    auto kern = q4_kernel<RT, NT, GROUP, D>;
    static std::once_flag once[64];
    static cudaError_t set_err[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::call_once(once[dev], [&] {
        set_err[dev] = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kQSmem);
    });
    if (set_err[dev] != cudaSuccess) return set_err[dev];
    const int warps = teams * a.team;
    const size_t sets = (tiles_of(a.N) + RT - 1) / RT, ctas = (sets + teams - 1) / teams;
    const size_t room = a.team > 1 ? ctas : (size_t)device_sms();
    const size_t smem = (size_t)warps * D * RT * piece_bytes(GROUP) +
                        (size_t)std::min(a.T, NT * 8) * x_stride(std::min(a.pieces, kQChunk / 128));
    return launch_pdl(kern, dim3((unsigned)std::min(ctas, room), (a.T + NT * 8 - 1) / (NT * 8)),
                      dim3(32 * warps), smem, st, a);
}

// Up to 14 row tiles an SM: a team for each of them, of as many warps as make 16 in all at most.  More:
// a warp for every two, as many warps (10 to 14) as leave the fewest of them idle in the last round.
// By the weights' sizes alone, so that a token's sums keep their order whatever the batch.  On either side of
// the rules' edges, K = 4096 in groups of 128, one token and 16 on 152 SMs: 152 tiles 3.3 and 5.3 us, 153 (two
// teams a CTA, half of the SMs) 4.1 and 6.4, as 304; 2128 tiles 14.4 and 20.2, 2129 (pairs) 19.2 and 27.7; 4256
// 27.7 and 35.7, 4257 (a second round) 37.0 and 51.1, 6384 38.6 and 50.9.
template <int GROUP>
cudaError_t product(Q4Args& a, cudaStream_t st) {
    const long long tiles = (long long)tiles_of(a.N), sms = device_sms();
    a.team = 1;
    if (tiles <= 14 * sms) {
        const int teams = (int)((tiles + sms - 1) / sms);
        while (a.team * teams * 2 <= kQWarps && a.team < a.pieces) a.team *= 2;
        return a.T <= 8 ? launch_q4<1, 1, GROUP, 8>(a, teams, st) : launch_q4<1, 2, GROUP, 5>(a, teams, st);
    }
    const long long pairs = (tiles + 1) / 2;
    int warps = 14;
    long long best = 1ll << 60;
    for (int w = 14; w >= 10; --w) {
        const long long idle = (pairs + w * sms - 1) / (w * sms) * w * sms - pairs;
        if (idle < best) {
            best = idle;
            warps = w;
        }
    }
    return a.T <= 8 ? launch_q4<2, 1, GROUP, 5>(a, warps, st) : launch_q4<2, 2, GROUP, 3>(a, warps, st);
}

int check_weights(int N, int K, int group) {
    if (N < 1 || K < 1 || (group != 32 && group != 64 && group != 128)) return HCW_ERR_INVALID_ARG;
    if (N > kQMaxN || K > kQMaxK || K % 8) return HCW_ERR_UNSUPPORTED;
    return HCW_OK;
}

size_t packed_bytes(int N, int K, int group) {
    return tiles_of(N) * pieces_of(K) * piece_bytes(group);
}

}  // namespace

}  // namespace hcw

using namespace hcw;

extern "C" size_t hcw_q4_bytes(int N, int K, int group) {
    return check_weights(N, K, group) ? 0 : packed_bytes(N, K, group);
}

extern "C" int hcw_q4_quantize(const void* W, int N, int K, int group, int dtype, signed char* codes,
                               void* scales, void* stream) {
    if (dtype != HCW_BF16 && dtype != HCW_F32) return HCW_ERR_INVALID_ARG;
    const int rc = check_weights(N, K, group);
    if (rc) return rc;
    if (!W || !codes || !scales) return HCW_ERR_INVALID_ARG;
    if (!on_16_bytes(W) || !on_16_bytes(codes) || !on_16_bytes(scales)) return HCW_ERR_ALIGNMENT;
    const size_t n = (size_t)N * K, G = groups_of(K, group), wb = n * (dtype == HCW_F32 ? 4 : 2);
    if (spans_meet(codes, n, W, wb) || spans_meet(scales, N * G * 2, W, wb) ||
        spans_meet(codes, n, scales, N * G * 2))
        return HCW_ERR_ALIASING;
    const size_t blocks = (N * G + 7) / 8;
    if (blocks > 0x7fffffff) return HCW_ERR_UNSUPPORTED;
    const cudaStream_t st = (cudaStream_t)stream;
    __nv_bfloat16* s = static_cast<__nv_bfloat16*>(scales);
    const dim3 grid((unsigned)blocks), block(256);
    return count_launch(
        dtype == HCW_BF16
            ? launch_pdl(q4_quantize_kernel<__nv_bfloat16>, grid, block, 0, st,
                         static_cast<const __nv_bfloat16*>(W), N, K, group, codes, s)
            : launch_pdl(q4_quantize_kernel<float>, grid, block, 0, st, static_cast<const float*>(W),
                         N, K, group, codes, s),
        1);
}

extern "C" int hcw_q4_pack(const signed char* codes, const void* scales, int N, int K, int group,
                           void* packed, void* stream) {
    const int rc = check_weights(N, K, group);
    if (rc) return rc;
    if (!codes || !scales || !packed) return HCW_ERR_INVALID_ARG;
    if (!on_16_bytes(codes) || !on_16_bytes(scales) || !on_16_bytes(packed)) return HCW_ERR_ALIGNMENT;
    const size_t n = packed_bytes(N, K, group);
    if (spans_meet(packed, n, codes, (size_t)N * K) ||
        spans_meet(packed, n, scales, N * groups_of(K, group) * 2))
        return HCW_ERR_ALIASING;
    const size_t blocks = std::min<size_t>((n / 4 + 255) / 256, 16 * (size_t)device_sms());
    return count_launch(launch_pdl(q4_pack_kernel, dim3((unsigned)blocks), dim3(256), 0,
                                   (cudaStream_t)stream, codes,
                                   static_cast<const unsigned short*>(scales), N, K, group,
                                   static_cast<uint32_t*>(packed)),
                        1);
}

extern "C" int hcw_q4_matmul(const void* x, const void* packed, const float* bias, int T, int N, int K,
                             int group, int y_dtype, void* y, void* stream) {
    if (T < 0 || (y_dtype != HCW_BF16 && y_dtype != HCW_F32)) return HCW_ERR_INVALID_ARG;
    const int rc = check_weights(N, K, group);
    if (rc) return rc;
    if (T > kQMaxT) return HCW_ERR_UNSUPPORTED;
    if (!on_16_bytes(x) || !on_16_bytes(packed) || !on_4_bytes(bias) || !on_16_bytes(y))
        return HCW_ERR_ALIGNMENT;
    const size_t yb = (size_t)T * N * (y_dtype == HCW_F32 ? 4 : 2);
    if (spans_meet(y, yb, x, (size_t)T * K * 2) || spans_meet(y, yb, packed, packed_bytes(N, K, group)) ||
        spans_meet(y, yb, bias, (size_t)N * 4))
        return HCW_ERR_ALIASING;
    if (T == 0) return HCW_OK;
    if (!x || !packed || !y) return HCW_ERR_INVALID_ARG;
    Q4Args a = {};
    a.x = static_cast<const __nv_bfloat16*>(x);
    a.packed = static_cast<const char*>(packed);
    a.bias = bias;
    a.y = y;
    a.T = T;
    a.N = N;
    a.K = K;
    a.pieces = (int)pieces_of(K);
    a.f32 = y_dtype == HCW_F32;
    const cudaStream_t st = (cudaStream_t)stream;
    return count_launch(group == 32   ? product<32>(a, st)
                        : group == 64 ? product<64>(a, st)
                                      : product<128>(a, st),
                        1);
}
