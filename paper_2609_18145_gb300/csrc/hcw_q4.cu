// hcw_q4.cu -- products of a few tokens with weights of 4 bits and a scale for each group of
// them (hcw_q4_matmul), and the weights' way there (hcw_q4_quantize, hcw_q4_pack):
//
//   y_to = sum over k of x_tk s_{o, k / group} q_ok (+ b_o),   q in -8 .. 7
//
// Bound by memory: half a byte a weight (and two bytes a group), read once for all tokens of a call.
// The warp-level MMA does the products, 16 rows of weights against 8 tokens: at the memory's rate an
// SM meets 46 weights a cycle, which is too many for a multiply-add each and all tokens.
//
// Packed weights: tiles of 16 rows x 64 k, 512 bytes each, in which a lane's 16 bytes are its
// operand words of four MMAs.  The k of an MMA may be any 16, as long as both operands agree: lane
// (g, t) = (lane / 4, lane % 4) has rows g and g + 8 and, in MMAs 0 and 1, k = 8 t + 0 .. 7, in 2
// and 3 another 32 further, so that its activations are two vectors of 16 bytes.  Codes are stored
// as q + 8, two of them 16 bits apart: with the bits of 128 above them they are the bf16 numbers
// 136 + q, and 136 comes off exactly.  The products of a group are added in fp32 by the MMAs and
// then multiplied by its scale, in fp32.
#include "hcw.h"
#include "hcw_internal.h"
#include "hcw_ptx.cuh"

#include <math.h>

#include <algorithm>

namespace hcw {

namespace {

constexpr int kQMaxN = 1 << 24, kQMaxK = 1 << 20, kQMaxT = 1 << 19;

__host__ __device__ __forceinline__ size_t tiles_of(int N) { return ((size_t)N + 15) / 16; }
__host__ __device__ __forceinline__ size_t blocks_of(int K) { return ((size_t)K + 63) / 64; }
__host__ __device__ __forceinline__ size_t groups_of(int K, int group) {
    return ((size_t)K + group - 1) / group;
}
// The scales' place behind the codes: for each tile its groups' 16 scales one group after the other.
__host__ __device__ __forceinline__ size_t codes_bytes(int N, int K) {
    return tiles_of(N) * blocks_of(K) * 512;
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

// A thread a word of the packed codes (eight weights of rows g and g + 8), then one a scale.
__global__ void __launch_bounds__(256) q4_pack_kernel(const signed char* codes,
                                                      const __nv_bfloat16* scales, int N, int K,
                                                      int group, uint32_t* packed) {
    pdl_wait();
    pdl_trigger();
    const long long words = (long long)codes_bytes(N, K) / 4;
    const int G = (int)groups_of(K, group);
    const long long all = words + (long long)tiles_of(N) * G * 8;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all;
         i += (long long)gridDim.x * 256) {
        if (i < words) {
            const int s = (int)(i & 3), lane = (int)(i >> 2) & 31, g = lane >> 2, t = lane & 3;
            const long long block = i >> 7, nb = (long long)blocks_of(K);
            const long long row = block / nb * 16 + g;
            const long long k = block % nb * 64 + 32 * (s >> 1) + 8 * t + 4 * (s & 1);
            uint32_t w = 0;
#pragma unroll
            for (int p = 0; p < 4; ++p)       // a0 .. a3: rows g, g + 8, g, g + 8
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const long long r = row + 8 * (p & 1), kk = k + 2 * (p >> 1) + h;
                    const int q = r < N && kk < K ? codes[r * K + kk] : 0;
                    w |= (uint32_t)((q + 8) & 15) << (4 * p + 16 * h);
                }
            packed[i] = w;
        } else {   // two scales
            const long long j = (i - words) * 2;
            uint32_t w = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const long long tg = (j + h) >> 4, r = tg / G * 16 + ((j + h) & 15);
                const unsigned short b =
                    r < N ? __bfloat16_as_ushort(scales[r * G + tg % G]) : (unsigned short)0;
                w |= (uint32_t)b << (16 * h);
            }
            packed[i] = w;
        }
    }
}

// ------------------------------------------------------------------ product
struct Q4Args {
    const __nv_bfloat16* x;
    const uint4* codes;
    const __nv_bfloat16* scales;   // [tiles][G][16]
    const float* bias;
    void* y;
    int T, N, K;
    int G, blocks, f32;
};

// D += A B of m16n8k16: 16 rows of weights, 8 tokens.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The four operand words of one MMA from a word of codes.
__device__ __forceinline__ void expand(uint32_t w, uint32_t (&a)[4]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t m = ((w >> (4 * p)) & 0x000f000fu) | 0x43004300u;   // 128 + code
        __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&m);
        v = __hsub2(v, __nv_bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308)));
        a[p] = *reinterpret_cast<const uint32_t*>(&v);
    }
}

// RT row tiles a CTA, NT blocks of 8 tokens; eight warps share the k range, a warp takes units of
// UB blocks of 64 k (a whole number of groups, GB MMAs each).
template <int RT, int NT, int GROUP>
__global__ void __launch_bounds__(256) q4_kernel(const Q4Args a) {
    constexpr int UB = GROUP == 128 ? 2 : 1;       // blocks of a unit
    constexpr int GM = GROUP / 16;                 // MMAs of a group
    constexpr int UG = UB * 4 / GM;                // groups of a unit
    __shared__ float part[8][RT * 16][NT * 8 + 1];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const long long tile0 = (long long)blockIdx.x * RT, tiles = (long long)tiles_of(a.N);
    const int tok0 = blockIdx.y * (NT * 8);
    float sum[RT][NT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[r][n][c] = 0.f;
    const int units = (a.blocks + UB - 1) / UB;
    for (int u = warp; u < units; u += 8) {
        uint4 w[RT][UB];
        float sc[RT][UG][2];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const long long tile = min(tile0 + r, tiles - 1);
#pragma unroll
            for (int b = 0; b < UB; ++b) {
                const int block = u * UB + b;
                w[r][b] = block < a.blocks ? a.codes[(tile * a.blocks + block) * 32 + lane]
                                           : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < UG; ++j) {
                const int gr = u * UG + j;
                const __nv_bfloat16* s = a.scales + (tile * a.G + min(gr, a.G - 1)) * 16;
                sc[r][j][0] = gr < a.G ? __bfloat162float(s[g]) : 0.f;
                sc[r][j][1] = gr < a.G ? __bfloat162float(s[g + 8]) : 0.f;
            }
        }
        float acc[RT][NT][4];
#pragma unroll
        for (int b = 0; b < UB; ++b) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // 32 k
                const int k = (u * UB + b) * 64 + 32 * h + 8 * t;
                uint4 xv[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int tok = tok0 + 8 * n + g;
                    xv[n] = make_uint4(0, 0, 0, 0);
                    if (tok < a.T && k < a.K)
                        xv[n] = *reinterpret_cast<const uint4*>(a.x + (size_t)tok * a.K + k);
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int m = b * 4 + h * 2 + q;   // the unit's MMA
                        const uint32_t word = h == 0 ? (q == 0 ? w[r][b].x : w[r][b].y)
                                                     : (q == 0 ? w[r][b].z : w[r][b].w);
                        uint32_t av[4];
                        expand(word, av);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (m % GM == 0) {
#pragma unroll
                                for (int c = 0; c < 4; ++c) acc[r][n][c] = 0.f;
                            }
                            if (q == 0)
                                mma(acc[r][n], av, xv[n].x, xv[n].y);
                            else
                                mma(acc[r][n], av, xv[n].z, xv[n].w);
                            if (m % GM == GM - 1) {
                                const float s0 = sc[r][m / GM][0], s1 = sc[r][m / GM][1];
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
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                part[warp][r * 16 + g + 8 * (c >> 1)][n * 8 + 2 * t + (c & 1)] = sum[r][n][c];
    __syncthreads();
    for (int i = threadIdx.x; i < RT * 16 * NT * 8; i += 256) {
        const int o = i % (RT * 16), n = i / (RT * 16);
        const long long row = tile0 * 16 + o;
        if (tok0 + n >= a.T || row >= a.N) continue;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += part[w][o][n];
        if (a.bias) s += a.bias[row];
        const size_t at = (size_t)(tok0 + n) * a.N + row;
        if (a.f32)
            static_cast<float*>(a.y)[at] = s;
        else
            static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(s);
    }
}

template <int RT, int NT>
cudaError_t launch_q4(const Q4Args& a, int group, cudaStream_t st) {
    const dim3 grid((unsigned)((tiles_of(a.N) + RT - 1) / RT), (a.T + NT * 8 - 1) / (NT * 8));
    if (group == 32) return launch_pdl(q4_kernel<RT, NT, 32>, grid, dim3(256), 0, st, a);
    if (group == 64) return launch_pdl(q4_kernel<RT, NT, 64>, grid, dim3(256), 0, st, a);
    return launch_pdl(q4_kernel<RT, NT, 128>, grid, dim3(256), 0, st, a);
}

int check_weights(int N, int K, int group) {
    if (N < 1 || K < 1 || (group != 32 && group != 64 && group != 128)) return HCW_ERR_INVALID_ARG;
    if (N > kQMaxN || K > kQMaxK || K % 8) return HCW_ERR_UNSUPPORTED;
    return HCW_OK;
}

size_t packed_bytes(int N, int K, int group) {
    return codes_bytes(N, K) + tiles_of(N) * groups_of(K, group) * 32;
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
                                   static_cast<const __nv_bfloat16*>(scales), N, K, group,
                                   static_cast<uint32_t*>(packed)),
                        1);
}

extern "C" int hcw_q4_matmul(const void* x, const void* packed, const float* bias, int T, int N, int K,
                             int group, int y_dtype, void* y, void* stream) {
    if (T < 0 || (y_dtype != HCW_BF16 && y_dtype != HCW_F32)) return HCW_ERR_INVALID_ARG;
    const int rc = check_weights(N, K, group);
    if (rc) return rc;
    if (T > kQMaxT) return HCW_ERR_UNSUPPORTED;
    if (!on_16_bytes(x) || !on_16_bytes(packed) || !on_16_bytes(bias) || !on_16_bytes(y))
        return HCW_ERR_ALIGNMENT;
    const size_t yb = (size_t)T * N * (y_dtype == HCW_F32 ? 4 : 2);
    if (spans_meet(y, yb, x, (size_t)T * K * 2) || spans_meet(y, yb, packed, packed_bytes(N, K, group)) ||
        spans_meet(y, yb, bias, (size_t)N * 4))
        return HCW_ERR_ALIASING;
    if (T == 0) return HCW_OK;
    if (!x || !packed || !y) return HCW_ERR_INVALID_ARG;
    Q4Args a = {};
    a.x = static_cast<const __nv_bfloat16*>(x);
    a.codes = static_cast<const uint4*>(packed);
    a.scales = reinterpret_cast<const __nv_bfloat16*>(static_cast<const char*>(packed) +
                                                      codes_bytes(N, K));
    a.bias = bias;
    a.y = y;
    a.T = T;
    a.N = N;
    a.K = K;
    a.G = (int)groups_of(K, group);
    a.blocks = (int)blocks_of(K);
    a.f32 = y_dtype == HCW_F32;
    const cudaStream_t st = (cudaStream_t)stream;
    return count_launch(T <= 8 ? launch_q4<1, 1>(a, group, st) : launch_q4<1, 2>(a, group, st), 1);
}
