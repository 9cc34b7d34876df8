// hcw_ffn.cu -- the gated feed-forward block, bf16 (hcw_gated_ffn_fwd / _bwd):
//
//   [g | u] = x W1^T,  a = act(g) u,  y = a W2^T
//   da = dy W2,  du = da act(g),  dg = da u act'(g)
//   dx = [dg | du] W1,  dW1 = [dg | du]^T x,  dW2 = dy^T a
//
// with x [T][d], W1 [2h][d] (gate rows, then up rows), W2 [d][h].  Bound by the tensor
// cores: 6 T d h flops forward, 12 T d h backward and 4 T d h more to compute g and u
// again (the forward saves nothing: its 8 bytes a hidden value would be rounded to bf16
// once more, or cost more traffic in fp32 than the products take at small d).
//
// All products run as pairs of SMs on tcgen05.mma.cta_group::2, operands by TMA
// into a ring, fp32 accumulators in TMEM, results through shared-memory patches and TMA
// stores.  A launch is persistent: the pairs take its units (output tiles) in turn.
//   gate    256 rows x 128 hidden columns: the pair's first CTA loads the gate rows
//           of W1, the second the up rows, so one MMA of N = 256 gives both projections
//           of the tile side by side, and the epilogue writes act(g) u, rounded once.
//           Two accumulators: a tile's epilogue runs under the next tile's products.
//   grad    256 rows x 256 hidden columns, two accumulators of 256 columns: g and u of the
//           first 128, da of all, g and u of the second 128.  (Of 128 columns a K step of da
//           takes 0.75 of the time of 256, not half: at 8192 x 2048 x 2816 this pass took 214 us
//           so and takes 177.)  The epilogue draws g and u into registers at once, so that
//           the next products run under it, and writes dg, du and a.
//   gemm    y, or dx, dW1 and dW2 together: up to three products in one launch.  Each pair
//           takes the same number of whole tiles; the tiles left over form a line of K
//           steps that is cut into even shares.  A tile that was cut is added up from its
//           parts' fp32 sums, in the order of K, by a second kernel.
//
// g, u and da stay in fp32; a, dg and du are rounded to bf16 once, because they are the
// next products' operands (16 bits of each would take a second product; error of y and the
// gradients 0.0023 against 0.0017 for their own rounding alone); y, dx, dW1 and dW2 once more when they are stored (dW in fp32
// on request).  Every wait is bounded as in the library's other tensor-core kernels.
//
// Bound by the tensor cores from about 500 tokens on.  At 8192 x 2048 x 2816 (us and TFLOP/s, single
// launches): gate 104, 1811; y 57, 1655; gradient pass 177, 1600; dx, dW1 and dW2 272, 1737.  A
// tile is 256 x 256 for a pair: 64 KB of operands a K step of 0.33 us, 15 TB/s from L2 over all
// pairs, which a tile of 128 columns would exceed.
#include "hcw.h"
#include "hcw_internal.h"
#include "hcw_ptx.cuh"

#include <mutex>
#include <string.h>

namespace hcw {

namespace {

constexpr int kFM = 128;                     // tile rows per CTA (256 per pair)
constexpr int kFK = 64;                      // K step: one 128-byte row of bf16
constexpr int kFA = kFM * kFK * 2;           // 16 KB: a CTA's rows of A of a stage
constexpr int kFStage = 2 * kFA;             // and its columns of B (128 at most)
constexpr int kFWarps = 8;                   // epilogue warps, two per TMEM lane quarter
constexpr int kFThreads = 64 + 32 * kFWarps;
constexpr uint32_t kFTmem = 512;
constexpr int kFPatch = 2048;                // 32 rows x 64 bytes
constexpr int kFMaxStages = 6;
constexpr unsigned long long kFTimeoutNs = 2000000000ull;

enum FfnMode { FFN_GEMM = 0, FFN_GATE = 1, FFN_GRAD = 2 };

// Stages of the ring and patches of an epilogue warp.  A stage takes about 2,000 cycles from
// its copies' start to their landing, its products 256 to 512: the ring takes the
// shared memory, the patches the rest.
constexpr int ffn_stages(int mode) { return mode == FFN_GRAD ? 5 : 6; }
constexpr int ffn_patches(int mode) { return mode == FFN_GRAD ? 4 : 2; }

struct __align__(8) FfnBars {
    uint64_t full[kFMaxStages];    // leader: both CTAs' copies of a stage landed
    uint64_t empty[kFMaxStages];   // each CTA: the pair's MMAs have read the stage
    uint64_t tfull[2];             // each CTA: accumulators are complete (FFN_GRAD: g, u; da)
    uint64_t tempty[2];            // leader: both CTAs have drained them
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
};

constexpr size_t ffn_smem(int mode) {
    return 1024 + (size_t)ffn_stages(mode) * kFStage + (size_t)kFWarps * ffn_patches(mode) * kFPatch +
           sizeof(FfnBars);
}
static_assert(ffn_smem(FFN_GEMM) <= 232448 && ffn_smem(FFN_GRAD) <= 232448, "shared memory");

// A product C[M][N] = A B over K.  Operands as the library's GEMM reads them: K-major rows
// (box 64 x 128), or MN-major (_mn: a row-major [K][cols] matrix in 64 x 64 boxes).
struct FfnProd {
    CUtensorMap mA, mB;
    CUtensorMap mOut;     // bf16 (N, M) box (32, 32), or fp32 (N, M, 1) box (16, 32, 1)
    int a_mn, b_mn;
    int M, N;
    int bn;               // tile columns: 256 or 128
    int nkb;              // K steps
    int mt, nt;           // tiles
    int unit0, whole;     // first unit of the tiles taken whole, their number
    int line0;            // place on the line of the first tile left over
    int f32;              // fp32 output (mOut)
};

constexpr int kFCuts = 256;   // shares of the line at most
constexpr int kFSlot = 256 * 256;   // floats of a part's sums

// Where the line's shares begin: a tile (by its place on the line) and a K step in it.  Share j
// ends where share j + 1 begins.  Tiles cut alike (`each` parts of each of `tiles`) are taken
// part by part: the pairs that run together then read the same K steps.
struct FfnLine {
    int shares, each, tiles;
    unsigned short tile[kFCuts + 1];
    int step[kFCuts + 1];
};

struct FfnArgs {
    // FFN_GATE: p[0] = (x, W1) -> a.  FFN_GRAD: p[0] = (dy, W2) with mOut dg,
    // p[1] = (x, W1) with mOut du, p[2].mOut a.
    FfnProd p[3];
    int n_prod, n_units;  // units: whole tiles
    CUtensorMap mPart;    // FFN_GEMM: the parts' sums, fp32 (256, 256, slots) box (16, 32, 1)
    FfnLine line;
    int h;                // FFN_GATE / FFN_GRAD: hidden columns (first up row of W1)
    int wide, cut;        // FFN_GRAD: units of 256 hidden columns, and those cut into two of 128
    unsigned long long timeout_ns;
};

__device__ __forceinline__ float ffn_ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float ffn_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// act(g), and in *d its derivative
template <int ACT>
__device__ __forceinline__ float ffn_act(float g, float* d) {
    if (ACT == HCW_GATE_SILU) {
        const float s = ffn_rcp(1.f + ffn_ex2(g * -1.4426950408889634f));
        if (d) *d = s * (1.f + g * (1.f - s));
        return g * s;
    }
    if (ACT == HCW_GATE_GELU) {
        const float c = 0.5f + 0.5f * erff(g * 0.70710678118654752f);
        if (d) *d = c + g * 0.39894228040143268f * ffn_ex2(g * g * -0.72134752044448170f);
        return g * c;
    }
    // (NaN stays NaN, here and in the derivative)
    if (d) *d = g > 0.f ? 1.f : g <= 0.f ? 0.f : g;
    return g <= 0.f ? 0.f : g;
}

// Warp 0 loads, warp 1 issues the products (the pair's leader), eight warps drain TMEM.
template <int MODE, int ACT>
__global__ void __launch_bounds__(kFThreads, 1) ffn_pair_kernel(const __grid_constant__ FfnArgs a) {
    constexpr int kStages = ffn_stages(MODE), kPatches = ffn_patches(MODE);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* staging = smem + (size_t)kStages * kFStage;
    FfnBars* bars = reinterpret_cast<FfnBars*>(staging + kFWarps * kPatches * kFPatch);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = (int)blockIdx.x >> 1, n_pairs = (int)gridDim.x >> 1;
    const uint64_t tmo = a.timeout_ns;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&bars->full[s], 1);
            mbar_init(&bars->empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars->tfull[i], 1);
            mbar_init(&bars->tempty[i], 2 * kFWarps);
        }
        mbar_init(&bars->drain, 1);
        bars->abort = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc_pair(&bars->tmem_base, kFTmem);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();   // both CTAs' barriers exist before any cross-CTA arrive
    tc_fence_after();
    // nothing before this touches global memory
    pdl_wait();
    pdl_trigger();
    const uint32_t tmem_base = bars->tmem_base;
    volatile int* abort = &bars->abort;

    // A unit: a tile (columns fastest: the pairs that run together share rows of A), or K steps
    // [kb0, kb1) of one, whose sums go to a slot.
    struct Unit {
        int q, mi, ni;
        int kb0, kb1, slot;   // FFN_GEMM; slot -1: the whole tile
        bool wide;            // FFN_GRAD
    };
    // The pair's units in turn: whole tiles, then its shares of the line.
    struct Walk {
        int v, turn, j, tile, step;
        bool open;   // inside share j (the turn's), at (tile, step)
    };
    auto next = [&](Walk& w, Unit& t) {
        t.q = t.kb0 = 0;
        t.slot = -1;
        t.wide = false;
        int v = w.v;
        if (v < a.n_units) {
            w.v += n_pairs;
            if (MODE == FFN_GRAD) {
                // ni: the first block of 128 hidden columns; last the odd block of each row
                // tile
                const int cols = a.p[0].nt / 2, k = v - a.wide;
                if (k < 2 * a.cut) {
                    t.wide = k < 0;
                    const int x = t.wide ? v : a.wide + (k >> 1);
                    t.mi = x / cols;
                    t.ni = 2 * (x - t.mi * cols) + (t.wide ? 0 : k & 1);
                } else {
                    t.mi = k - 2 * a.cut;
                    t.ni = a.p[0].nt - 1;
                }
                return true;
            }
            if (MODE == FFN_GEMM) {
                while (t.q + 1 < a.n_prod && v >= a.p[t.q + 1].unit0) ++t.q;
                v -= a.p[t.q].unit0;
            }
            t.kb1 = a.p[t.q].nkb;
        } else if constexpr (MODE != FFN_GEMM) {
            return false;
        } else {
            for (;;) {
                if (w.turn >= a.line.shares) return false;
                if (!w.open) {
                    w.j = a.line.each ? w.turn % a.line.tiles * a.line.each + w.turn / a.line.tiles
                                      : w.turn;
                    w.tile = a.line.tile[w.j];
                    w.step = a.line.step[w.j];
                    w.open = true;
                }
                if (w.tile < a.line.tile[w.j + 1] ||
                    (w.tile == a.line.tile[w.j + 1] && w.step < a.line.step[w.j + 1]))
                    break;
                w.turn += n_pairs;
                w.open = false;
            }
            while (t.q + 1 < a.n_prod && w.tile >= a.p[t.q + 1].line0) ++t.q;
            v = a.p[t.q].whole + w.tile - a.p[t.q].line0;
            const int nkb = a.p[t.q].nkb;
            t.kb0 = w.step;
            t.kb1 = w.tile < a.line.tile[w.j + 1] ? nkb : a.line.step[w.j + 1];
            if (t.kb0 > 0 || t.kb1 < nkb) t.slot = w.tile + w.j;
            ++w.tile;
            w.step = 0;
        }
        t.mi = v / a.p[t.q].nt;
        t.ni = v - t.mi * a.p[t.q].nt;
        return true;
    };
    const Walk start = {pair, pair, 0, 0, 0, false};
    // A unit's passes over K: one product; FFN_GRAD: g and u of the first 128 hidden columns,
    // da of all (under which the first g and u are drained), g and u of the second 128.
    auto passes = [&](const Unit& t) { return MODE != FFN_GRAD ? 1 : t.wide ? 3 : 2; };
    auto product = [&](const Unit& t, int pass) -> const FfnProd& {
        return a.p[MODE == FFN_GEMM ? t.q : MODE == FFN_GRAD && pass != 1 ? 1 : 0];
    };
    auto tile_cols = [&](const Unit& t, int pass, const FfnProd& p) {
        return MODE == FFN_GRAD && pass == 1 ? (t.wide ? 256 : 128) : p.bn;
    };
    auto k_range = [&](const Unit& t, const FfnProd& p, int& kb0, int& kb1) {
        kb0 = t.kb0;
        kb1 = MODE == FFN_GEMM ? t.kb1 : p.nkb;
    };

    if (warp == 0) {
        // ------------------------------------------------------------ producer (both CTAs)
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, issued_mask = 0, issued_phase = 0;
            bool ok = true;
            Walk walk = start;
            for (Unit t; ok && next(walk, t);) {
                for (int pass = 0; pass < passes(t) && ok; ++pass) {
                    const FfnProd& p = product(t, pass);
                    int kb0, kb1;
                    k_range(t, p, kb0, kb1);
                    const int a_mn = p.a_mn, b_mn = p.b_mn;
                    const int bc = tile_cols(t, pass, p) / 2;   // this CTA's columns of B
                    // g and u: gate rows on one CTA, up rows on the other
                    const bool split_b = MODE == FFN_GATE || (MODE == FFN_GRAD && pass != 1);
                    const int a_row = (2 * t.mi + (int)rank) * kFM;
                    const int b_row = split_b ? (int)rank * a.h + (t.ni + (pass >> 1)) * 128
                                              : t.ni * (MODE == FFN_GRAD ? 128 : p.bn) + (int)rank * bc;
                    const uint32_t tx = 2u * (uint32_t)(kFA + bc * kFK * 2);
                    for (int kb = kb0; kb < kb1; ++kb) {
                        if (!mbar_wait(&bars->empty[stage], phase ^ 1, abort, tmo)) {
                            ok = false;
                            break;
                        }
                        uint8_t* sA = smem + (size_t)stage * kFStage;
                        uint8_t* sB = sA + kFA;
                        if (rank == 0) mbar_arrive_expect_tx(&bars->full[stage], tx);
                        issued_mask |= 1u << stage;
                        issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
                        const uint32_t fb = mapa_shared(&bars->full[stage], 0);
                        const int k = kb * kFK;
                        if (a_mn) {
                            tma_load_2d_pair(sA, &p.mA, fb, a_row, k);
                            tma_load_2d_pair(sA + 8192, &p.mA, fb, a_row + 64, k);
                        } else {
                            tma_load_2d_pair(sA, &p.mA, fb, k, a_row);
                        }
                        if (b_mn) {
                            tma_load_2d_pair(sB, &p.mB, fb, b_row, k);
                            if (bc > 64) tma_load_2d_pair(sB + 8192, &p.mB, fb, b_row + 64, k);
                        } else {
                            tma_load_2d_pair(sB, &p.mB, fb, k, b_row);
                        }
                        if (++stage == kStages) {
                            stage = 0;
                            phase ^= 1;
                        }
                    }
                }
            }
            if (rank == 0)
                // every copy of the pair completes on the leader's barriers; also when this
                // warp has issued them all and the one that reads them gave up
                for (int s = 0; s < kStages; ++s)
                    if (issued_mask & (1u << s))
                        mbar_wait_drain(&bars->full[s], (issued_phase >> s) & 1u, tmo);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (leader)
        if (lane == 0 && rank == 0) {
            int stage = 0, it = 0, ig = 0;   // ig: passes of g and u
            uint32_t phase = 0;
            bool ok = true, any = false;
            Walk walk = start;
            for (Unit t; ok && next(walk, t); ++it) {
                for (int pass = 0; pass < passes(t) && ok; ++pass) {
                    const FfnProd& p = product(t, pass);
                    int kb0, kb1;
                    k_range(t, p, kb0, kb1);
                    const uint32_t idesc =
                        idesc_bf16_f32(2 * kFM, tile_cols(t, pass, p), p.a_mn, p.b_mn);
                    // bytes from one 16-deep step to the next within a stage
                    const uint32_t a_step = p.a_mn ? 2048 : 32, b_step = p.b_mn ? 2048 : 32;
                    const uint32_t a_lbo = p.a_mn ? 8192 : 16, b_lbo = p.b_mn ? 8192 : 16;
                    // the accumulator: it % 2, drained of unit it - 2; FFN_GRAD: 0 (g and u) or
                    // 1 (da), drained of its last pass
                    const int acc = MODE == FFN_GRAD ? pass & 1 : it & 1;
                    const int use = MODE != FFN_GRAD ? it >> 1 : acc ? it : ig++;
                    if (!mbar_wait(&bars->tempty[acc], (use & 1) ^ 1, abort, tmo)) ok = false;
                    const uint32_t d_tmem = tmem_base + (uint32_t)acc * 256;
                    if (!ok) break;
                    tc_fence_after();
                    for (int kb = kb0; kb < kb1; ++kb) {
                        if (!mbar_wait(&bars->full[stage], phase, abort, tmo)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        const uint32_t sa = smem_u32(smem + (size_t)stage * kFStage);
                        const uint32_t sb = sa + kFA;
#pragma unroll
                        for (int kk = 0; kk < kFK / 16; ++kk)
                            mma_bf16_f32_pair(d_tmem, smem_desc_sw128(sa + kk * a_step, a_lbo, 1024),
                                              smem_desc_sw128(sb + kk * b_step, b_lbo, 1024), idesc,
                                              (kb != kb0 || kk != 0) ? 1u : 0u);
                        any = true;
                        mma_commit_pair(&bars->empty[stage], 3);
                        if (++stage == kStages) {
                            stage = 0;
                            phase ^= 1;
                        }
                    }
                    if (ok) mma_commit_pair(&bars->tfull[acc], 3);
                }
            }
            if (any) {
                // the pair's MMAs have completed before TMEM can be freed
                mma_commit_pair(&bars->drain, 1);
                mbar_wait_drain(&bars->drain, 0, tmo);
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue (both CTAs)
        // warp e drains TMEM lane quarter warp % 4 (rows 32 q .. 32 q + 31 of this CTA's
        // 128) and half e / 4 of the unit's columns
        const int e = warp - 2;
        const int quarter = warp & 3, chalf = e >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        // Patches of 32 rows x 64 bytes (64-byte swizzle) in a ring.  kTaken of them are
        // filled before the next store is issued, so all but the last kPatches - kTaken stores
        // have to have read theirs first.
        uint8_t* const patches = staging + (size_t)e * kPatches * kFPatch;
        int nbuf = 0;
        constexpr int kTaken = MODE == FFN_GRAD ? 3 : 1;
        auto patches_free = [&]() {
            if (lane == 0) bulk_wait_read<kPatches - kTaken>();
            __syncwarp();
        };
        auto patch = [&]() {
            uint8_t* buf = patches + nbuf * kFPatch;
            nbuf = nbuf + 1 == kPatches ? 0 : nbuf + 1;
            return buf;
        };
        // 16-byte chunk m of this lane's row
        auto chunk = [&](uint8_t* buf, int m) {
            return reinterpret_cast<uint4*>(buf + lane * 64 + ((m ^ (lane >> 1 & 3)) << 4));
        };
        auto store_2d = [&](const CUtensorMap* m, uint8_t* buf, int c, int r) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                tma_store_2d(m, buf, c, r);
                bulk_commit();
            }
        };
        // accumulator i has been read by this warp
        auto release = [&](int i) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote_tmem(mapa_shared(&bars->tempty[i], 0));
        };
        int it = 0, ig = 0;
        bool ok = true;
        Walk walk = start;
        for (Unit t; ok && next(walk, t); ++it) {
            if constexpr (MODE == FFN_GRAD) {
                const int row0 = (2 * t.mi + (int)rank) * kFM + quarter * 32;
#pragma unroll 1
                for (int half = 0; half < (t.wide ? 2 : 1) && ok; ++half, ++ig) {
                    const int col = (t.ni + half) * 128 + chalf * 64;   // the warp's 64 columns
                    const bool st = row0 < a.p[0].M && col < a.h;       // warp-uniform
                    // g and u go to registers at once: the next pass takes their place while
                    // these are worked on
                    const uint32_t tg = tmem_base + lanes + (uint32_t)(chalf * 64);
                    const uint32_t td = tg + 256u + (uint32_t)(half * 128);
                    uint32_t g[64], u[64];
                    ok = __all_sync(0xffffffffu, mbar_wait(&bars->tfull[0], ig & 1, abort, tmo));
                    if (!ok) break;
                    tc_fence_after();
                    if (st) {
#pragma unroll
                        for (int c = 0; c < 64; c += 32) {
                            tmem_ld_32x32b_x32(tg + (uint32_t)c,
                                               *reinterpret_cast<uint32_t(*)[32]>(g + c));
                            tmem_ld_32x32b_x32(tg + (uint32_t)(128 + c),
                                               *reinterpret_cast<uint32_t(*)[32]>(u + c));
                        }
#pragma unroll
                        for (int c = 0; c < 64; c += 32) {
                            tmem_ld_wait_regs(*reinterpret_cast<uint32_t(*)[32]>(g + c));
                            tmem_ld_wait_regs(*reinterpret_cast<uint32_t(*)[32]>(u + c));
                        }
                    }
                    release(0);
                    if (half == 0) {
                        ok = __all_sync(0xffffffffu, mbar_wait(&bars->tfull[1], it & 1, abort, tmo));
                        if (!ok) break;
                        tc_fence_after();
                    }
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        if (!st || col + c >= a.h) break;   // warp-uniform
                        patches_free();
                        uint8_t *const bg = patch(), *const bu = patch(), *const ba = patch();
                        uint32_t d[16];
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            uint32_t wg[4], wu[4], wa[4];
                            if (m % 2 == 0) {
                                __syncwarp();
                                tmem_ld_32x32b_x16(td + (uint32_t)(c + 8 * m), d);
                                tmem_ld_wait_regs(d);
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float og[2], ou[2], oa[2];
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const int q = 8 * m + 2 * j + i;
                                    const float da = __uint_as_float(d[q & 15]);
                                    const float uu = __uint_as_float(u[c + q]);
                                    float dact;
                                    const float ag = ffn_act<ACT>(__uint_as_float(g[c + q]), &dact);
                                    og[i] = da * uu * dact;
                                    ou[i] = da * ag;
                                    oa[i] = ag * uu;
                                }
                                wg[j] = pack_bf16x2(og[0], og[1]);
                                wu[j] = pack_bf16x2(ou[0], ou[1]);
                                wa[j] = pack_bf16x2(oa[0], oa[1]);
                            }
                            *chunk(bg, m) = make_uint4(wg[0], wg[1], wg[2], wg[3]);
                            *chunk(bu, m) = make_uint4(wu[0], wu[1], wu[2], wu[3]);
                            *chunk(ba, m) = make_uint4(wa[0], wa[1], wa[2], wa[3]);
                        }
                        store_2d(&a.p[0].mOut, bg, col + c, row0);
                        store_2d(&a.p[1].mOut, bu, col + c, row0);
                        store_2d(&a.p[2].mOut, ba, col + c, row0);
                    }
                    if (half == (t.wide ? 1 : 0)) release(1);
                }
                continue;
            }
            const FfnProd& p = a.p[MODE == FFN_GEMM ? t.q : 0];
            const int row0 = (2 * t.mi + (int)rank) * kFM + quarter * 32;
            const bool okw = mbar_wait(&bars->tfull[it & 1], (it >> 1) & 1, abort, tmo);
            if (!__all_sync(0xffffffffu, okw)) break;
            tc_fence_after();
            if (MODE == FFN_GEMM) {
                const int cw = p.bn / 2;                       // the warp's columns
                const int colw = t.ni * p.bn + chalf * cw;
                const uint32_t tb = tmem_base + lanes + (uint32_t)((it & 1) * 256 + chalf * cw);
#pragma unroll 1
                for (int c = 0; c < cw; c += 32) {
                    const bool st = row0 < p.M && colw + c < p.N;   // warp-uniform
                    uint32_t r[32];
                    if (st) {
                        __syncwarp();
                        tmem_ld_32x32b_x32(tb + (uint32_t)c, r);
                        tmem_ld_wait_regs(r);
                    }
                    if (c + 32 == cw) release(it & 1);
                    if (!st) continue;
                    if (p.f32 || t.slot >= 0) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (colw + c + 16 * h >= p.N) break;   // warp-uniform
                            patches_free();
                            uint8_t* buf = patch();
#pragma unroll
                            for (int m = 0; m < 4; ++m)
                                *chunk(buf, m) = make_uint4(r[16 * h + 4 * m], r[16 * h + 4 * m + 1],
                                                            r[16 * h + 4 * m + 2], r[16 * h + 4 * m + 3]);
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) {
                                if (t.slot >= 0)
                                    tma_store_3d(&a.mPart, buf, chalf * cw + c + 16 * h,
                                                 (int)rank * kFM + quarter * 32, t.slot);
                                else
                                    tma_store_3d(&p.mOut, buf, colw + c + 16 * h, row0, 0);
                                bulk_commit();
                            }
                        }
                    } else {
                        patches_free();
                        uint8_t* buf = patch();
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            uint32_t w[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                w[j] = pack_bf16x2(__uint_as_float(r[8 * m + 2 * j]),
                                                   __uint_as_float(r[8 * m + 2 * j + 1]));
                            *chunk(buf, m) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        store_2d(&p.mOut, buf, colw + c, row0);
                    }
                }
                continue;
            }
            const int col = t.ni * 128 + chalf * 64;   // the warp's 64 hidden columns
            const bool st = row0 < p.M && col < a.h;
            if (!st) {
                release(it & 1);
                continue;
            }
            if constexpr (MODE == FFN_GATE) {
                const uint32_t tg = tmem_base + lanes + (uint32_t)((it & 1) * 256 + chalf * 64);
#pragma unroll 1
                for (int c = 0; c < 64; c += 32) {
                    uint32_t g[32], u[32];
                    __syncwarp();
                    tmem_ld_32x32b_x32(tg + (uint32_t)c, g);
                    tmem_ld_32x32b_x32(tg + (uint32_t)(128 + c), u);
                    tmem_ld_wait_regs(g);
                    tmem_ld_wait_regs(u);
                    if (c) release(it & 1);
                    if (col + c >= a.h) continue;   // warp-uniform
                    patches_free();
                    uint8_t* buf = patch();
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int i = 8 * m + 2 * j;
                            w[j] = pack_bf16x2(
                                ffn_act<ACT>(__uint_as_float(g[i]), nullptr) * __uint_as_float(u[i]),
                                ffn_act<ACT>(__uint_as_float(g[i + 1]), nullptr) *
                                    __uint_as_float(u[i + 1]));
                        }
                        *chunk(buf, m) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    store_2d(&p.mOut, buf, col + c, row0);
                }
            }
        }
        // every store of this warp is complete before the CTA exits
        if (lane == 0) bulk_wait<0>();
        __syncwarp();
    }

    tc_fence_before();
    __syncthreads();
    cluster_sync_all();   // neither CTA frees the pair's TMEM while the other uses it
    if (*abort) settle_after_abort();   // copies of one CTA that the leader did not get to count
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, kFTmem);
    }
}

// The tiles that were cut, from their parts in the order of K: slots [slot, slot + parts) of tile
// `tile` (by its place on the line).  A block adds 4 rows of a tile; 64 blocks a tile.
struct FfnReduce {
    const float* part;
    struct {
        void* out;
        int M, N, bn, nt, whole, line0, f32;
    } p[3];
    int n_prod;
    struct {
        unsigned short tile, slot, parts;
    } t[kFCuts];
};

__global__ void __launch_bounds__(256) ffn_reduce_kernel(const __grid_constant__ FfnReduce a) {
    pdl_wait();
    pdl_trigger();
    const auto& t = a.t[blockIdx.x >> 6];
    int q = 0;
    while (q + 1 < a.n_prod && t.tile >= a.p[q + 1].line0) ++q;
    const auto& p = a.p[q];
    const int v = p.whole + t.tile - p.line0, mi = v / p.nt, ni = v - mi * p.nt;
    const int r = (int)(blockIdx.x & 63) * 4 + (int)(threadIdx.x >> 6), row = mi * 256 + r;
    const int c = (threadIdx.x & 63) * 4, col = ni * p.bn + c;
    if (c >= p.bn || col >= p.N || row >= p.M) return;
    const float4* src =
        reinterpret_cast<const float4*>(a.part + (size_t)t.slot * kFSlot + r * 256 + c);
    float4 s = *src;
#pragma unroll 4
    for (int i = 1; i < t.parts; ++i) {
        const float4 x = src[(size_t)i * (kFSlot / 4)];
        s.x += x.x;
        s.y += x.y;
        s.z += x.z;
        s.w += x.w;
    }
    const size_t at = (size_t)row * p.N + col;
    if (p.f32)
        *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = s;
    else
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at) =
            make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
}

// Zeros (the weight gradients of no tokens).
__global__ void __launch_bounds__(256) ffn_zero_kernel(uint4* a, size_t na, uint4* b, size_t nb) {
    pdl_wait();
    pdl_trigger();
    for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < na + nb;
         i += (size_t)gridDim.x * blockDim.x)
        (i < na ? a[i] : b[i - na]) = make_uint4(0u, 0u, 0u, 0u);
}

// ------------------------------------------------------------------ few tokens
// out[t][n] = sum_k A[t][k] B[n][k] over T <= 16 MT rows, or with GATED the gate and up
// sums of B's rows n and n_cols + n and act(g) u.  Bound by reading B once (the weights), and
// for narrow blocks by latency.  A CTA (one an SM) takes 8 columns at a time; their weights
// come through a ring in shared memory (bulk copies of row pieces of up to 2048 k, as many on
// their way as fit), and its 16 warps contract a slice of each piece with the warp-level MMA
// (16 rows x 8 columns x 16; of tcgen05's 128 rows all but a few would be empty).  The warps'
// sums are added in warp order.  A lane's 16 bytes of 8 neighbouring k stand for the MMA's
// k in an order of their own, the same for both operands.  The second product's launch
// starts its ring before it waits for the first's.
// Up to 8 tokens (LO) half of the MMA's rows would be empty; they hold what the rounding of a
// to bf16 leaves, itself in bf16, so that a carries 16 bits into the second product at no cost
// and y is rounded once: the first product writes the tokens' rows and, after them, the rows of
// the remainders, the second adds the sums of both.
constexpr int kRowWarps = 16;
constexpr int kRowMax = 32;        // tokens at most
constexpr int kRowLo = 8;          // tokens whose a is kept in two parts, at most
constexpr int kRowPiece = 2048;    // k of a piece at most
constexpr int kRowMaxBufs = 8;

struct FfnRowArgs {
    const __nv_bfloat16* A;   // [T][K]; the second product with LO: [2 T][K]
    const __nv_bfloat16* B;   // [n_cols][K], GATED: [2 n_cols][K]
    __nv_bfloat16* out;       // [T][n_cols]; the first product with LO: [2 T][n_cols]
    int T, K, n_cols;
    int kc, pieces;           // k of a piece (a multiple of 32), pieces of a row
    int bufs;
    int resident;             // A in shared memory, its rows a_stride bytes apart
    int a_stride;
};

// shared memory bytes from one row of a piece to the next: 64 beside the row, so that the MMA
// lanes' 16-byte reads of neighbouring rows fall into different banks
__host__ __device__ constexpr int ffn_row_stride(int kc) { return kc * 2 + 64; }

__device__ __forceinline__ void ffn_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, "
        "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int MT, bool GATED, int ACT, bool LO>
__global__ void __launch_bounds__(32 * kRowWarps + 32) ffn_rows_kernel(const FfnRowArgs a) {
    static_assert(!LO || MT == 1, "the remainders take the second 8 rows of one MMA");
    constexpr int NB = GATED ? 2 : 1;
    constexpr bool kTwo = LO && !GATED;           // two rows of A a token
    constexpr int kRed = MT * NB * 16 * 9;        // floats of a warp's sums
    extern __shared__ __align__(128) uint8_t row_smem[];
    __shared__ uint64_t full[kRowMaxBufs], empty[kRowMaxBufs], a_full;
    __shared__ volatile int gave_up, verdict[2];   // verdict: gave_up as a tile's barrier saw it
    float* const sums = reinterpret_cast<float*>(row_smem);   // [2][kRowWarps][kRed]
    uint8_t* const ring = row_smem + 2 * kRowWarps * kRed * sizeof(float);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, q = lane & 3;   // MMA row (and column of B), and 8 k of a block
    const int tiles = a.n_cols / 8;
    const int n_rows = kTwo ? 2 * a.T : a.T;
    const int stride = ffn_row_stride(a.kc), buf_bytes = NB * 8 * stride;
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.bufs; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], kRowWarps);
        }
        mbar_init(&a_full, 1);
        gave_up = 0;
        fence_mbar_init();
    }
    __syncthreads();
    uint8_t* const a_mem = ring + a.bufs * buf_bytes;
    if (warp == kRowWarps) {
        // producer: a lane a row
        int buf = 0, n_bufs = 0, done = 0;
        uint32_t round = 0;
        bool ok = true, a_done = false;
        // the rows of A, which the kernel before may still be writing
        auto rows_of_a = [&]() {
            if (a_done) return;
            a_done = true;
            pdl_wait();
            if (!a.resident) return;
            if (lane == 0) mbar_arrive_expect_tx(&a_full, (uint32_t)(n_rows * a.K * 2));
            __syncwarp();
            if (lane < n_rows)
                asm volatile(
                    "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes "
                    "[%0], [%1], %2, [%3];" ::"r"(smem_u32(a_mem + lane * a.a_stride)),
                    "l"(a.A + (size_t)lane * a.K), "r"((uint32_t)(a.K * 2)), "r"(smem_u32(&a_full))
                    : "memory");
        };
        // (the second product: first as many weights as the ring holds, which nobody has
        // written since the launch before this one began)
        if (GATED) rows_of_a();
        for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x)
            for (int piece = 0; piece < a.pieces; ++piece) {
                bool w = true;
                if (round) {
                    rows_of_a();
                    w = mbar_wait(&empty[buf], (round & 1) ^ 1, &gave_up, kFTimeoutNs);
                }
                ok = __all_sync(0xffffffffu, w);
                if (!ok) break;
                const int k = piece * a.kc, n = a.K - k < a.kc ? a.K - k : a.kc;
                if (lane == 0) mbar_arrive_expect_tx(&full[buf], (uint32_t)(NB * 8 * n * 2));
                __syncwarp();
                if (lane < NB * 8)
                    asm volatile(
                        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes "
                        "[%0], [%1], %2, [%3];" ::"r"(smem_u32(ring + buf * buf_bytes + lane * stride)),
                        "l"(a.B + ((size_t)(lane >> 3) * a.n_cols + tile * 8 + (lane & 7)) * a.K + k),
                        "r"((uint32_t)(n * 2)), "r"(smem_u32(&full[buf]))
                        : "memory");
                if (n_bufs < a.bufs) ++n_bufs;
                ++done;
                if (++buf == a.bufs) {
                    buf = 0;
                    ++round;
                }
            }
        rows_of_a();
        // every copy has landed before the CTA leaves, also when the others gave up
        if (lane == 0) {
            for (int i = 0; i < n_bufs; ++i)
                mbar_wait_drain(&full[i], ((done - 1 - i) / a.bufs) & 1, kFTimeoutNs);
            if (a.resident) mbar_wait_drain(&a_full, 0, kFTimeoutNs);
        }
        return;
    }
    pdl_wait();
    pdl_trigger();
    const int per = a.kc / 32 + kRowWarps - 1 >> 4;   // blocks of 32 k of a piece a warp takes
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    int b = 0, round = 0, parity = 0;
    bool ok = true;
    const uint8_t* const rows_at = a.resident ? a_mem : reinterpret_cast<const uint8_t*>(a.A);
    if (a.resident) ok = __all_sync(0xffffffffu, mbar_wait(&a_full, 0, &gave_up, kFTimeoutNs));
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, parity ^= 1) {
        float acc[MT][NB][4] = {};
        for (int piece = 0; piece < a.pieces && ok; ++piece) {
            const int k0 = piece * a.kc + warp * per * 32 + q * 8;
            const uint8_t* buf = ring + b * buf_bytes + g * stride + (warp * per * 32 + q * 8) * 2;
            // this warp's part of the rows of A
            auto rows = [&](uint4 (&x)[MT][2], int i) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int t = kTwo ? a.T * h + g : 16 * m + 8 * h + g, k = k0 + 32 * i;
                        const bool row = kTwo ? g < a.T : t < a.T;
                        x[m][h] = i < per && warp * per + i < a.kc / 32 && k < a.K && row
                                      ? *reinterpret_cast<const uint4*>(rows_at + t * a.a_stride + k * 2)
                                      : zero;
                    }
            };
            uint4 x[MT][2];
            rows(x, 0);
            const bool okw = mbar_wait(&full[b], round & 1, &gave_up, kFTimeoutNs);
            ok = __all_sync(0xffffffffu, okw);
            if (!ok) break;
            for (int i = 0; i < per; ++i) {
                uint4 y[MT][2];
                rows(y, i + 1);
                // past the row's end (or the warp's share) A is zero, B nothing that was read
                const bool in = warp * per + i < a.kc / 32 && k0 + 32 * i < a.K;
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const uint4 v = in ? *reinterpret_cast<const uint4*>(buf + n * 8 * stride + i * 64)
                                       : zero;
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        ffn_mma(acc[m][n], x[m][0].x, x[m][1].x, x[m][0].y, x[m][1].y, v.x, v.y);
                        ffn_mma(acc[m][n], x[m][0].z, x[m][1].z, x[m][0].w, x[m][1].w, v.z, v.w);
                    }
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) x[m][h] = y[m][h];
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[b]);
            if (++b == a.bufs) {
                b = 0;
                ++round;
            }
        }
        float* const red = sums + parity * kRowWarps * kRed;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    red[warp * kRed + ((m * NB + n) * 16 + g + 8 * (i >> 1)) * 9 + 2 * q + (i & 1)] =
                        acc[m][n][i];
        // (two buffers: whoever fills this one again has passed the next tile's barrier, which
        // this tile's readers pass after reading)
        if (threadIdx.x == 0) verdict[parity] = gave_up;
        named_bar_sync(1, 32 * kRowWarps);
        ok = !verdict[parity];
        if (!ok) break;
        if ((int)threadIdx.x < MT * 128) {
            const int o = threadIdx.x, m = o >> 7, r = o >> 3 & 15, c = o & 7, t = 16 * m + r;
            float s[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const float* p = red + ((m * NB + n) * 16 + r) * 9 + c;
                s[n] = p[0];
#pragma unroll
                for (int k = 1; k < kRowWarps; ++k) s[n] += p[k * kRed];
                if (kTwo && r < 8) {
                    float lo = p[8 * 9];
#pragma unroll
                    for (int k = 1; k < kRowWarps; ++k) lo += p[k * kRed + 8 * 9];
                    s[n] += lo;
                }
            }
            const float v = GATED ? ffn_act<ACT>(s[0], nullptr) * s[NB - 1] : s[0];
            if (t < a.T) {
                const __nv_bfloat16 hi = __float2bfloat16_rn(v);
                a.out[(size_t)t * a.n_cols + tile * 8 + c] = hi;
                // (an infinite a has no remainder)
                if (LO && GATED)
                    a.out[(size_t)(a.T + t) * a.n_cols + tile * 8 + c] =
                        __float2bfloat16_rn(fabsf(__bfloat162float(hi)) < INFINITY
                                                ? v - __bfloat162float(hi) : 0.f);
            }
        }
    }
}

// ------------------------------------------------------------------ host
typedef CUresult (*FfnEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

FfnEncodeFn ffn_encode() {
    static FfnEncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000,
                                             cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<FfnEncodeFn>(p);
    });
    return fn;
}

// bf16 [rows][cols], ld elements from row to row, in boxes of box_c x box_r
bool ffn_map(CUtensorMap* m, const void* base, long long rows, long long cols, long long ld,
             int box_c, int box_r, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    FfnEncodeFn enc = ffn_encode();
    if (!enc) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    cuuint32_t box[2] = {(cuuint32_t)box_c, (cuuint32_t)box_r};
    cuuint32_t estr[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box,
               estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// an output in patches of 32 x 32
bool ffn_map_out(CUtensorMap* m, void* base, long long rows, long long cols, long long ld) {
    return ffn_map(m, base, rows, cols, ld, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B);
}

// fp32 [splits][M][N] in patches of 32 rows x 16 columns
bool ffn_map_f32(CUtensorMap* m, void* base, int M, int N, int splits) {
    FfnEncodeFn enc = ffn_encode();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)N, (cuuint64_t)M, (cuuint64_t)splits};
    cuuint64_t strides[2] = {(cuuint64_t)N * 4, (cuuint64_t)M * N * 4};
    cuuint32_t box[3] = {16, 32, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, base, dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// An operand: K-major (the row-major [outer][K] matrix) or MN-major (row-major [K][outer]).
bool ffn_operand(CUtensorMap* m, const void* base, long long outer, long long K, bool mn, int rows) {
    return mn ? ffn_map(m, base, K, outer, outer, 64, 64) : ffn_map(m, base, outer, K, K, 64, rows);
}

template <int MODE, int ACT>
cudaError_t ffn_launch(const FfnArgs& a, int pairs, cudaStream_t st) {
    auto kern = ffn_pair_kernel<MODE, ACT>;
    static std::once_flag once[64];
    static cudaError_t set_err[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::call_once(once[dev], [&] {
        set_err[dev] = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                            (int)ffn_smem(MODE));
    });
    if (set_err[dev] != cudaSuccess) return set_err[dev];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.blockDim = dim3((unsigned)kFThreads);
    cfg.dynamicSmemBytes = ffn_smem(MODE);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

template <int MODE>
cudaError_t ffn_launch_act(int act, const FfnArgs& a, int pairs, cudaStream_t st) {
    switch (act) {
        case HCW_GATE_SILU: return ffn_launch<MODE, HCW_GATE_SILU>(a, pairs, st);
        case HCW_GATE_GELU: return ffn_launch<MODE, HCW_GATE_GELU>(a, pairs, st);
        default: return ffn_launch<MODE, HCW_GATE_RELU>(a, pairs, st);
    }
}

template <int MT, bool GATED, int ACT, bool LO>
cudaError_t ffn_rows_launch_mt(FfnRowArgs a, cudaStream_t st) {
    auto kern = ffn_rows_kernel<MT, GATED, ACT, LO>;
    constexpr size_t sums = 2 * kRowWarps * MT * (GATED ? 2 : 1) * 16 * 9 * sizeof(float);
    constexpr size_t room = 232448 - 1024;   // beside the barriers
    static std::once_flag once[64];
    static cudaError_t set_err[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::call_once(once[dev], [&] {
        set_err[dev] =
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)room);
    });
    if (set_err[dev] != cudaSuccess) return set_err[dev];
    a.pieces = (a.K + kRowPiece - 1) / kRowPiece;
    a.kc = ((a.K + a.pieces - 1) / a.pieces + 31) / 32 * 32;
    a.pieces = (a.K + a.kc - 1) / a.kc;
    // A stays in shared memory where it leaves the ring half of it
    a.a_stride = ffn_row_stride(a.K);
    const size_t rows = (size_t)(LO && !GATED ? 2 * a.T : a.T) * a.a_stride;
    a.resident = rows <= (room - sums) / 2;
    if (!a.resident) a.a_stride = a.K * 2;
    const size_t kept = a.resident ? rows : 0;
    const size_t buf = (size_t)(GATED ? 16 : 8) * ffn_row_stride(a.kc);
    const int tiles = a.n_cols / 8, most = device_sms();
    const int grid = tiles < most ? tiles : most;
    const int work = (tiles + grid - 1) / grid * a.pieces;   // pieces of a CTA
    a.bufs = (int)((room - sums - kept) / buf);
    if (a.bufs > work) a.bufs = work;
    if (a.bufs > kRowMaxBufs) a.bufs = kRowMaxBufs;
    return launch_pdl(kern, dim3((unsigned)grid), dim3(32 * kRowWarps + 32),
                      sums + a.bufs * buf + kept, st, a);
}

template <bool GATED, int ACT>
cudaError_t ffn_rows_launch(const FfnRowArgs& a, cudaStream_t st) {
    return a.T <= kRowLo ? ffn_rows_launch_mt<1, GATED, ACT, true>(a, st)
           : a.T <= 16   ? ffn_rows_launch_mt<1, GATED, ACT, false>(a, st)
                         : ffn_rows_launch_mt<2, GATED, ACT, false>(a, st);
}

// Whether the rows kernels are the faster way (us a forward, rows kernels and SM pairs:
// T = 1, d = 512, h = 1024: 6.2, 14.9; 32, 512, 1024: 8.3, 15.2; 1, 2048, 5632: 18, 33;
// 16, 2048, 5632: 22, 27; 32, 2048, 5632: 38, 25; 32, 1024, 4096: 18.6, 19.4;
// 8, 4096, 14336: 88, 88; 16, 4096, 14336: 102, 78).
bool ffn_few(int T, int d, int h) {
    const double work = (double)T * d * h;
    return T <= 16 ? work <= 1 << 28 : T <= kRowMax && work <= 1 << 27;
}

// row tiles of T rows (T up to 2^31 - 1)
int ffn_row_tiles(int T) { return (int)(((long long)T + 255) / 256); }

size_t ffn_round(size_t n) { return (n + 255) & ~(size_t)255; }

// a of up to T tokens: its rows and, up to kRowLo tokens, those of the remainders
size_t ffn_rows_ws_up_to(int T, int h) {
    const size_t two = T < kRowLo ? 2 * T : 2 * kRowLo, rows = (size_t)T > two ? (size_t)T : two;
    return ffn_round(rows * h * 2);
}

// The forward of a few tokens: two launches.
int ffn_rows_fwd(const void* x, const void* W1, const void* W2, int T, int d, int h, int act,
                 void* y, void* ws, cudaStream_t st) {
    FfnRowArgs a = {static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(W1),
                    static_cast<__nv_bfloat16*>(ws), T, d, h, 0, 0, 0, 0, 0};
    const int rc = count_launch(act == HCW_GATE_SILU   ? ffn_rows_launch<true, HCW_GATE_SILU>(a, st)
                                : act == HCW_GATE_GELU ? ffn_rows_launch<true, HCW_GATE_GELU>(a, st)
                                                       : ffn_rows_launch<true, HCW_GATE_RELU>(a, st),
                                1);
    if (rc) return rc;
    FfnRowArgs b = {static_cast<const __nv_bfloat16*>(ws), static_cast<const __nv_bfloat16*>(W2),
                    static_cast<__nv_bfloat16*>(y), T, h, d, 0, 0, 0, 0, 0};
    return count_launch(ffn_rows_launch<false, 0>(b, st), 1);
}

// One product of a gemm launch, as the planner sees it.
struct FfnShape {
    long long M, N, K;
    int out_f32;       // the output itself is fp32
    // filled by the plan
    int bn, nkb, mt, nt;
    int whole, line0;  // tiles taken whole; place on the line of the first of the others
    int tiles() const { return mt * nt; }
    double step() const { return bn == 256 ? 1.0 : 0.75; }   // time of a K step
};

// The products of one launch: s in the order in which the caller named them, order[] in that of
// the launch (the longest tiles first).
struct FfnPlan {
    FfnShape s[3];
    int n, order[3];
    int on_line, slots;
    FfnLine line;
};

// Cuts the line into `shares`: evenly, or (`each` > 0) every tile into that many parts.  No part
// is shorter than kFLeast steps: a cut nearer to a tile's end moves there, one nearer to the cut
// before it (or on it) is left out.
constexpr int kFLeast = 3;
void ffn_cut(FfnPlan& p, int shares, int each) {
    int n = 0;
    double total = 0;
    for (int i = 0; i < p.n; ++i) {
        const FfnShape& s = p.s[p.order[i]];
        total += (double)(s.tiles() - s.whole) * s.nkb * s.step();
    }
    int i = 0;
    double before = 0;   // the line's length up to product i's first tile
    for (int j = 0; j <= shares; ++j) {
        int tile = p.on_line, step = 0;
        if (j < shares && each > 0) {
            tile = j / each;
            while (tile >= p.s[p.order[i]].line0 + p.s[p.order[i]].tiles() - p.s[p.order[i]].whole) ++i;
            step = (int)((long long)p.s[p.order[i]].nkb * (j - tile * each) / each);
        } else if (j < shares) {
            const double at = total * j / shares;
            const FfnShape* s = &p.s[p.order[i]];
            for (;;) {
                const double len = (double)(s->tiles() - s->whole) * s->nkb * s->step();
                if (at < before + len || i + 1 == p.n) break;
                before += len;
                s = &p.s[p.order[++i]];
            }
            const long long steps = (long long)((at - before) / s->step());
            tile = s->line0 + (int)(steps / s->nkb);
            step = (int)(steps % s->nkb);
        }
        if (tile >= p.on_line) {
            tile = p.on_line;
            step = 0;
        } else {
            const int nkb = p.s[p.order[i]].nkb;
            if (step < kFLeast) step = 0;
            if (step > 0 && nkb - step < kFLeast) {
                step = 0;
                ++tile;
            }
        }
        if (n && tile == p.line.tile[n - 1] && step - p.line.step[n - 1] < kFLeast) continue;
        p.line.tile[n] = (unsigned short)tile;
        p.line.step[n++] = step;
    }
    p.line.shares = n - 1;
    p.line.tiles = p.on_line;
    p.line.each = each > 0 && n - 1 == each * p.on_line ? each : 0;
}

// Time of a plan: the busiest pair's K steps (and 2 a unit) at 0.3 us, the parts' sums written
// and read at 15 TB/s where they stay in L2 and at 6 elsewhere, and 3 us for the kernel that adds them.
double ffn_plan_us(FfnPlan& p, int pairs) {
    double most = 0, bytes = 0;
    p.slots = 0;
    for (int pair = 0; pair < pairs; ++pair) {
        double steps = 0;
        int unit0 = 0;
        for (int i = 0; i < p.n; ++i) {   // units pair, pair + pairs, ... of the whole tiles
            const FfnShape& s = p.s[p.order[i]];
            const int first = ((pair - unit0) % pairs + pairs) % pairs;
            if (s.whole > first)
                steps += ((s.whole - first + pairs - 1) / pairs) * (s.nkb * s.step() + 2);
            unit0 += s.whole;
        }
        for (int turn = pair; turn < p.line.shares; turn += pairs) {
            const int j = p.line.each ? turn % p.line.tiles * p.line.each + turn / p.line.tiles : turn;
            int tile = p.line.tile[j], step = p.line.step[j], i = 0;
            const int end = p.line.tile[j + 1], last = p.line.step[j + 1];
            for (; tile < end || (tile == end && step < last); ++tile, step = 0) {
                while (i + 1 < p.n && tile >= p.s[p.order[i + 1]].line0) ++i;
                const FfnShape& s = p.s[p.order[i]];
                const int to = tile < end ? s.nkb : last;
                steps += (to - step) * s.step() + 2;
                if (step > 0 || to < s.nkb) {
                    bytes += 8.0 * s.M * s.N / s.tiles();
                    if (p.slots < tile + j + 1) p.slots = tile + j + 1;
                }
            }
        }
        most = steps > most ? steps : most;
    }
    return most * 0.3 + (bytes > 0 ? bytes / (bytes < 100e6 ? 15.0e6 : 6.0e6) + 3.0 : 0.0);
}

// Every pair takes the same number of whole tiles of each product, and the rest is cut evenly or
// into equal parts of each tile; or all tiles are taken whole.  The least time of these.
// (Backward with even shares, and with dW1's and dW2's tiles in equal parts and all of dx's whole:
// 16384 x 512 x 1024 116 us, 120; 1000 x 2048 x 5632 157, 164; 2048 x 1024 x 2816 101, 107.)
void ffn_plan(FfnPlan& best, int pairs) {
    FfnPlan p = best;
    for (int i = 0; i < p.n; ++i) {
        FfnShape& s = p.s[i];
        s.bn = s.N <= 128 ? 128 : 256;
        s.nkb = (int)((s.K + kFK - 1) / kFK);
        s.mt = (int)((s.M + 255) / 256);
        s.nt = (int)((s.N + s.bn - 1) / s.bn);
        p.order[i] = i;
    }
    for (int i = 0; i < p.n; ++i)
        for (int j = i + 1; j < p.n; ++j)
            if (p.s[p.order[j]].nkb > p.s[p.order[i]].nkb) {
                const int k = p.order[i];
                p.order[i] = p.order[j];
                p.order[j] = k;
            }
    auto lay = [&](bool all) {
        p.on_line = 0;
        for (int i = 0; i < p.n; ++i) {
            FfnShape& s = p.s[p.order[i]];
            s.whole = all ? s.tiles() : s.tiles() / pairs * pairs;
            s.line0 = p.on_line;
            p.on_line += s.tiles() - s.whole;
        }
    };
    double least = -1;
    auto offer = [&]() {
        const double us = ffn_plan_us(p, pairs);
        if (least < 0 || us < least) {
            least = us;
            best = p;
        }
    };
    lay(true);
    ffn_cut(p, 0, 0);
    offer();
    lay(false);
    if (p.on_line < 1 || p.on_line > kFCuts) return;
    // (even shares read K steps all over the operands at a time: only where a product's operands
    // stay in L2.  16384 x 1024 x 2816 backward, 218 MB: 474 us with whole tiles, 511 so)
    double operands = 0;
    for (int i = 0; i < p.n; ++i) {
        const double b = 2.0 * (double)(p.s[i].M + p.s[i].N) * (double)p.s[i].K;
        operands = b > operands ? b : operands;
    }
    if (pairs <= kFCuts && operands < 120e6) {
        ffn_cut(p, pairs, 0);
        offer();
    }
    for (int each = 2; each * p.on_line <= kFCuts && each <= 64; ++each) {
        ffn_cut(p, each * p.on_line, each);
        offer();
    }
}

// The parts' slots.
size_t ffn_part_bytes(const FfnPlan& p) { return (size_t)p.slots * kFSlot * sizeof(float); }

// The most slots of any plan of these products and of ones with smaller M and K (a workspace for
// the longest batch then does for every shorter one, whose tiles may be cut where the longest's
// are not).  On the line lie at most pairs - 1 tiles of a product; a slot is a place on the line
// plus a share, and there are at most kFCuts shares, each with kFLeast steps of a tile at least
// or the tile itself.
size_t ffn_part_bytes_up_to(const FfnShape* s, int n, int pairs) {
    long long line = 0, shares = 0;
    for (int i = 0; i < n; ++i) {
        const long long bn = s[i].N <= 128 ? 128 : 256, nkb = (s[i].K + kFK - 1) / kFK;
        const long long tiles = ((s[i].M + 255) / 256) * ((s[i].N + bn - 1) / bn);
        const long long left = tiles < pairs - 1 ? tiles : pairs - 1;
        line += left;
        shares += left * (nkb < 2 * kFLeast ? 1 : nkb / kFLeast);
    }
    return (size_t)(line + (shares < kFCuts ? shares : kFCuts)) * kFSlot * sizeof(float);
}

// Units of the gradient pass: 256 hidden columns, whose da runs at the rate of 256-column
// products (of 128 columns a K step takes 0.75 of that time, not half), and 128 columns for odd
// ends.  The last round's units are cut in two where that shortens the busiest pair's share.
void ffn_grad_units(FfnArgs& a, int pairs) {
    const int mt = a.p[0].mt, nt = a.p[0].nt, all = mt * (nt / 2), odd = mt * (nt & 1);
    const double k = a.p[0].nkb, whole = 3 * k + 3, half = 1.75 * k + 2;
    double best = 0;
    for (int i = 0; i < 3; ++i) {
        const int cut = i == 0 ? 0 : i == 1 ? all % pairs : all;
        const int wide = all - cut, units = all + cut + odd;
        double most = 0;
        for (int p = 0; p < pairs; ++p) {   // pair p: units p, p + pairs, ...
            const int n = units > p ? (units - p + pairs - 1) / pairs : 0;
            const int w = wide > p ? (wide - p + pairs - 1) / pairs : 0;
            const double t = w * whole + (n - w) * half;
            most = t > most ? t : most;
        }
        if (i == 0 || most < best) {
            best = most;
            a.wide = wide;
            a.cut = cut;
            a.n_units = units;
        }
    }
}

struct FfnOperands {
    const void* A;
    bool a_mn;
    const void* B;
    bool b_mn;
    void* out;
};

// The products of one launch (planned), and the launch that adds the parts of cut tiles.
int ffn_gemms(const FfnPlan& pl, const FfnOperands* o, uint8_t* part, cudaStream_t st) {
    FfnArgs a;
    memset(&a, 0, sizeof(a));
    FfnReduce r;
    r.part = reinterpret_cast<const float*>(part);
    r.n_prod = pl.n;
    int units = 0;
    for (int i = 0; i < pl.n; ++i) {
        const FfnShape& t = pl.s[pl.order[i]];
        const FfnOperands& q = o[pl.order[i]];
        FfnProd& p = a.p[i];
        p.a_mn = q.a_mn;
        p.b_mn = q.b_mn;
        p.M = (int)t.M;
        p.N = (int)t.N;
        p.bn = t.bn;
        p.nkb = t.nkb;
        p.mt = t.mt;
        p.nt = t.nt;
        p.unit0 = units;
        p.whole = t.whole;
        p.line0 = t.line0;
        p.f32 = t.out_f32;
        units += t.whole;
        r.p[i] = {q.out, p.M, p.N, p.bn, p.nt, p.whole, p.line0, p.f32};
        if (!ffn_operand(&p.mA, q.A, t.M, t.K, q.a_mn, kFM) ||
            !ffn_operand(&p.mB, q.B, t.N, t.K, q.b_mn, t.bn / 2) ||
            !(p.f32 ? ffn_map_f32(&p.mOut, q.out, p.M, p.N, 1)
                    : ffn_map_out(&p.mOut, q.out, p.M, p.N, p.N)))
            return HCW_ERR_CUDA;
    }
    a.n_prod = pl.n;
    a.n_units = units;
    a.line = pl.line;
    if (pl.slots && !ffn_map_f32(&a.mPart, part, 256, 256, pl.slots)) return HCW_ERR_CUDA;
    a.timeout_ns = kFTimeoutNs;
    // the tiles that share j + 1 continues, with all their parts
    int cut = 0;
    for (int j = 1; j < pl.line.shares; ++j) {
        if (!pl.line.step[j]) continue;
        const int tile = pl.line.tile[j];
        if (cut && r.t[cut - 1].tile == tile) {
            r.t[cut - 1].parts = (unsigned short)(tile + j - r.t[cut - 1].slot + 1);
        } else {
            r.t[cut].tile = (unsigned short)tile;
            r.t[cut].slot = (unsigned short)(tile + j - 1);
            r.t[cut++].parts = 2;
        }
    }
    const int pairs = device_sms() / 2, most = units > pl.line.shares ? units : pl.line.shares;
    const int rc = count_launch(ffn_launch<FFN_GEMM, 0>(a, most < pairs ? most : pairs, st), 1);
    if (rc || !cut) return rc;
    return count_launch(launch_pdl(ffn_reduce_kernel, dim3((unsigned)cut * 64u), dim3(256), 0, st, r), 1);
}

// The plan of these products (their sizes in `want`), kept by its sizes: the thread's last few
// (a plan costs 10 to 25 us of the host's time, and a training step or a served model repeats
// the same ones).
const FfnPlan& ffn_planned(const FfnShape* want, int n, int pairs) {
    struct Entry {
        FfnPlan p;
        int pairs;
    };
    constexpr int kEntries = 8;
    thread_local Entry kept[kEntries];
    thread_local int next = 0;
    for (const Entry& e : kept) {
        bool same = e.p.n == n && e.pairs == pairs;
        for (int i = 0; i < n && same; ++i)
            same = e.p.s[i].M == want[i].M && e.p.s[i].N == want[i].N && e.p.s[i].K == want[i].K &&
                   e.p.s[i].out_f32 == want[i].out_f32;
        if (same) return e.p;
    }
    Entry& e = kept[next];
    next = (next + 1) % kEntries;
    memset(&e.p, 0, sizeof(e.p));
    e.pairs = pairs;
    e.p.n = n;
    for (int i = 0; i < n; ++i) e.p.s[i] = want[i];
    ffn_plan(e.p, pairs);
    return e.p;
}

// Forward workspace: a [T][h] bf16, then the parts of y.
const FfnPlan& ffn_down_plan(int T, int d, int h) {
    const FfnShape s = {T, d, h};
    return ffn_planned(&s, 1, device_sms() / 2);
}

size_t ffn_fwd_ws_bytes(int T, int d, int h) {
    const size_t rows = ffn_rows_ws_up_to(T, h);
    if (ffn_few(T, d, h)) return rows;   // and so are fewer tokens
    const FfnShape s = {T, d, h};
    return rows + ffn_part_bytes_up_to(&s, 1, device_sms() / 2);
}

// Backward workspace: [dg | du] [T][2h] and a [T][h] bf16, then the parts of dx, dW1 and dW2.
struct FfnBwdWs {
    size_t act, part, bytes;   // dgu at 0
    const FfnPlan* plan;       // until the thread's next plan
};

int ffn_bwd_shapes(FfnShape (&s)[3], int T, int d, int h, bool dx, bool dw, bool f32) {
    int n = 0;
    if (dx) s[n++] = {T, d, 2ll * h};
    if (dw) {
        s[n++] = {2ll * h, d, T, f32};
        s[n++] = {d, h, T, f32};
    }
    return n;
}

FfnBwdWs ffn_bwd_ws(int T, int d, int h, bool dx, bool dw, bool f32) {
    FfnBwdWs w;
    FfnShape s[3] = {};
    const int n = ffn_bwd_shapes(s, T, d, h, dx, dw, f32);
    w.plan = &ffn_planned(s, n, device_sms() / 2);
    w.act = ffn_round((size_t)T * 2 * h * 2);
    w.part = w.act + ffn_round((size_t)T * h * 2);
    w.bytes = w.part + ffn_part_bytes(*w.plan);
    return w;
}

size_t ffn_bwd_ws_bytes(int T, int d, int h) {
    FfnShape s[3] = {};
    const int n = ffn_bwd_shapes(s, T, d, h, true, true, false);
    return ffn_round((size_t)T * 2 * h * 2) + ffn_round((size_t)T * h * 2) +
           ffn_part_bytes_up_to(s, n, device_sms() / 2);
}

bool ffn_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct FfnSpan {
    const void* p;
    size_t n;
};

bool ffn_meet(const FfnSpan& a, const FfnSpan& b) {
    if (!a.p || !b.p || !a.n || !b.n) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x < y + b.n && y < x + a.n;
}

int ffn_sizes(int T, int d, int h, int act) {
    if (T < 0 || d < 1 || h < 1 || (act != HCW_GATE_SILU && act != HCW_GATE_GELU && act != HCW_GATE_RELU))
        return HCW_ERR_INVALID_ARG;
    // TMA reads rows of a multiple of 16 bytes; the tiles of a product are counted in ints
    if (d % 8 || h % 8 || d > (1 << 20) || h > (1 << 20)) return HCW_ERR_UNSUPPORTED;
    return HCW_OK;
}

int ffn_check(const FfnSpan* in, int n_in, const FfnSpan* out, int n_out) {
    for (int i = 0; i < n_in; ++i)
        if (!ffn_aligned(in[i].p)) return HCW_ERR_ALIGNMENT;
    for (int i = 0; i < n_out; ++i)
        if (!ffn_aligned(out[i].p)) return HCW_ERR_ALIGNMENT;
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (ffn_meet(out[i], in[j])) return HCW_ERR_ALIASING;
        for (int j = i + 1; j < n_out; ++j)
            if (ffn_meet(out[i], out[j])) return HCW_ERR_ALIASING;
    }
    return HCW_OK;
}

}  // namespace

cudaError_t ffn_error_word_read_clear(int* word) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(word, g_error_word, sizeof(int));
    if (e == cudaSuccess && *word) e = cudaMemcpyToSymbol(g_error_word, &zero, sizeof(int));
    return e;
}

}  // namespace hcw

using namespace hcw;

extern "C" {

size_t hcw_gated_ffn_fwd_workspace_bytes(int T, int d, int h) {
    return T < 1 || ffn_sizes(T, d, h, HCW_GATE_SILU) ? 0 : ffn_fwd_ws_bytes(T, d, h);
}

int hcw_gated_ffn_fwd(const void* x, const void* W1, const void* W2, int T, int d, int h, int act,
                      void* y, void* workspace, size_t ws_bytes, void* stream) {
    int rc = ffn_sizes(T, d, h, act);
    if (rc) return rc;
    const size_t xb = (size_t)T * d * 2, wb = (size_t)d * h * 2;
    const FfnSpan in[] = {{x, xb}, {W1, 2 * wb}, {W2, wb}};
    const FfnSpan out[] = {{y, xb}, {workspace, workspace ? ws_bytes : 0}};
    rc = ffn_check(in, 3, out, 2);
    if (rc) return rc;
    if (T == 0) return HCW_OK;
    if (!x || !W1 || !W2 || !y) return HCW_ERR_INVALID_ARG;
    if (!workspace || ws_bytes < ffn_fwd_ws_bytes(T, d, h)) return HCW_ERR_WORKSPACE;
    const size_t act_bytes = ffn_round((size_t)T * h * 2);
    const cudaStream_t st = (cudaStream_t)stream;
    if (ffn_few(T, d, h)) return ffn_rows_fwd(x, W1, W2, T, d, h, act, y, workspace, st);
    const FfnPlan& plan = ffn_down_plan(T, d, h);
    if (ws_bytes < act_bytes + ffn_part_bytes(plan)) return HCW_ERR_WORKSPACE;
    const int pairs = device_sms() / 2;
    FfnArgs a;
    memset(&a, 0, sizeof(a));
    FfnProd& p = a.p[0];
    p.M = T;
    p.N = h;
    p.bn = 256;
    p.nkb = (d + kFK - 1) / kFK;
    p.mt = ffn_row_tiles(T);
    p.nt = (h + 127) / 128;
    a.n_prod = 1;
    a.n_units = p.mt * p.nt;
    a.h = h;
    a.timeout_ns = kFTimeoutNs;
    if (!ffn_operand(&p.mA, x, T, d, false, kFM) || !ffn_operand(&p.mB, W1, 2ll * h, d, false, 128) ||
        !ffn_map_out(&p.mOut, workspace, T, h, h))
        return HCW_ERR_CUDA;
    rc = count_launch(ffn_launch_act<FFN_GATE>(act, a, a.n_units < pairs ? a.n_units : pairs, st), 1);
    if (rc) return rc;
    const FfnOperands o = {workspace, false, W2, false, y};
    return ffn_gemms(plan, &o, static_cast<uint8_t*>(workspace) + act_bytes, st);
}

size_t hcw_gated_ffn_bwd_workspace_bytes(int T, int d, int h) {
    return T < 1 || ffn_sizes(T, d, h, HCW_GATE_SILU) ? 0 : ffn_bwd_ws_bytes(T, d, h);
}

int hcw_gated_ffn_bwd(const void* x, const void* dy, const void* W1, const void* W2, int T, int d,
                      int h, int act, int dw_dtype, void* dx, void* dW1, void* dW2,
                      void* workspace, size_t ws_bytes, void* stream) {
    int rc = ffn_sizes(T, d, h, act);
    if (rc) return rc;
    if (dw_dtype != HCW_BF16 && dw_dtype != HCW_F32) return HCW_ERR_INVALID_ARG;
    const bool f32 = dw_dtype == HCW_F32;
    const size_t xb = (size_t)T * d * 2, wb = (size_t)d * h * 2, gb = f32 ? 2 * wb : wb;
    const FfnSpan in[] = {{x, xb}, {dy, xb}, {W1, 2 * wb}, {W2, wb}};
    const FfnSpan out[] = {{dx, xb}, {dW1, 2 * gb}, {dW2, gb}, {workspace, workspace ? ws_bytes : 0}};
    rc = ffn_check(in, 4, out, 4);
    if (rc) return rc;
    if (!dW1 != !dW2) return HCW_ERR_INVALID_ARG;
    const cudaStream_t st = (cudaStream_t)stream;
    if (T == 0) {
        if (!dW1) return HCW_OK;
        return count_launch(launch_pdl(ffn_zero_kernel, dim3((unsigned)device_sms() * 4), dim3(256), 0,
                                       st, static_cast<uint4*>(dW1), 2 * gb / 16,
                                       static_cast<uint4*>(dW2), gb / 16), 1);
    }
    if (!x || !dy || !W1 || !W2 || (!dx && !dW1)) return HCW_ERR_INVALID_ARG;
    const FfnBwdWs w = ffn_bwd_ws(T, d, h, dx != nullptr, dW1 != nullptr, f32);
    if (!workspace || ws_bytes < ffn_bwd_ws_bytes(T, d, h) || ws_bytes < w.bytes)
        return HCW_ERR_WORKSPACE;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const int pairs = device_sms() / 2;
    FfnArgs a;
    memset(&a, 0, sizeof(a));
    for (int i = 0; i < 2; ++i) {
        FfnProd& p = a.p[i];
        p.M = T;
        p.N = h;
        p.bn = i == 0 ? 128 : 256;
        p.b_mn = i == 0;
        p.nkb = (d + kFK - 1) / kFK;
        p.mt = ffn_row_tiles(T);
        p.nt = (h + 127) / 128;
    }
    a.n_prod = 2;
    ffn_grad_units(a, pairs);
    a.h = h;
    a.timeout_ns = kFTimeoutNs;
    if (!ffn_operand(&a.p[0].mA, dy, T, d, false, kFM) ||
        !ffn_operand(&a.p[0].mB, W2, h, d, true, 0) ||
        !ffn_operand(&a.p[1].mA, x, T, d, false, kFM) ||
        !ffn_operand(&a.p[1].mB, W1, 2ll * h, d, false, 128) ||
        !ffn_map_out(&a.p[0].mOut, ws, T, h, 2ll * h) ||
        !ffn_map_out(&a.p[1].mOut, ws + (size_t)h * 2, T, h, 2ll * h) ||
        !ffn_map_out(&a.p[2].mOut, ws + w.act, T, h, h))
        return HCW_ERR_CUDA;
    rc = count_launch(ffn_launch_act<FFN_GRAD>(act, a, a.n_units < pairs ? a.n_units : pairs, st), 1);
    if (rc) return rc;
    FfnOperands o[3];
    int n = 0;
    if (dx) o[n++] = {ws, false, W1, true, dx};
    if (dW1) {
        o[n++] = {ws, true, x, true, dW1};
        o[n++] = {dy, true, ws + w.act, true, dW2};
    }
    return ffn_gemms(*w.plan, o, ws + w.part, st);
}

}  // extern "C"
