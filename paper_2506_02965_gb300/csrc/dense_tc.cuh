// Dense matrix products on the tensor cores (tcgen05, sm_103a) with a caller's epilogue:
//   acc[g][m][n] = sum over k of A[g][m][k] * B[g][n][k],   16-bit operands (bf16, or fp16), fp32 accumulators,
// for G matrices of one size, each operand stored with its contraction dimension inside (K-major) or outside
// (MN-major). What is not here, and is in the experts' grouped kernel: groups of rows of their own lengths. What is
// here: contractions cut into splits, only the tiles on and below the diagonal of a symmetric product, matrices that are
// left out, and epilogues as types.
//
// A persistent grid of CTA pairs with 256 x 256 tiles (cta_group::2: each CTA holds half of both operands'
// rows), or of single CTAs with 128 x 128 tiles for problems of few tiles. Warp 0 copies by TMA, a stage is 128
// contraction terms as two 64 x 128 boxes of each operand (64 KiB, three stages; see AR), warp 1 issues the MMAs into one of
// two accumulators, the others run the epilogue of the other. What bounds a launch with a contraction of some
// thousand terms is the tensor pipe under the power cap; the epilogues are measured where they are.
//
// Waits are bounded: on a timeout the CTA records MOE_ERR_TIMEOUT, lets its copies and MMAs land, frees TMEM, returns.
#pragma once

#include <cuda_fp16.h>

#include <algorithm>

#include "moe_internal.h"
#include "tc_ptx.cuh"

namespace moe {
namespace dense {

using namespace tc;

constexpr int KST = 128;                      // contraction terms per stage
constexpr uint32_t BOX_BYTES = 64 * 128 * 2;  // one operand box (128 rows, or 128 contraction terms)
// AR: rows of A that a CTA holds, 128, or 32 (single CTAs, K-major A): a few rows leave room for more stages, and what
// such a launch waits for is B on its way (7 rows against 65536 x 2048: 75 us with three stages of 128 rows of both;
// narrower tiles of B only make more stages of the same 1.1 us). The MMA reads 128 rows all the same: what follows the
// box, bytes that only reach accumulator rows that nobody reads.
constexpr uint32_t stage_bytes(int ar) { return 2 * (uint32_t)ar * 128 + 2 * BOX_BYTES; }
constexpr int stages_of(int ar) { return ar == 128 ? 3 : 5; }
constexpr int OUT_BOX = 32, OUT_BOX_BYTES = OUT_BOX * OUT_BOX * 2;  // epilogue staging: 32 x 32 of 16 bits
constexpr int out_boxes(int ar) { return ar == 128 ? 16 : 8; }
constexpr int smem_bytes(int ar) { return 1024 + stages_of(ar) * (int)stage_bytes(ar) + out_boxes(ar) * OUT_BOX_BYTES; }
constexpr int MAX_GROUPS = 256;
static_assert(smem_bytes(128) + 2048 <= 227 * 1024 && smem_bytes(32) + 2048 <= 227 * 1024, "shared memory of one SM");

__host__ __device__ constexpr int threads(int ew) { return 64 + 32 * ew; }

struct Problem {
    int M, N, K, G;
    int splits;     // of the contraction, each of `per_split` stages (the last may have fewer)
    int per_split;
    int tri;        // tiles on and below the diagonal only (M == N)
    int tail;       // tiles in flight at once, if a last round of few is cut into parts (see Tail; splits == 1); else 0
    int band;       // tile order: bands of this many rows of tiles
    int tn;         // AR = 32: a tile's columns, a multiple of 16 up to 128
    const int32_t* counts;  // [G]: matrices with counts <= 0 are left out; null: none
    uint64_t wait_ns;
};

struct Tile {
    int g, split;
    int m0, n0;    // of this CTA's accumulator rows, and of the tile's columns
    int kb0, kb1;  // stages
    bool diag;     // (tri) a tile that the diagonal crosses
    int part;      // of a cut tile, counted over all of them; -1: a whole one
};

// The last round of tiles: `rest` of them behind `whole`, each in `parts` parts of `each` stages (1: not cut), so that
// as many parts as there are places fill it. Sums of the parts are left to another launch.
struct Tail {
    int whole, rest, parts, each;
};
__host__ __device__ __forceinline__ Tail tail_of(int tiles, int places, int stages) {
    Tail t{tiles, 0, 1, stages};
    const int rest = places ? tiles % places : 0;
    if (rest == 0 || places / rest < 2 || stages < 2) return t;
    t.each = (stages + places / rest - 1) / (places / rest);
    t.parts = (stages + t.each - 1) / t.each;
    t.rest = rest;
    t.whole = tiles - rest;
    return t;
}
// The matrices that take part, in order; by a warp. Returns how many.
__device__ __forceinline__ int called_groups(const int32_t* counts, int G, unsigned char* list) {
    const int lane = threadIdx.x & 31;
    int run = 0;
    for (int g0 = 0; g0 < G; g0 += 32) {
        const int g = g0 + lane;
        const bool in = g < G && (!counts || counts[g] > 0);
        const uint32_t m = __ballot_sync(0xffffffffu, in);
        if (in) list[run + __popc(m & ((1u << lane) - 1))] = (unsigned char)g;
        run += __popc(m);
    }
    return run;
}
// Row and column of tiles of the i-th tile on and below the diagonal
__device__ __forceinline__ int2 lower_tile(int i) {
    int m = (int)((sqrtf(8.f * (float)i + 1.f) - 1.f) * 0.5f);
    while (m * (m + 1) / 2 > i) --m;
    while ((m + 1) * (m + 2) / 2 <= i) ++m;
    return make_int2(m, i - m * (m + 1) / 2);
}

// What an epilogue gets besides its tile: this warp's TMEM address, its lane quarter, the share of the columns
// [c0, c1) that it drains, and its staging boxes.
struct Warp {
    uint32_t tmem;
    int q, lane, c0, c1;
    uint8_t* box;
    uint32_t box_u32;
    uint32_t seq;  // boxes used so far
};

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, uint32_t cluster_bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"((uint64_t)map), "r"(cluster_bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"((uint64_t)map), "r"(src),
                 "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}
// An epilogue that reads nothing beside the product.
struct Plain {
    static constexpr bool CUT = false;  // takes parts of cut tiles (see Tail)
    template <int CHUNKS> struct Held {};
    template <int NBUF, typename H> __device__ __forceinline__ void fetch(H&, const Problem&, const Tile&, Warp&) const {}
};
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// A product's fp32 sums, [splits][G][M][N] (N a multiple of 4), stored or (ADD) added to what is there.
template <bool ADD> struct SumEpi {
    static constexpr bool CUT = false;
    template <int CHUNKS> struct Held {};
    template <int NBUF, typename H> __device__ __forceinline__ void fetch(H&, const Problem&, const Tile&, Warp&) const {}
    float* sums;

    template <int NBUF, typename H> __device__ __forceinline__ void run(const H&, const Problem& p, const Tile& ti, Warp& w, const CUtensorMap*) const {
        const int m = ti.m0 + w.q * 32 + w.lane;
        float* at = sums + (((int64_t)ti.split * p.G + ti.g) * p.M + m) * p.N;
#pragma unroll 1
        for (int c = w.c0; c < w.c1 && ti.n0 + c < p.N; c += 32) {
            float v[32];
            tmem_ld32(w.tmem + c, v);
            if (m < p.M) {
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    if (ti.n0 + c + i >= p.N) break;
                    float4* to = reinterpret_cast<float4*>(at + ti.n0 + c + i);
                    float4 s = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    if (ADD) {
                        const float4 b = *to;
                        s = make_float4(s.x + b.x, s.y + b.y, s.z + b.z, s.w + b.w);
                    }
                    *to = s;
                }
            }
        }
    }
};

// 32 columns of this lane's row, as 16 words of two 16-bit values, through a staging box to the output map (which
// cuts what lies outside the matrix). NBUF boxes per warp, each store in flight until its box is needed again.
template <int NBUF>
__device__ __forceinline__ void store_box(Warp& w, const CUtensorMap* map, const uint32_t (&v)[16], int col, int row, int g) {
    const uint32_t b = w.seq % NBUF;
    if (w.lane == 0) bulk_wait_read<NBUF - 1>();
    __syncwarp();
    uint8_t* base = w.box + b * OUT_BOX_BYTES + w.lane * 64;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *reinterpret_cast<uint4*>(base + ((c ^ ((w.lane >> 1) & 3)) << 4)) = make_uint4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
    fence_proxy_async();
    __syncwarp();
    if (w.lane == 0) {
        tma_store_3d(map, w.box_u32 + b * OUT_BOX_BYTES, col, row, g);
        bulk_commit();
    }
    ++w.seq;
}

template <bool A_MN, bool B_MN, bool PAIR, bool F16, int EW, int AR, typename Epi>
__global__ void __launch_bounds__(threads(EW), 1)
    dense_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmO,
                 const __grid_constant__ Problem p, const __grid_constant__ Epi epi) {
    // as pdl_begin(), but what needs no other kernel's writes comes before the wait: barriers, TMEM, the copies' descriptors
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int NPAIR = PAIR ? 2 : 1;
    constexpr int TM = 128 * NPAIR, TN = 128 * NPAIR;
    static_assert(AR == 128 || (AR == 32 && !PAIR && !A_MN), "rows of A");
    constexpr int NST = stages_of(AR);
    constexpr uint32_t STAGE_BYTES = stage_bytes(AR), BOX_A = (uint32_t)AR * 128;
    constexpr uint32_t IDESC = instr_desc<TN, A_MN, B_MN, TM>() & ~(F16 ? (1u << 7) | (1u << 10) : 0u);
    constexpr int TMEM_COLS = 2 * TN;
    constexpr int SPLIT = EW / 4;  // warps that share a lane quarter's columns
    constexpr int NBUF = out_boxes(AR) / EW;
    static_assert(EW == 4 || EW == 8, "epilogue warps");

    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * NST + 5];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_active;
    __shared__ uint32_t s_fills;
    __shared__ unsigned char s_group[MAX_GROUPS];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &s_abort;
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int tile0 = (int)blockIdx.x / NPAIR, tile_step = (int)gridDim.x / NPAIR;

    // 1024-byte aligned ring, the staging boxes behind it
    const uint32_t raw_u32 = smem_u32(smem_raw);
    const uint32_t ring = raw_u32 + ((1024u - (raw_u32 & 1023u)) & 1023u);
    uint8_t* stage_out = smem_raw + (ring - raw_u32) + NST * STAGE_BYTES;
    const uint32_t bar0 = smem_u32(&bars[0]);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (NST + s); };
    auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * NST + a); };
    auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * NST + 2 + a); };
    const uint32_t drain_bar = bar0 + 8u * (2 * NST + 4);
    auto wait_bar = [&](uint32_t bar, uint32_t parity) -> bool {
        if constexpr (PAIR) {
            if (mbar_try_cluster(bar, parity)) return true;
            const uint64_t t0 = gtimer();
            for (;;) {
                if (mbar_try_cluster(bar, parity)) return true;
                if (*abort_flag) return false;
                if (gtimer() - t0 > p.wait_ns) {
                    *abort_flag = 1;
                    record_status(MOE_ERR_TIMEOUT);
                    return false;
                }
            }
        } else {
            return mbar_wait(bar, parity, abort_flag, p.wait_ns);
        }
    };
    auto warp_wait = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, wait_bar(bar, parity)); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < NST; ++s) {
            mbar_init(full_bar(s), 1);  // the (leader's) producer arms it for both CTAs' bytes
            mbar_init(empty_bar(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), EW * NPAIR);
        }
        mbar_init(drain_bar, 1);
        s_fills = 0;
        s_abort = 0;
        for (const CUtensorMap* m : {&tmA, &tmB, &tmO}) asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)m) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(TMEM_COLS)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(TMEM_COLS)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 0) {  // the matrices that take part
        const int run = called_groups(p.counts, p.G, s_group);
        if (lane == 0) s_active = run;
    }
    fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();  // the peer's barriers are initialised
    fence_after();
    const int tn = AR == 32 ? p.tn : TN;  // a tile's columns
    const int mt = (p.M + TM - 1) / TM, nt = (p.N + tn - 1) / tn;
    const int per = p.tri ? mt * (mt + 1) / 2 : mt * nt;
    const int stages = (p.K + KST - 1) / KST;
    Tail tail{s_active * p.splits * per, 0, 1, stages};
    if constexpr (Epi::CUT) tail = tail_of(tail.whole, p.tail, stages);
    const int total = tail.whole + tail.rest * tail.parts;

    auto tile_at = [&](int t) -> Tile {
        Tile ti;
        ti.part = -1;
        int k = 0;
        if (Epi::CUT && t >= tail.whole) {
            ti.part = t - tail.whole;
            k = ti.part % tail.parts;
            t = tail.whole + ti.part / tail.parts;
        }
        const int gs = t / per;
        const int local = t - gs * per;
        ti.g = s_group[gs / p.splits];
        ti.split = gs % p.splits;
        int m, n;
        if (p.tri) {
            const int2 mn = lower_tile(local);
            m = mn.x;
            n = mn.y;
        } else {  // bands of p.band rows of tiles, swept along N, a band's rows innermost
            const int b = local / (p.band * nt);
            const int first = b * p.band, rows = min(p.band, mt - first);
            const int rem = local - first * nt;
            m = first + rem % rows;
            n = rem / rows;
        }
        ti.diag = m == n;
        ti.m0 = m * TM + (int)rank * 128;
        ti.n0 = n * tn;
        ti.kb0 = ti.split * p.per_split;
        ti.kb1 = min(stages, ti.kb0 + p.per_split);
        if (Epi::CUT && ti.part >= 0) {
            ti.kb0 = k * tail.each;
            ti.kb1 = min(stages, ti.kb0 + tail.each);
        }
        return ti;
    };

    const uint32_t tmem_base = s_tmem;
    // waits for work in flight (microseconds): not shortened with the caller's limit
    const uint64_t drain_limit = p.wait_ns > 200000000ull ? p.wait_ns : 200000000ull;
    auto drain = [&](uint32_t bar, uint32_t parity) {
        const uint64_t t0 = gtimer();
        while (!mbar_try(bar, parity) && gtimer() - t0 < drain_limit) {
        }
    };

    if (warp == 0) {
        // ------------------------------------------------------------ copies
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0, fills = 0;
            bool ok = true;
            const uint32_t full0 = PAIR ? map_to_rank(bar0, 0) : bar0;
            auto load = [&](uint32_t dst, const CUtensorMap* map, uint32_t fb, int c0, int c1, int c2) {
                if constexpr (PAIR) tma_load_3d_pair(dst, map, fb, c0, c1, c2);
                else tma_load_3d(dst, map, fb, c0, c1, c2);
            };
            for (int t = tile0; t < total && ok; t += tile_step) {
                const Tile ti = tile_at(t);
                const int n0 = ti.n0 + (int)rank * 128;
                for (int kb = ti.kb0; kb < ti.kb1; ++kb) {
                    if (!wait_bar(empty_bar(stage), phase ^ 1u)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sa = ring + stage * STAGE_BYTES, sb = sa + 2 * BOX_A;
                    const uint32_t fb = full0 + 8u * stage;
                    // only the leader arrives, for the bytes of both CTAs; the peer's copies complete on its
                    // barrier, after the leader's MMAs released the stage to both
                    if (rank == 0) mbar_expect_tx(full_bar(stage), AR == 32 ? 2u * BOX_A + 256u * (uint32_t)tn : NPAIR * STAGE_BYTES);
                    const int k0 = kb * KST;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if constexpr (A_MN) load(sa + i * BOX_A, &tmA, fb, ti.m0 + 64 * i, k0, ti.g);
                        else load(sa + i * BOX_A, &tmA, fb, k0 + 64 * i, ti.m0, ti.g);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if constexpr (B_MN) load(sb + i * BOX_BYTES, &tmB, fb, n0 + 64 * i, k0, ti.g);
                        else load(sb + i * BOX_BYTES, &tmB, fb, k0 + 64 * i, n0, ti.g);
                    }
                    ++fills;
                    if (++stage == NST) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            s_fills = fills;
            if (rank == 0)  // every copy lands before the CTAs exit (after a whole launch at once)
                for (uint32_t i = fills > NST ? fills - NST : 0; i < fills; ++i) drain(full_bar(i % NST), (i / NST) & 1u);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMAs (a pair's leader for both)
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool issued = false;
        const uint32_t idesc = AR == 32 ? (IDESC & ~(63u << 17)) | (uint32_t)(tn >> 3) << 17 : IDESC;
        for (int t = tile0; t < total && rank == 0; t += tile_step) {
            const Tile ti = tile_at(t);
            bool ok = warp_wait(tempty_bar(acc), acc_phase ^ 1u);
            if (!ok) break;
            fence_after();
            const uint32_t d = tmem_base + (uint32_t)(acc * TN);
            for (int kb = ti.kb0; kb < ti.kb1; ++kb) {
                const bool got = wait_bar(full_bar(stage), phase);
                fence_after();
                if (lane == 0 && got) {
                    const uint32_t sa = ring + stage * STAGE_BYTES, sb = sa + 2 * BOX_A;
#pragma unroll
                    for (int kk = 0; kk < KST / 16; ++kk) {
                        const uint64_t ad = A_MN ? smem_desc(sa + kk * 2048, BOX_BYTES, 1024)
                                                 : smem_desc(sa + (kk / 4) * BOX_A + (kk % 4) * 32, 16, 1024);
                        const uint64_t bd = B_MN ? smem_desc(sb + kk * 2048, BOX_BYTES, 1024)
                                                 : smem_desc(sb + (kk / 4) * BOX_BYTES + (kk % 4) * 32, 16, 1024);
                        const uint32_t more = kb > ti.kb0 || kk > 0 ? 1u : 0u;
                        if constexpr (PAIR) mma_bf16_pair(d, ad, bd, idesc, more);
                        else mma_bf16(d, ad, bd, idesc, more);
                    }
                    if constexpr (PAIR) mma_commit_pair(empty_bar(stage), 3);
                    else mma_commit(empty_bar(stage));
                    issued = true;
                }
                if (!__all_sync(0xffffffffu, got)) {
                    ok = false;
                    break;
                }
                if (++stage == NST) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (!ok) break;
            if (lane == 0) {
                if constexpr (PAIR) mma_commit_pair(tfull_bar(acc), 3);
                else mma_commit(tfull_bar(acc));
            }
            __syncwarp();
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
            }
        }
        if (lane == 0 && issued) {  // every MMA of this CTA has run before TMEM is released
            if constexpr (PAIR) mma_commit_pair(drain_bar, 1);
            else mma_commit(drain_bar);
            drain(drain_bar, 0);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue: warp w drains lane quarter w % 4
        Warp w;
        w.q = warp & 3;
        w.lane = lane;
        const int part = (warp - 2) >> 2;
        w.c0 = part * (TN / SPLIT);
        w.c1 = w.c0 + TN / SPLIT;
        w.box = stage_out + (warp - 2) * NBUF * OUT_BOX_BYTES;
        w.box_u32 = smem_u32(w.box);
        w.seq = 0;
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int t = tile0; t < total; t += tile_step) {
            const Tile ti = tile_at(t);
            typename Epi::template Held<TN / SPLIT / 32> held;  // what the epilogue reads, on its way during the product
            epi.template fetch<NBUF>(held, p, ti, w);
            if (!warp_wait(tfull_bar(acc), acc_phase)) break;
            fence_after();
            w.tmem = tmem_base + ((uint32_t)(w.q * 32) << 16) + (uint32_t)(acc * TN);
            epi.template run<NBUF>(held, p, ti, w, &tmO);
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) {
                    fence_release_smem_cluster();
                    mbar_arrive_remote(map_to_rank(tempty_bar(acc), 0));
                } else {
                    mbar_arrive(tempty_bar(acc));
                }
            }
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
            }
        }
        if (lane == 0) bulk_wait0();
    }
    fence_before();
    __syncthreads();
    if constexpr (PAIR) {
        if (threadIdx.x == 0 && *abort_flag) st_cluster(map_to_rank(smem_u32(&s_abort), rank ^ 1u), 1u);
        __syncwarp();
        cluster_sync_all();  // neither CTA leaves while the pair's MMAs run
        if (*abort_flag) {   // (both CTAs see it)
            // stages that the peer filled and the leader, giving up first, never armed
            if (rank == 0 && threadIdx.x == 0) {
                const uint32_t theirs = ld_cluster(map_to_rank(smem_u32(&s_fills), 1));
                for (uint32_t i = s_fills; i < theirs; ++i) {
                    mbar_expect_tx(full_bar(i % NST), STAGE_BYTES);
                    drain(full_bar(i % NST), (i / NST) & 1u);
                }
            }
            __syncwarp();
            cluster_sync_all();
        }
    }
    fence_after();
    if (warp == 1) {
        if constexpr (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// ------------------------------------------------------------------------ host side
// A stack of G matrices [outer, inner], rows `ld` and matrices `group` elements apart (16 bytes or a multiple). As an
// operand: boxes of 64 x 128 (box_rows: an A of 32 rows, a K-major B of tn), zeros outside; as an output: boxes of 32 x 32, nothing written outside.
bool make_map3(CUtensorMap* m, const void* base, int64_t inner, int64_t outer, int64_t ld, int G, int64_t group, bool store,
               int box_rows = 128);

template <bool A_MN, bool B_MN, bool PAIR, bool F16, int EW, int AR = 128, typename Epi>
static cudaError_t launch_as(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, Problem p, const Epi& epi, cudaStream_t s) {
    constexpr int TM = PAIR ? 256 : 128, TN = TM, SMEM = smem_bytes(AR);
    auto kern = dense_kernel<A_MN, B_MN, PAIR, F16, EW, AR, Epi>;
    cudaError_t e = allow_dynamic_smem<dense_kernel<A_MN, B_MN, PAIR, F16, EW, AR, Epi>>(SMEM);
    if (e != cudaSuccess) return e;
    if (AR != 32) p.tn = TN;
    const int64_t mt = (p.M + TM - 1) / TM, nt = (p.N + p.tn - 1) / p.tn;
    const int64_t tiles = (int64_t)p.G * p.splits * (p.tri ? mt * (mt + 1) / 2 : mt * nt);
    if (tiles <= 0) return cudaSuccess;
    if (tiles > 0x7fffff00) return cudaErrorInvalidValue;  // (terabytes)
    int most = sm_count();
    if constexpr (PAIR) {  // clusters that fit at once
        static std::atomic<int> resident[kMaxDevices] = {};
        const int dev = current_device();
        most = dev >= 0 && dev < kMaxDevices ? resident[dev].load() : 0;
        if (!most) {
            cudaLaunchConfig_t q = {};
            q.gridDim = dim3(2 * (sm_count() / 2));
            q.blockDim = dim3(threads(EW));
            q.dynamicSmemBytes = SMEM;
            cudaLaunchAttribute qa[1];
            qa[0].id = cudaLaunchAttributeClusterDimension;
            qa[0].val.clusterDim.x = 2;
            qa[0].val.clusterDim.y = qa[0].val.clusterDim.z = 1;
            q.attrs = qa;
            q.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&most, kern, &q) != cudaSuccess || most <= 0) {
                (void)cudaGetLastError();
                most = sm_count() / 2;
            }
            if (dev >= 0 && dev < kMaxDevices) resident[dev] = most;
        }
    }
    const int at_once = (int)std::min<int64_t>(p.tail ? std::max<int64_t>(tiles, p.tail) : tiles, most);
    // Tile order: where one operand of a matrix fits the L2 beside what streams past it, the other is read once;
    // else bands of about the square root of the tiles in flight, which read the fewest blocks per round.
    constexpr int64_t kResident = 48ll << 20;
    if ((int64_t)p.N * p.K * 2 <= kResident) p.band = 1;
    else if ((int64_t)p.M * p.K * 2 <= kResident) p.band = (int)mt;
    else {
        p.band = 1;
        while ((p.band + 1) * (p.band + 1) <= at_once) ++p.band;
    }
    p.wait_ns = wait_limit_ns();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)at_once * (PAIR ? 2 : 1));
    cfg.blockDim = dim3(threads(EW));
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = PAIR ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a, b, o, p, epi);
}

static inline Problem problem(int M, int N, int K, int G = 1) {
    Problem p{};
    p.M = M;
    p.N = N;
    p.K = K;
    p.G = G;
    p.splits = 1;
    p.per_split = (K + KST - 1) / KST;
    p.tn = 128;
    return p;
}
static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kPairs = 76;  // CTA pairs of the part: the rules below also size workspaces, and do not ask the device
struct Shape {
    bool pair;
    int splits;
};
// Pair tiles or single ones, and splits: those by which a launch takes least from first to last, in units of a pair's
// stage: rounds of tiles times the stages of one (and two for its start and end), a 128 x 128 tile's stage being 0.92
// of a pair's (a quarter of the operations, half of the operands' bytes per SM). With splits, also the partial
// sums' way through memory (a stage is 0.7 us; 6.5 TB/s) and a launch.
static inline Shape pick_shape(int64_t M, int64_t N, int64_t K, int max_splits, int64_t G = 1, bool tri = false) {
    const int64_t stages = ceil_div(K, KST);
    Shape best{true, 1};
    double least = 0;
    for (int pair = 1; pair >= 0; --pair) {
        const int64_t t = pair ? 256 : 128, mt = ceil_div(M, t), tiles = G * (tri ? mt * (mt + 1) / 2 : mt * ceil_div(N, t));
        for (int s = 1; s <= max_splits && s <= stages; ++s) {
            const int64_t each = ceil_div(stages, s), real = ceil_div(stages, each);
            const int64_t rounds = ceil_div(tiles * real, pair ? kPairs : 2 * kPairs);
            const double cost = (double)rounds * ((double)each + 2) * (pair ? 1.0 : 0.92) +
                                (real > 1 ? 5 + (double)real * G * M * N * 8 / (6.5e6 * 0.7) : 0);
            if (least == 0 || cost < least) {
                least = cost;
                best = {pair != 0, (int)real};
            }
        }
    }
    return best;
}

// cuts the contraction into about n splits of whole stages, none empty
static inline void split_k(Problem& p, int n) {
    const int stages = (p.K + KST - 1) / KST;
    p.per_split = (stages + n - 1) / n;
    p.splits = (stages + p.per_split - 1) / p.per_split;
}

}  // namespace dense
}  // namespace moe
