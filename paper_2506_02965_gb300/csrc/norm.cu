// Layer norm in front of a layer: h = x + residual, y = (h - mean) rstd gamma + beta, and its
// backward with the reduction of the weights' gradients. Both directions are HBM-bound: every input
// is read once and every output written once.
//
// A team of TEAM threads (8 to 1024) takes one row after another, VPT spans of 16 bytes a thread, and
// holds it in registers: the mean, then the variance about it (no difference of large sums), then
// the row is written. CTAs are persistent; every thread copies its own spans of the team's next rows
// to shared memory (cp.async, read back by the same thread, so that no thread waits for another's
// copy), which keeps the memory busy across the team's reductions with few registers.
//
// Rows that are no whole number of 16-byte spans start at any element of one. A span then belongs to
// the row from its element `lo` = span * VW - shift on, shift = (row * d) mod VW; the rows of a team are
// a multiple of VW / gcd(d, VW) apart, so that a team's shift, and with it the columns of a thread and
// their gamma, stay the same. The first span of a row may hold the end of the row before it
// (masked), the last is copied up to the row's end.
//
// Measured (of the copy rate, 6781 GB/s): 16384 x 4096 bf16 with residual and checkpoint, forward 92.1 us (0.97), backward
// from the checkpoint 80.3 (0.87); without a residual 47.9 (0.83) and 68.0 (0.87); 8000 x 8192 with one 88.8 and 85.3;
// 8000 x 4096 fp32 42.7 and 63.7; 60000 x 333 (spans at every shift, a third of a team's idle) 32.4 (0.36) and 39.4
// (0.45); 4000 x 16384 (one team of 1024 threads an SM, no second one to work while it waits) 85 and 133 (0.45). A CTA per
// row took 92.7 and 116 us for the first, 60.9 and 210 for the 333.
// Farthest from the copy rate: narrow ragged rows, whose teams idle most and whose checkpoint is a pass of its own (60000 x
// 130 bf16, residual, checkpoint, 48.2 us, 0.22, and 30.1, 0.27; 60000 x 333 67.4 and 52.8, 0.39; 30000 x 1001 0.54 and 0.57), and
// ragged rows of more than 1024 spans, whose teams of 1024 threads hold 64 registers each and whose backwards spill (4000 x
// 16383 bf16, four spans a thread: 224 us, 0.17, and 271, 0.21, 540 bytes spilled; of two spans 144, from a checkpoint 568 and 232).
#include <algorithm>
#include <numeric>

#include "moe_common.cuh"
#include "moe_internal.h"
#include "span.cuh"

namespace moe {

constexpr int NORM_SMEM = 216 * 1024;  // of an SM, for the rows on their way

// Sum over the team, the same in all its threads. `red` holds TEAM / 32 floats per value that no
// earlier reduction still reads; teams of several warps have a barrier each (bar: 1 + the team's
// number; 0 where the team is the CTA).
template <int TEAM, int N> __device__ __forceinline__ void team_sum(float (&v)[N], float* red, int bar) {
    constexpr int LANES = TEAM < 32 ? TEAM : 32, W = TEAM / 32;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (TEAM > 32) {
        const int w = threadIdx.x % TEAM / 32;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) red[w * N + i] = v[i];
        }
        asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(TEAM) : "memory");
        float r[W * N];
        static_assert(W * N % 2 == 0);
        if constexpr (W * N % 4 == 0) {
#pragma unroll
            for (int j = 0; j < W * N; j += 4) *reinterpret_cast<float4*>(r + j) = *reinterpret_cast<const float4*>(red + j);
        } else {
#pragma unroll
            for (int j = 0; j < W * N; j += 2) *reinterpret_cast<float2*>(r + j) = *reinterpret_cast<const float2*>(red + j);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += r[j * N + i];
    }
}

// BYTES (4, 8, 16) to shared memory, `valid` of them from src and zeros after
template <int BYTES> __device__ __forceinline__ void copy_async(void* dst, const void* src, int valid) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(valid) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(d), "l"(src), "n"(BYTES), "r"(valid) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until at most n of the latest groups are on their way (n < 4)
__device__ __forceinline__ void copy_wait(int n) {
    if (n >= 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// A thread's spans of its team's rows. AL: rows are whole spans (d % VW == 0, no shift).
template <typename T, int VPT, int TEAM, bool AL> struct Spans {
    static constexpr int VW = 16 / (int)sizeof(T);
    int d, shift, tid;
    __device__ __forceinline__ Spans(int d_, int64_t row) : d(d_), shift(AL ? 0 : (int)((row * d_) % VW)), tid(threadIdx.x % TEAM) {}
    __device__ __forceinline__ int lo(int i) const { return (i * TEAM + tid) * VW - (AL ? 0 : shift); }  // the span's first column
    __device__ __forceinline__ bool any(int i) const { return lo(i) < d; }
    __device__ __forceinline__ bool whole(int i) const { return AL ? lo(i) < d : lo(i) >= 0 && lo(i) + VW <= d; }
    __device__ __forceinline__ int valid(int i) const { return AL ? VW : min(VW, d - lo(i)); }  // elements up to the row's end
    // elements before the row's start as zeros (those past its end were copied as such)
    __device__ __forceinline__ void mask(int i, float (&f)[VW]) const {
        if constexpr (!AL) {
            if (lo(i) < 0) {
#pragma unroll
                for (int j = 0; j < VW; ++j)
                    if (lo(i) + j < 0) f[j] = 0.f;
            }
        }
    }
    // where span 0 of a row starts; span i lies i * STEP elements on
    static constexpr int STEP = TEAM * VW;
    __device__ __forceinline__ int64_t start(int64_t row) const { return row * d + lo(0); }
    __device__ __forceinline__ void store(T* p, int i, const float (&f)[VW]) const {
        Span<T, VW> s;
        s.pack(f);
        store(p, i, s);
    }
    __device__ __forceinline__ void store(T* p, int i, const Span<T, VW>& s) const {
        if (whole(i)) {
            s.store(p + i * STEP);
        } else if constexpr (!AL) {
            float f[VW];
            s.unpack(f);
#pragma unroll
            for (int j = 0; j < VW; ++j)
                if (lo(i) + j >= 0 && lo(i) + j < d) Elem<T>::store(p + i * STEP + j, f[j]);
        }
    }
    // a vector over the columns, 0 outside of the row
    __device__ __forceinline__ void columns(const float* p, int i, float (&f)[VW]) const {
        if ((AL || shift == 0) && whole(i) && ((uintptr_t)p & 15) == 0) {
#pragma unroll
            for (int j = 0; j < VW; j += 4) {
                const float4 v = *reinterpret_cast<const float4*>(p + lo(i) + j);
                f[j] = v.x; f[j + 1] = v.y; f[j + 2] = v.z; f[j + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < VW; ++j) f[j] = lo(i) + j >= 0 && lo(i) + j < d ? p[lo(i) + j] : 0.f;
        }
    }
};

struct NormFwdArgs {
    int64_t rows;
    int d;
    const void *x, *res;
    const float *gamma, *beta;
    float eps;
    void *h, *y;
    float *mean, *rstd;
    int8_t* q;  // with d % VW == 0 only
    float* q_scale;
    int stages;
};

template <int TEAM> constexpr int norm_fwd_threads() { return TEAM < 256 ? 256 : TEAM; }
// gamma and beta stay in registers where there is room: 128 a thread up to 512 threads an SM, 64 for 1024
constexpr bool norm_fwd_hold(int elems, int team, bool al) { return team <= 256 || elems <= 8 || (!al && team == 512); }  // elems: of a thread
constexpr int norm_fwd_resident(int elems, int team, bool al) { return team <= 256 || (team == 512 && (al || elems <= 8)) ? 2 : 1; }

template <typename T, int VPT, int TEAM, bool AL>
__global__ void __launch_bounds__(norm_fwd_threads<TEAM>(), norm_fwd_resident(VPT * 16 / (int)sizeof(T), TEAM, AL)) norm_fwd_kernel(
    const __grid_constant__ NormFwdArgs a) {
    pdl_begin();
    constexpr int THREADS = norm_fwd_threads<TEAM>(), TEAMS = THREADS / TEAM, VW = 16 / (int)sizeof(T);
    constexpr int W = TEAM < 32 ? 1 : TEAM / 32;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ __align__(16) float red[TEAMS][2][W < 4 ? 4 : W];
    const int team = threadIdx.x / TEAM, bar = TEAMS > 1 ? 1 + team : 0;
    const int64_t row0 = (int64_t)team * gridDim.x + blockIdx.x, step = (int64_t)gridDim.x * TEAMS;
    const int rounds = (int)((a.rows - blockIdx.x + step - 1) / step);  // of the CTA's first team: the others have as many or one less
    const Spans<T, VPT, TEAM, AL> sp(a.d, row0);
    // stage s of this thread: VPT spans of x, then of the residual, 16 bytes apart by threads
    const int S = a.stages, per = a.res ? 2 : 1;
    uint4* ring = reinterpret_cast<uint4*>(smem) + threadIdx.x;
    auto slot = [&](int s, int what, int i) { return ring + ((s * per + what) * VPT + i) * THREADS; };
    auto fetch = [&](int round, int s) {
        const int64_t r = row0 + round * step;
        if (r < a.rows) {
            const int64_t at = sp.start(r);
            const T *x = (const T*)a.x + at, *res = (const T*)a.res + at;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (sp.any(i)) {
                    const int bytes = sp.valid(i) * (int)sizeof(T);
                    copy_async<16>(slot(s, 0, i), x + i * sp.STEP, bytes);
                    if (a.res) copy_async<16>(slot(s, 1, i), res + i * sp.STEP, bytes);
                }
        }
        copy_commit();
    };
    for (int s = 0; s < S; ++s) fetch(s, s);
    constexpr bool HOLD = norm_fwd_hold(VPT * VW, TEAM, AL);
    float gm[HOLD ? VPT : 1][VW], bt[HOLD ? VPT : 1][VW];
    if constexpr (HOLD) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
#pragma unroll
            for (int j = 0; j < VW; ++j) gm[i][j] = bt[i][j] = 0.f;
            if (sp.any(i)) {
                sp.columns(a.gamma, i, gm[i]);
                if (a.beta) sp.columns(a.beta, i, bt[i]);
            }
        }
    }
    const float inv_d = 1.f / (float)a.d;
    for (int round = 0, s = 0; round < rounds; ++round, s = s + 1 == S ? 0 : s + 1) {
        const int64_t row = row0 + round * step, at = sp.start(row);
        const bool on = row < a.rows;
        copy_wait(S - 1);
        float v[VPT][VW];
        Span<T, VW> h[VPT];
        float sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const bool here = on && sp.any(i);
            h[i].zero();
            if (here) *reinterpret_cast<uint4*>(h[i].w) = *slot(s, 0, i);
            h[i].unpack(v[i]);
            if (a.res && here) {
                Span<T, VW> r;
                float f[VW];
                *reinterpret_cast<uint4*>(r.w) = *slot(s, 1, i);
                r.unpack(f);
#pragma unroll
                for (int j = 0; j < VW; ++j) v[i][j] += f[j];
                h[i].pack(v[i]);
                sp.store((T*)a.h + at, i, h[i]);
            }
            sp.mask(i, v[i]);
#pragma unroll
            for (int j = 0; j < VW; ++j) sum[0] += v[i][j];
        }
        fetch(round + S, s);
        // the statistics are those of the fp32 sum, before it is rounded for storing
        team_sum<TEAM>(sum, red[team][0], bar);
        const float mean = sum[0] * inv_d;
        float sq[1] = {0.f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
#pragma unroll
            for (int j = 0; j < VW; ++j) v[i][j] -= mean;
            if (sp.whole(i)) {
#pragma unroll
                for (int j = 0; j < VW; ++j) sq[0] = fmaf(v[i][j], v[i][j], sq[0]);
            } else if constexpr (!AL) {
#pragma unroll
                for (int j = 0; j < VW; ++j)
                    if (sp.lo(i) + j >= 0 && sp.lo(i) + j < a.d) sq[0] = fmaf(v[i][j], v[i][j], sq[0]);
            }
        }
        team_sum<TEAM>(sq, red[team][1], bar);
        const float rstd = rsqrtf(fmaf(sq[0], inv_d, a.eps));
        if (on && sp.tid == 0 && a.mean) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        if (AL && a.q) {  // the stored h, 128 columns in 128 / VW lanes (a team has that many, or the row is one block)
            constexpr int LANES = CKPT_BLOCK / VW < TEAM ? CKPT_BLOCK / VW : TEAM;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float f[VW], scale, inv;
                block_scale(lanes_max<LANES>(h[i].largest_bits()), scale, inv);
                if (on && sp.any(i)) {
                    const int c = i * TEAM + sp.tid;
                    int8_t* q = a.q + at + i * sp.STEP;
                    h[i].unpack(f);
                    if constexpr (VW == 8)
                        *reinterpret_cast<uint2*>(q) = make_uint2(quant4(f[0], f[1], f[2], f[3], inv), quant4(f[4], f[5], f[6], f[7], inv));
                    else *reinterpret_cast<uint32_t*>(q) = quant4(f[0], f[1], f[2], f[3], inv);
                    if (c % (CKPT_BLOCK / VW) == 0)
                        a.q_scale[row * ((a.d + CKPT_BLOCK - 1) / CKPT_BLOCK) + c / (CKPT_BLOCK / VW)] = scale;
                }
            }
        }
        if (on) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (sp.any(i)) {
                    float f[VW], g[VW], b[VW];
                    if constexpr (!HOLD) {
#pragma unroll
                        for (int j = 0; j < VW; ++j) b[j] = 0.f;
                        sp.columns(a.gamma, i, g);
                        if (a.beta) sp.columns(a.beta, i, b);
                    }
#pragma unroll
                    for (int j = 0; j < VW; ++j)
                        f[j] = fmaf(v[i][j] * rstd, HOLD ? gm[HOLD ? i : 0][j] : g[j], HOLD ? bt[HOLD ? i : 0][j] : b[j]);
                    sp.store((T*)a.y + at, i, f);
                }
        }
    }
    copy_wait(0);
}

struct NormBwdArgs {
    int64_t rows;
    int d;
    const void *dy, *h;
    const int8_t* q;
    const float* q_scale;
    const float *mean, *rstd, *gamma;
    const void* dh;
    void* dx;
    float *part_g, *part_b;  // [CTAs, d]; part_b null without dbeta
    int stages;
};

// With xh = (h - mean) rstd and g = dy gamma,
//   dx = dh + rstd (g - <g>/d - xh <g, xh>/d),
// and the thread's columns of sum dy xh and sum dy in registers over all rows of its team. A CTA's teams' are
// added up in order in shared memory, and norm_reduce_kernel the CTAs', in order too. Where there is room g, xh and
// gamma of a row stay in registers over its reduction (128 a thread up to 512 threads an SM); larger teams make
// them again from the copies in shared memory. Q: the states come from their 8-bit checkpoint.
template <int TEAM> constexpr int norm_bwd_threads() { return TEAM < 512 ? 512 : TEAM; }
constexpr bool norm_bwd_hold(int team) { return team <= 512; }
constexpr int norm_bwd_resident(int elems, int team) { return team == 512 && elems <= 8 ? 2 : 1; }  // elems: of a thread

template <typename T, int VPT, int TEAM, bool Q, bool AL>
__global__ void __launch_bounds__(norm_bwd_threads<TEAM>(), norm_bwd_resident(VPT * 16 / (int)sizeof(T), TEAM)) norm_bwd_kernel(const __grid_constant__ NormBwdArgs a) {
    pdl_begin();
    constexpr int THREADS = norm_bwd_threads<TEAM>(), TEAMS = THREADS / TEAM, VW = 16 / (int)sizeof(T);
    constexpr int W = TEAM < 32 ? 1 : TEAM / 32;
    constexpr bool HOLD = norm_bwd_hold(TEAM);
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ __align__(16) float red[TEAMS][2][W < 2 ? 4 : 2 * W];
    // per stage the row's mean and rstd and, of a checkpoint of whole spans, its blocks' scales, copied by the first
    // of the SL or QL lanes that read them
    constexpr int SL = TEAM < 32 ? TEAM : 32, QL = CKPT_BLOCK / VW < TEAM ? CKPT_BLOCK / VW : TEAM;
    __shared__ float s_stat[4][2][THREADS / SL], s_scale[4][Q && AL ? VPT : 1][Q && AL ? THREADS / QL : 1];
    const int team = threadIdx.x / TEAM, bar = TEAMS > 1 ? 1 + team : 0;
    const int64_t row0 = (int64_t)team * gridDim.x + blockIdx.x, step = (int64_t)gridDim.x * TEAMS;
    const int rounds = (int)((a.rows - blockIdx.x + step - 1) / step);
    const int nb = (a.d + CKPT_BLOCK - 1) / CKPT_BLOCK;
    const float inv_d = 1.f / (float)a.d;
    const Spans<T, VPT, TEAM, AL> sp(a.d, row0);
    // stage s of this thread: spans of dy, of dh, of h (or VW bytes of its checkpoint)
    const int S = a.stages, per = a.dh ? 2 : 1;
    constexpr int HB = Q ? VW : 16;  // bytes of a span of the states
    uint4* ring = reinterpret_cast<uint4*>(smem) + threadIdx.x;
    uint8_t* ring_h = smem + (size_t)S * per * VPT * THREADS * 16 + threadIdx.x * HB;
    auto slot = [&](int s, int what, int i) { return ring + ((s * per + what) * VPT + i) * THREADS; };
    auto slot_h = [&](int s, int i) { return ring_h + (size_t)(s * VPT + i) * THREADS * HB; };
    auto fetch = [&](int round, int s) {
        const int64_t r = row0 + round * step;
        if (r < a.rows) {
            const int64_t at = sp.start(r);
            const T *dy = (const T*)a.dy + at, *dh = (const T*)a.dh + at, *h = (const T*)a.h + at;
            const int8_t* q = a.q + at;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (sp.any(i)) {
                    const int n = sp.valid(i);
                    copy_async<16>(slot(s, 0, i), dy + i * sp.STEP, n * (int)sizeof(T));
                    if (a.dh) copy_async<16>(slot(s, 1, i), dh + i * sp.STEP, n * (int)sizeof(T));
                    if constexpr (Q) copy_async<HB>(slot_h(s, i), q + i * sp.STEP, n);
                    else copy_async<HB>(slot_h(s, i), h + i * sp.STEP, n * (int)sizeof(T));
                    if (Q && AL && sp.tid % QL == 0)
                        copy_async<4>(&s_scale[s][i][threadIdx.x / QL], a.q_scale + r * nb + sp.lo(i) / CKPT_BLOCK, 4);
                }
            if (sp.tid % SL == 0) {
                copy_async<4>(&s_stat[s][0][threadIdx.x / SL], a.mean + r, 4);
                copy_async<4>(&s_stat[s][1][threadIdx.x / SL], a.rstd + r, 4);
            }
        }
        copy_commit();
    };
    for (int s = 0; s < S; ++s) fetch(s, s);
    float pg[VPT][VW], pb[VPT][VW], gm[HOLD ? VPT : 1][VW];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
#pragma unroll
        for (int j = 0; j < VW; ++j) pg[i][j] = pb[i][j] = 0.f;
        if constexpr (HOLD) {
#pragma unroll
            for (int j = 0; j < VW; ++j) gm[i][j] = 0.f;
            if (sp.any(i)) sp.columns(a.gamma, i, gm[i]);
        }
    }
    // The scales of rows that are no whole spans one row ahead: a span's columns lie in one block or in two, the
    // second from its element `split` on.
    float sc_n[VPT][2];
    auto ahead = [&](int round) {
        const int64_t r = row0 + round * step;
        if (r >= a.rows) return;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (sp.any(i)) {
                const int b = max(sp.lo(i), 0) / CKPT_BLOCK;
                sc_n[i][0] = a.q_scale[r * nb + b];
                sc_n[i][1] = b + 1 < nb ? a.q_scale[r * nb + b + 1] : 0.f;
            }
    };
    if constexpr (Q && !AL) ahead(0);
    for (int round = 0, s = 0; round < rounds; ++round, s = s + 1 == S ? 0 : s + 1) {
        const int64_t row = row0 + round * step, at = sp.start(row);
        const bool on = row < a.rows;
        copy_wait(S - 1);
        __syncwarp();  // its first lanes' copies
        const float mean = s_stat[s][0][threadIdx.x / SL], rs = s_stat[s][1][threadIdx.x / SL];  // (past the rows: of no use)
        float sc[VPT][2];
        if constexpr (Q) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                sc[i][0] = (AL ? s_scale[s][i][threadIdx.x / QL] : sc_n[i][0]) * rs;
                if constexpr (!AL) sc[i][1] = sc_n[i][1] * rs;
            }
            if constexpr (!AL) ahead(round + 1);
        }
        float hg[HOLD ? VPT : 1][VW], hx[HOLD ? VPT : 1][VW], sum[2] = {0.f, 0.f};
        // dy, xh and gamma of a span
        auto take = [&](int i, float (&dy)[VW], float (&xh)[VW]) {
            Span<T, VW> sy, sh;
            *reinterpret_cast<uint4*>(sy.w) = *slot(s, 0, i);
            sy.unpack(dy);
            sp.mask(i, dy);
            if constexpr (Q) {
                uint32_t w[VW / 4];
                float f[VW];
                if constexpr (VW == 8) {
                    const uint2 u = *reinterpret_cast<const uint2*>(slot_h(s, i));
                    w[0] = u.x;
                    w[1] = u.y;
                } else w[0] = *reinterpret_cast<const uint32_t*>(slot_h(s, i));
#pragma unroll
                for (int j = 0; j < VW / 4; ++j) unquant4(w[j], f + 4 * j);
                // q scale rstd - mean rstd: off by the rounding of the held value, as its difference with the mean is
                const float mr = -mean * rs;
                if (AL || sp.shift == 0) {
#pragma unroll
                    for (int j = 0; j < VW; ++j) xh[j] = fmaf(f[j], sc[i][0], mr);
                } else {
                    const int split = (max(sp.lo(i), 0) / CKPT_BLOCK + 1) * CKPT_BLOCK - sp.lo(i);
#pragma unroll
                    for (int j = 0; j < VW; ++j) xh[j] = fmaf(f[j], j < split ? sc[i][0] : sc[i][1], mr);
                }
            } else {
                *reinterpret_cast<uint4*>(sh.w) = *reinterpret_cast<const uint4*>(slot_h(s, i));
                sh.unpack(xh);
#pragma unroll
                for (int j = 0; j < VW; ++j) xh[j] = (xh[j] - mean) * rs;
            }
        };
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (on && sp.any(i)) {
                float dy[VW], xh[VW], w[VW];
                take(i, dy, xh);
                if constexpr (HOLD) {
#pragma unroll
                    for (int j = 0; j < VW; ++j) w[j] = gm[i][j];
                } else sp.columns(a.gamma, i, w);
                sp.mask(i, xh);  // (a NaN of the row before would get through dy = 0)
#pragma unroll
                for (int j = 0; j < VW; ++j) {
                    pg[i][j] = fmaf(dy[j], xh[j], pg[i][j]);
                    pb[i][j] += dy[j];
                    const float g = dy[j] * w[j];
                    sum[0] += g;
                    sum[1] = fmaf(g, xh[j], sum[1]);
                    if constexpr (HOLD) hg[i][j] = g, hx[i][j] = xh[j];
                }
            }
        }
        team_sum<TEAM>(sum, red[team][round & 1], bar);  // (the other buffer's readers have passed this barrier since)
        const float s0 = sum[0] * inv_d * rs, s1 = sum[1] * inv_d * rs;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (on && sp.any(i)) {
                float f[VW];
                if constexpr (HOLD) {
#pragma unroll
                    for (int j = 0; j < VW; ++j) f[j] = fmaf(-hx[i][j], s1, fmaf(rs, hg[i][j], -s0));
                } else {
                    float dy[VW], xh[VW], w[VW];
                    take(i, dy, xh);
                    sp.columns(a.gamma, i, w);
#pragma unroll
                    for (int j = 0; j < VW; ++j) f[j] = fmaf(-xh[j], s1, fmaf(rs, dy[j] * w[j], -s0));
                }
                if (a.dh) {
                    Span<T, VW> sd;
                    float r[VW];
                    *reinterpret_cast<uint4*>(sd.w) = *slot(s, 1, i);
                    sd.unpack(r);
#pragma unroll
                    for (int j = 0; j < VW; ++j) f[j] += r[j];
                }
                sp.store((T*)a.dx + at, i, f);
            }
        }
        fetch(round + S, s);
    }
    copy_wait(0);
    // the teams' sums side by side in the copies' memory, added in order
    __syncthreads();
    float* acc = reinterpret_cast<float*>(smem);
    if (row0 < a.rows) {
        float *g = acc + 2 * team * a.d, *b = g + a.d;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if constexpr (AL) {
                if (sp.any(i)) {
#pragma unroll
                    for (int j = 0; j < VW; j += 4) {
                        *reinterpret_cast<float4*>(g + sp.lo(i) + j) = make_float4(pg[i][j], pg[i][j + 1], pg[i][j + 2], pg[i][j + 3]);
                        *reinterpret_cast<float4*>(b + sp.lo(i) + j) = make_float4(pb[i][j], pb[i][j + 1], pb[i][j + 2], pb[i][j + 3]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < VW; ++j) {
                    const int c = sp.lo(i) + j;
                    if (c >= 0 && c < a.d) {
                        g[c] = pg[i][j];
                        b[c] = pb[i][j];
                    }
                }
            }
        }
    }
    __syncthreads();
    const int teams = (int)min64(TEAMS, (a.rows - blockIdx.x + gridDim.x - 1) / gridDim.x);  // those with rows
    for (int c = threadIdx.x; c < a.d; c += THREADS) {
        float g = 0.f, b = 0.f;
        for (int t = 0; t < teams; ++t) {
            g += acc[2 * t * a.d + c];
            b += acc[(2 * t + 1) * a.d + c];
        }
        a.part_g[(int64_t)blockIdx.x * a.d + c] = g;
        if (a.part_b) a.part_b[(int64_t)blockIdx.x * a.d + c] = b;
    }
}

// dgamma and dbeta from the CTAs' partials, in order: 32 columns per CTA, 16 slices of the
// partials, the slices added in order. blockIdx.y: gamma, beta.
constexpr int NR_SLICES = 16;
__global__ void __launch_bounds__(32 * NR_SLICES) norm_reduce_kernel(const float* part_g, const float* part_b, int ctas, int d,
                                                                     float* dgamma, float* dbeta) {
    pdl_begin();
    __shared__ float acc[NR_SLICES][32];
    const float* part = blockIdx.y ? part_b : part_g;
    float* out = blockIdx.y ? dbeta : dgamma;
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
    float s = 0.f;
    if (col < d)
#pragma unroll 8
        for (int c = slice; c < ctas; c += NR_SLICES) s += part[(int64_t)c * d + col];
    acc[slice][threadIdx.x & 31] = s;
    __syncthreads();
    if (slice == 0 && col < d) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NR_SLICES; ++i) s += acc[i][threadIdx.x];
        out[col] = s;
    }
}

// ---------------------------------------------------------------------------- buffers of any alignment
// Base addresses off a 16-byte boundary (or fp32 rows of 16382, 16383 elements): a CTA per row, element by element, the row from memory for each
// pass over it (it is in the L2 after the first). Right for any buffers, at some of the speed.
constexpr int NA_THREADS = 512;
__device__ __forceinline__ float cta_sum(float v, float* red) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < NA_THREADS / 32; ++i) v += red[i];
    return v;
}

template <typename T>
__global__ void __launch_bounds__(NA_THREADS) norm_fwd_any_kernel(const __grid_constant__ NormFwdArgs a) {
    pdl_begin();
    __shared__ float red[NA_THREADS / 32];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = (const T*)a.x + row * a.d;
        const T* r = a.res ? (const T*)a.res + row * a.d : nullptr;
        auto at = [&](int c) { return r ? Elem<T>::load(x + c) + Elem<T>::load(r + c) : Elem<T>::load(x + c); };
        float v = 0.f;
        for (int c = threadIdx.x; c < a.d; c += NA_THREADS) v += at(c);
        const float mean = cta_sum(v, red) / (float)a.d;
        v = 0.f;
        for (int c = threadIdx.x; c < a.d; c += NA_THREADS) {
            const float t = at(c) - mean;
            v = fmaf(t, t, v);
        }
        const float rstd = 1.f / sqrtf(cta_sum(v, red) / (float)a.d + a.eps);
        if (threadIdx.x == 0 && a.mean) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        for (int c = threadIdx.x; c < a.d; c += NA_THREADS) {
            const float t = at(c);
            Elem<T>::store((T*)a.y + row * a.d + c, fmaf((t - mean) * rstd, a.gamma[c], a.beta ? a.beta[c] : 0.f));
            if (r) Elem<T>::store((T*)a.h + row * a.d + c, t);
        }
    }
}

// A CTA's columns' sums are kept in shared memory, a thread's own ones
template <typename T>
__global__ void __launch_bounds__(NA_THREADS) norm_bwd_any_kernel(const __grid_constant__ NormBwdArgs a) {
    pdl_begin();
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float red[NA_THREADS / 32];
    float *pg = reinterpret_cast<float*>(smem), *pb = pg + a.d;
    for (int c = threadIdx.x; c < a.d; c += NA_THREADS) pg[c] = pb[c] = 0.f;
    const int nb = (a.d + CKPT_BLOCK - 1) / CKPT_BLOCK;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rs = a.rstd[row];
        const T* dy = (const T*)a.dy + row * a.d;
        auto state = [&](int c) {
            const float h = a.q ? (float)a.q[row * a.d + c] * a.q_scale[row * nb + c / CKPT_BLOCK] : Elem<T>::load((const T*)a.h + row * a.d + c);
            return (h - mean) * rs;
        };
        float s0 = 0.f, s1 = 0.f;
        for (int c = threadIdx.x; c < a.d; c += NA_THREADS) {
            const float y = Elem<T>::load(dy + c), xh = state(c), g = y * a.gamma[c];
            pg[c] = fmaf(y, xh, pg[c]);
            pb[c] += y;
            s0 += g;
            s1 = fmaf(g, xh, s1);
        }
        s0 = cta_sum(s0, red) / (float)a.d;
        s1 = cta_sum(s1, red) / (float)a.d;
        for (int c = threadIdx.x; c < a.d; c += NA_THREADS) {
            float f = rs * (Elem<T>::load(dy + c) * a.gamma[c] - s0 - state(c) * s1);
            if (a.dh) f += Elem<T>::load((const T*)a.dh + row * a.d + c);
            Elem<T>::store((T*)a.dx + row * a.d + c, f);
        }
    }
    for (int c = threadIdx.x; c < a.d; c += NA_THREADS) {
        a.part_g[(int64_t)blockIdx.x * a.d + c] = pg[c];
        if (a.part_b) a.part_b[(int64_t)blockIdx.x * a.d + c] = pb[c];
    }
}

// ---------------------------------------------------------------------------- launchers
constexpr int NORM_MAX_CTAS = 512;  // of the backward: the partials' rows

size_t norm_workspace_bytes(int64_t rows, int d) {
    return (size_t)std::min<int64_t>(std::max<int64_t>(rows, 1), NORM_MAX_CTAS) * d * 2 * sizeof(float);
}

static bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// CTAs for `rows` rows: `most`, or one per row while there are fewer rows; a number that keeps a team's rows a
// multiple of `period` apart (its teams alone may do that).
static int64_t norm_ctas(int64_t rows, int64_t most, int teams, int period) {
    const int64_t n = std::min(rows, std::max<int64_t>(most, period));
    const int unit = period / std::gcd(period, teams);
    return rows <= n * teams ? n : n / unit * unit;
}

template <typename T, int VPT, int TEAM, bool AL>
static cudaError_t norm_fwd_launch(NormFwdArgs a, cudaStream_t s) {
    constexpr int THREADS = norm_fwd_threads<TEAM>(), TEAMS = THREADS / TEAM, VW = 16 / (int)sizeof(T), RES = norm_fwd_resident(VPT * VW, TEAM, AL);
    const size_t stage = (size_t)THREADS * VPT * 16 * (a.res ? 2 : 1);
    a.stages = (int)std::max<size_t>(1, std::min<size_t>(4, NORM_SMEM / RES / stage));
    const cudaError_t e = allow_dynamic_smem<norm_fwd_kernel<T, VPT, TEAM, AL>>(NORM_SMEM / RES);
    if (e != cudaSuccess) return e;
    const int64_t ctas = norm_ctas(a.rows, RES * (int64_t)sm_count(), TEAMS, VW / std::gcd(a.d, VW));
    (void)launch_pdl(norm_fwd_kernel<T, VPT, TEAM, AL>, dim3((unsigned)ctas), dim3(THREADS), stage * a.stages, s, a);
    return cudaGetLastError();
}

template <typename T, int VPT, int TEAM, bool Q, bool AL>
static cudaError_t norm_bwd_launch(NormBwdArgs a, int* ctas, cudaStream_t s) {
    constexpr int THREADS = norm_bwd_threads<TEAM>(), TEAMS = THREADS / TEAM, VW = 16 / (int)sizeof(T), RES = norm_bwd_resident(VPT * VW, TEAM);
    const size_t stage = (size_t)THREADS * VPT * (16 * (a.dh ? 2 : 1) + (Q ? VW : 16)), sums = (size_t)TEAMS * a.d * 2 * sizeof(float);
    a.stages = (int)std::max<size_t>(1, std::min<size_t>(4, NORM_SMEM / RES / stage));
    const cudaError_t e = allow_dynamic_smem<norm_bwd_kernel<T, VPT, TEAM, Q, AL>>(NORM_SMEM / RES);
    if (e != cudaSuccess) return e;
    *ctas = (int)norm_ctas(a.rows, RES * (int64_t)sm_count(), TEAMS, VW / std::gcd(a.d, VW));
    (void)launch_pdl(norm_bwd_kernel<T, VPT, TEAM, Q, AL>, dim3((unsigned)*ctas), dim3(THREADS), std::max(stage * a.stages, sums), s, a);
    return cudaGetLastError();
}

// Rows of whole spans end at kNormMaxWidth elements, in bf16 before the largest team's (the one below holds that many)
template <typename T, int VPT, int TEAM> constexpr bool whole_rows() { return VPT * TEAM / 2 * (16 / (int)sizeof(T)) < kNormMaxWidth; }

template <typename T, int VPT, int TEAM> static cudaError_t norm_fwd_rows(const NormFwdArgs& a, cudaStream_t s) {
    if constexpr (whole_rows<T, VPT, TEAM>())
        if (a.d % (16 / (int)sizeof(T)) == 0) return norm_fwd_launch<T, VPT, TEAM, true>(a, s);
    return norm_fwd_launch<T, VPT, TEAM, false>(a, s);
}
template <typename T, int VPT, int TEAM, bool Q> static cudaError_t norm_bwd_rows(const NormBwdArgs& a, int* ctas, cudaStream_t s) {
    if constexpr (whole_rows<T, VPT, TEAM>())
        if (a.d % (16 / (int)sizeof(T)) == 0) return norm_bwd_launch<T, VPT, TEAM, Q, true>(a, ctas, s);
    return norm_bwd_launch<T, VPT, TEAM, Q, false>(a, ctas, s);
}

// The team for rows of d elements: two spans a thread, from 8 threads on. (fp32 rows of 16382 and 16383
// elements can have 4097 spans: none.)
#define MOE_NORM_TEAM(LAUNCH)                                            \
    do {                                                                 \
        const int n = a.d % VW ? (a.d + 2 * VW - 2) / VW : a.d / VW; /* spans, at any shift */ \
        if (n <= 8) return LAUNCH(1, 8);                                 \
        if (n <= 16) return LAUNCH(1, 16);                               \
        if (n <= 32) return LAUNCH(1, 32);                               \
        if (n <= 64) return LAUNCH(2, 32);                               \
        if (n <= 128) return LAUNCH(2, 64);                              \
        if (n <= 256) return LAUNCH(2, 128);                             \
        if (n <= 512) return LAUNCH(2, 256);                             \
        if (n <= 1024) return LAUNCH(2, 512);                            \
        if (n <= 2048) return LAUNCH(2, 1024);                           \
        if (n <= 4096) return LAUNCH(4, 1024);                           \
    } while (0)

template <typename T> static cudaError_t norm_fwd_t(const NormFwdArgs& a0, cudaStream_t s) {
    constexpr int VW = 16 / (int)sizeof(T);
    NormFwdArgs a = a0;
    const bool spans = aligned_to(a.x, 16) && aligned_to(a.res, 16) && aligned_to(a.h, 16) && aligned_to(a.y, 16);
    // The checkpoint is a pass of its own where rows are no whole spans or the blocks are not those of the threads: of x
    // before the norm, which may write y over x, or with a residual of h after it
    const bool apart = a.q && (!spans || a.d % VW || !aligned_to(a.q, VW));
    auto pack = [&](const void* h) { return launch_ckpt_pack(h, a.rows, a.d, sizeof(T) == 2, a0.q, a.q_scale, s); };
    if (apart) a.q = nullptr;
    if (apart && !a.res) {
        const cudaError_t e = pack(a.x);
        if (e != cudaSuccess) return e;
    }
    auto run = [&]() -> cudaError_t {
        if (spans) {
#define MOE_NORM(VPT, TEAM) norm_fwd_rows<T, VPT, TEAM>(a, s)
            MOE_NORM_TEAM(MOE_NORM);
#undef MOE_NORM
        }
        (void)launch_pdl(norm_fwd_any_kernel<T>, dim3((unsigned)std::min<int64_t>(a.rows, 4 * (int64_t)sm_count())), dim3(NA_THREADS), 0, s, a);
        return cudaGetLastError();
    };
    const cudaError_t e = run();
    return e == cudaSuccess && apart && a.res ? pack(a.h) : e;
}

cudaError_t launch_norm_fwd(int64_t rows, int d, bool bf16, const void* x, const void* res, const float* gamma, const float* beta,
                            float eps, void* h, void* y, float* mean, float* rstd, int8_t* q, float* q_scale, cudaStream_t s) {
    const NormFwdArgs a{rows, d, x, res, gamma, beta, eps, h, y, mean, rstd, q, q_scale, 0};
    return bf16 ? norm_fwd_t<__nv_bfloat16>(a, s) : norm_fwd_t<float>(a, s);
}

template <typename T> static cudaError_t norm_bwd_t(const NormBwdArgs& a, int* ctas, cudaStream_t s) {
    constexpr int VW = 16 / (int)sizeof(T);
    if (aligned_to(a.dy, 16) && aligned_to(a.h, 16) && aligned_to(a.dh, 16) && aligned_to(a.dx, 16) && aligned_to(a.q, VW)) {
        if (a.q) {
#define MOE_NORM(VPT, TEAM) norm_bwd_rows<T, VPT, TEAM, true>(a, ctas, s)
            MOE_NORM_TEAM(MOE_NORM);
#undef MOE_NORM
        }
#define MOE_NORM(VPT, TEAM) norm_bwd_rows<T, VPT, TEAM, false>(a, ctas, s)
        MOE_NORM_TEAM(MOE_NORM);
#undef MOE_NORM
    }
    *ctas = (int)std::min<int64_t>(a.rows, std::min<int64_t>(NORM_MAX_CTAS, sm_count()));
    const cudaError_t e = allow_dynamic_smem<norm_bwd_any_kernel<T>>((size_t)kNormMaxWidth * 2 * sizeof(float));
    if (e != cudaSuccess) return e;
    (void)launch_pdl(norm_bwd_any_kernel<T>, dim3((unsigned)*ctas), dim3(NA_THREADS), (size_t)a.d * 2 * sizeof(float), s, a);
    return cudaGetLastError();
}

cudaError_t launch_norm_bwd(int64_t rows, int d, bool bf16, const void* dy, const void* h, const int8_t* q, const float* q_scale,
                            const float* mean, const float* rstd, const float* gamma, const void* dh, void* dx, float* dgamma,
                            float* dbeta, void* ws, cudaStream_t s) {
    int ctas = 0;
    float* part = (float*)ws;
    const int64_t most = std::min<int64_t>(rows, NORM_MAX_CTAS);
    if (rows > 0) {
        const NormBwdArgs a{rows, d, dy, h, q, q_scale, mean, rstd, gamma, dh, dx, part, dbeta ? part + most * d : nullptr, 0};
        const cudaError_t e = bf16 ? norm_bwd_t<__nv_bfloat16>(a, &ctas, s) : norm_bwd_t<float>(a, &ctas, s);
        if (e != cudaSuccess) return e;
    }
    (void)launch_pdl(norm_reduce_kernel, dim3((d + 31) / 32, dbeta ? 2 : 1), dim3(32 * NR_SLICES), 0, s, (const float*)part,
                     (const float*)(part + most * d), ctas, d, dgamma, dbeta);
    return cudaGetLastError();
}

}  // namespace moe
