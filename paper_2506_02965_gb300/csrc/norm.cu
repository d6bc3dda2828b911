// Layer norm in front of a layer: h = x + residual, y = (h - mean) rstd gamma + beta, and its
// backward with the reduction of the weights' gradients.
//
// A team of W warps holds a row in registers, VPT spans of VW elements per thread, so that x is
// read once: the mean, then the variance about it (no difference of large sums), then the row is
// written. Both directions are HBM-bound.
#include <algorithm>

#include "moe_common.cuh"
#include "moe_internal.h"
#include "span.cuh"

namespace moe {

constexpr int NORM_WARP_TEAMS = 8;  // teams per CTA where a team is one warp

// Sum over the team, the same in all its threads. `red` holds W floats that no other reduction
// of the row uses.
template <int W> __device__ __forceinline__ float team_sum(float v, float* red) {
    v = warp_sum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += red[i];
    }
    return v;
}

struct NormFwdArgs {
    int64_t rows;
    int d;
    const void *x, *res;
    const float *gamma, *beta;
    float eps;
    void *h, *y;
    float *mean, *rstd;
    int8_t* q;
    float* q_scale;
};

template <typename T, int VW, int VPT, int W>
__global__ void __launch_bounds__(W == 1 ? 32 * NORM_WARP_TEAMS : 32 * W) norm_fwd_kernel(NormFwdArgs a) {
    pdl_begin();
    __shared__ float red[2][W];
    constexpr int TEAM = 32 * W, TEAMS = W == 1 ? NORM_WARP_TEAMS : 1;
    const int tid = threadIdx.x % TEAM;
    const int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM;
    if (W == 1 && row >= a.rows) return;  // a whole warp
    const int n = a.d / VW;
    const T* x = (const T*)a.x + row * a.d;
    float v[VPT][VW];
    Span<T, VW> sx[VPT], sr[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int c = i * TEAM + tid;
        if (c < n) sx[i].load(x + c * VW);
        else sx[i].zero();
    }
    if (a.res) {
        const T* r = (const T*)a.res + row * a.d;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = i * TEAM + tid;
            if (c < n) sr[i].load(r + c * VW);
            else sr[i].zero();
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        sx[i].unpack(v[i]);
        if (a.res) {
            float f[VW];
            sr[i].unpack(f);
#pragma unroll
            for (int j = 0; j < VW; ++j) v[i][j] += f[j];
            sx[i].pack(v[i]);
            const int c = i * TEAM + tid;
            if (a.h && c < n) sx[i].store((T*)a.h + row * a.d + c * VW);
        }
#pragma unroll
        for (int j = 0; j < VW; ++j) sum += v[i][j];
    }
    // the statistics are those of the fp32 sum, before it is rounded for storing
    const float mean = team_sum<W>(sum, red[0]) / (float)a.d;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        if (i * TEAM + tid < n) {
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                const float t = v[i][j] - mean;
                sq = fmaf(t, t, sq);
            }
        }
    const float rstd = 1.f / sqrtf(team_sum<W>(sq, red[1]) / (float)a.d + a.eps);
    if (tid == 0 && a.mean) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int c = i * TEAM + tid;
        if constexpr (VW >= 4) {
            if (a.q) {  // the stored h, 128 columns in 128 / VW lanes
                constexpr int LANES = CKPT_BLOCK / VW;
                float f[VW], scale, inv;
                sx[i].unpack(f);
                block_scale(lanes_max<LANES>(largest_bits(f)), scale, inv);
                if (c < n) {
                    uint32_t w[VW / 4];
#pragma unroll
                    for (int j = 0; j < VW / 4; ++j) w[j] = quant4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3], inv);
                    int8_t* q = a.q + row * a.d + c * VW;
                    if constexpr (VW == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
                    else *reinterpret_cast<uint32_t*>(q) = w[0];
                    if (c % LANES == 0) a.q_scale[row * ((a.d + CKPT_BLOCK - 1) / CKPT_BLOCK) + c / LANES] = scale;
                }
            }
        }
        if (c < n) {
            Span<float, VW <= 4 ? VW : 4> sg, sb;
            constexpr int P = VW <= 4 ? VW : 4;
            float f[VW], g[P], b[P];
#pragma unroll
            for (int j = 0; j < VW; j += P) {
                sg.load(a.gamma + c * VW + j);
                sg.unpack(g);
                if (a.beta) {
                    sb.load(a.beta + c * VW + j);
                    sb.unpack(b);
                }
#pragma unroll
                for (int l = 0; l < P; ++l) f[j + l] = fmaf((v[i][j + l] - mean) * rstd, g[l], a.beta ? b[l] : 0.f);
            }
            sx[i].pack(f);
            sx[i].store((T*)a.y + row * a.d + c * VW);
        }
    }
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
};

// One CTA per `gridDim.x`-th row (or team of rows): with xh = (h - mean) rstd and g = dy gamma,
//   dx = dh + rstd (g - <g>/d - xh <g, xh>/d),
// and the thread's columns of sum dy xh and sum dy in registers over all rows of the CTA, written
// once as a partial per CTA and added by norm_reduce_kernel in a fixed order. The next row's
// loads are issued before this row's reduction, so that a CTA always has a row on its way.
// Q: the states come from their 8-bit checkpoint.
template <typename T, int VW, int VPT, int W, bool Q>
__global__ void __launch_bounds__(W == 1 ? 32 * NORM_WARP_TEAMS : 32 * W) norm_bwd_kernel(NormBwdArgs a) {
    pdl_begin();
    constexpr int TEAM = 32 * W, TEAMS = W == 1 ? NORM_WARP_TEAMS : 1;
    __shared__ float red[2][2 * W];
    const int tid = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const int n = a.d / VW, nb = (a.d + CKPT_BLOCK - 1) / CKPT_BLOCK;
    const float inv_d = 1.f / (float)a.d;
    const int64_t step = (int64_t)gridDim.x * TEAMS;
    float pg[VPT][VW], pb[VPT][VW];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < VW; ++j) pg[i][j] = pb[i][j] = 0.f;

    Span<T, VW> sy[VPT], sh[VPT];
    uint32_t qw[VPT][(VW + 3) / 4];
    float qs[VPT], mean = 0.f, rstd = 0.f;
    auto fetch = [&](int64_t r) {
        if (r >= a.rows) return;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = i * TEAM + tid;
            if (c < n) {
                sy[i].load((const T*)a.dy + r * a.d + c * VW);
                if constexpr (Q) {
                    load_q<VW>(a.q + r * a.d + c * VW, qw[i]);
                    qs[i] = a.q_scale[r * nb + c * VW / CKPT_BLOCK];
                } else {
                    sh[i].load((const T*)a.h + r * a.d + c * VW);
                }
            } else {
                sy[i].zero();
                sh[i].zero();
                qs[i] = 0.f;
#pragma unroll
                for (int j = 0; j < (VW + 3) / 4; ++j) qw[i][j] = 0;
            }
        }
        mean = a.mean[r];
        rstd = a.rstd[r];
    };
    int64_t row = (int64_t)blockIdx.x * TEAMS + team;
    fetch(row);
    for (int buf = 0; row < a.rows; row += step, buf ^= 1) {
        float g[VPT][VW], xh[VPT][VW];
        Span<T, VW> sd[VPT];
        float s0 = 0.f, s1 = 0.f;
        const float rs = rstd;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = i * TEAM + tid;
            if (a.dh && c < n) sd[i].load((const T*)a.dh + row * a.d + c * VW);
            sy[i].unpack(g[i]);
            if constexpr (Q) unquant<VW>(qw[i], qs[i], xh[i]);
            else sh[i].unpack(xh[i]);
            if (c < n) {
                constexpr int P = VW <= 4 ? VW : 4;
#pragma unroll
                for (int j = 0; j < VW; j += P) {
                    Span<float, P> sg;
                    float w[P];
                    sg.load(a.gamma + c * VW + j);
                    sg.unpack(w);
#pragma unroll
                    for (int l = 0; l < P; ++l) {
                        const float t = (xh[i][j + l] - mean) * rs;
                        xh[i][j + l] = t;
                        pg[i][j + l] = fmaf(g[i][j + l], t, pg[i][j + l]);
                        pb[i][j + l] += g[i][j + l];
                        g[i][j + l] *= w[l];
                        s0 += g[i][j + l];
                        s1 = fmaf(g[i][j + l], t, s1);
                    }
                }
            }
        }
        fetch(row + step);
        s0 = warp_sum(s0);
        s1 = warp_sum(s1);
        if constexpr (W > 1) {
            if ((threadIdx.x & 31) == 0) {
                red[buf][2 * (threadIdx.x >> 5)] = s0;
                red[buf][2 * (threadIdx.x >> 5) + 1] = s1;
            }
            __syncthreads();  // the other buffer's readers are past it before it is written again
            s0 = s1 = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                s0 += red[buf][2 * w];
                s1 += red[buf][2 * w + 1];
            }
        }
        s0 *= inv_d;
        s1 *= inv_d;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = i * TEAM + tid;
            if (c < n) {
                float f[VW], r[VW];
                if (a.dh) sd[i].unpack(r);
#pragma unroll
                for (int j = 0; j < VW; ++j) {
                    f[j] = rs * (g[i][j] - s0 - xh[i][j] * s1);
                    if (a.dh) f[j] += r[j];
                }
                Span<T, VW> o;
                o.pack(f);
                o.store((T*)a.dx + row * a.d + c * VW);
            }
        }
    }
    // this CTA's partials
    if constexpr (TEAMS > 1) {  // its warps' in order, through shared memory
        __shared__ float acc[TEAMS][2][32 * VW];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                acc[team][0][tid * VW + j] = pg[i][j];
                acc[team][1][tid * VW + j] = pb[i][j];
            }
            __syncthreads();
            for (int e = threadIdx.x; e < 2 * 32 * VW; e += 32 * TEAMS) {
                const int which = e / (32 * VW), o = e % (32 * VW), col = i * 32 * VW + o;
                float s = 0.f;
#pragma unroll
                for (int t = 0; t < TEAMS; ++t) s += acc[t][which][o];
                float* part = which ? a.part_b : a.part_g;
                if (part && col < a.d) part[(int64_t)blockIdx.x * a.d + col] = s;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = i * TEAM + tid;
            if (c < n) {
#pragma unroll
                for (int j = 0; j < VW; ++j) {
                    a.part_g[(int64_t)blockIdx.x * a.d + c * VW + j] = pg[i][j];
                    if (a.part_b) a.part_b[(int64_t)blockIdx.x * a.d + c * VW + j] = pb[i][j];
                }
            }
        }
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
#pragma unroll 4
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

// ---------------------------------------------------------------------------- launchers
constexpr int NORM_MAX_CTAS = 608;  // of the backward: the partials' rows

size_t norm_workspace_bytes(int64_t rows, int d) {
    return (size_t)std::min<int64_t>(std::max<int64_t>(rows, 1), NORM_MAX_CTAS) * d * 2 * sizeof(float);
}

static bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

template <typename T, int VW>
static cudaError_t norm_fwd_w(const NormFwdArgs& a, cudaStream_t s) {
    const int n = a.d / VW;
#define MOE_NORM(VPT, W)                                                                                        \
    (void)launch_pdl(norm_fwd_kernel<T, VW, VPT, W>, dim3((unsigned)(W == 1 ? (a.rows + NORM_WARP_TEAMS - 1) / NORM_WARP_TEAMS : a.rows)), \
                     dim3(W == 1 ? 32 * NORM_WARP_TEAMS : 32 * W), 0, s, a)
    if (n <= 32) MOE_NORM(1, 1);
    else if (n <= 64) MOE_NORM(2, 1);
    else if (n <= 128) MOE_NORM(4, 1);
    else if (n <= 256) MOE_NORM(2, 4);
    else if (n <= 512) MOE_NORM(4, 4);
    else if (n <= 1024) MOE_NORM(4, 8);
    else if (n <= 2048) MOE_NORM(4, 16);
    else if (n <= 4096) MOE_NORM(4, 32);
    else if constexpr (VW <= 2) {
        if (n <= 8192) MOE_NORM(8, 32);
        else MOE_NORM(16, 32);
    }
#undef MOE_NORM
    return cudaGetLastError();
}

template <typename T>
static cudaError_t norm_fwd_t(const NormFwdArgs& a, cudaStream_t s) {
    constexpr int VW = 16 / sizeof(T);
    const bool wide = a.d % VW == 0 && aligned_to(a.x, 16) && aligned_to(a.res, 16) && aligned_to(a.h, 16) && aligned_to(a.y, 16) &&
                      aligned_to(a.gamma, 16) && aligned_to(a.beta, 16) && aligned_to(a.q, VW);
    if (wide) return norm_fwd_w<T, VW>(a, s);
    NormFwdArgs b = a;
    b.q = nullptr;
    const cudaError_t e = norm_fwd_w<T, 1>(b, s);
    if (e != cudaSuccess || !a.q) return e;
    return launch_ckpt_pack(a.res ? a.h : a.x, a.rows, a.d, sizeof(T) == 2, a.q, a.q_scale, s);
}

cudaError_t launch_norm_fwd(int64_t rows, int d, bool bf16, const void* x, const void* res, const float* gamma, const float* beta,
                            float eps, void* h, void* y, float* mean, float* rstd, int8_t* q, float* q_scale, cudaStream_t s) {
    const NormFwdArgs a{rows, d, x, res, gamma, beta, eps, h, y, mean, rstd, q, q_scale};
    return bf16 ? norm_fwd_t<__nv_bfloat16>(a, s) : norm_fwd_t<float>(a, s);
}

template <typename T, int VW, bool Q>
static cudaError_t norm_bwd_w(const NormBwdArgs& a, int* ctas, cudaStream_t s) {
    const int n = a.d / VW;
    // four rows at least per team where that leaves every SM its share of CTAs
#define MOE_NORM(VPT, W)                                                                                       \
    do {                                                                                                       \
        const int64_t teams = W == 1 ? NORM_WARP_TEAMS : 1, most = std::min<int64_t>(NORM_MAX_CTAS, (int64_t)sm_count() * (W == 1 ? 2 : W < 16 ? 16 / W : 1)); \
        *ctas = (int)std::min<int64_t>(most, (a.rows + teams - 1) / teams);                                    \
        (void)launch_pdl(norm_bwd_kernel<T, VW, VPT, W, Q>, dim3((unsigned)*ctas), dim3(W == 1 ? 32 * NORM_WARP_TEAMS : 32 * W), 0, s, a); \
    } while (0)
    if (n <= 32) MOE_NORM(1, 1);
    else if (n <= 64) MOE_NORM(2, 1);
    else if (n <= 128) MOE_NORM(1, 4);
    else if (n <= 256) MOE_NORM(2, 4);
    else if (n <= 512) MOE_NORM(2, 8);
    else if (n <= 1024) MOE_NORM(2, 16);
    else if (n <= 2048) MOE_NORM(2, 32);
    else if constexpr (VW <= 4) {
        if (n <= 4096) MOE_NORM(4, 32);
        else if constexpr (VW <= 2) {
            if (n <= 8192) MOE_NORM(8, 32);
            else MOE_NORM(16, 32);
        }
    }
#undef MOE_NORM
    return cudaGetLastError();
}

template <typename T>
static cudaError_t norm_bwd_t(const NormBwdArgs& a, int* ctas, cudaStream_t s) {
    constexpr int VW = 16 / sizeof(T);
    const bool wide = a.d % VW == 0 && aligned_to(a.dy, 16) && aligned_to(a.h, 16) && aligned_to(a.dh, 16) && aligned_to(a.dx, 16) &&
                      aligned_to(a.gamma, 16) && aligned_to(a.q, VW);
    if (a.q) return wide ? norm_bwd_w<T, VW, true>(a, ctas, s) : norm_bwd_w<T, 1, true>(a, ctas, s);
    return wide ? norm_bwd_w<T, VW, false>(a, ctas, s) : norm_bwd_w<T, 1, false>(a, ctas, s);
}

cudaError_t launch_norm_bwd(int64_t rows, int d, bool bf16, const void* dy, const void* h, const int8_t* q, const float* q_scale,
                            const float* mean, const float* rstd, const float* gamma, const void* dh, void* dx, float* dgamma,
                            float* dbeta, void* ws, cudaStream_t s) {
    int ctas = 0;
    float* part = (float*)ws;
    const int64_t most = std::min<int64_t>(rows, NORM_MAX_CTAS);
    if (rows > 0) {
        const NormBwdArgs a{rows, d, dy, h, q, q_scale, mean, rstd, gamma, dh, dx, part, dbeta ? part + most * d : nullptr};
        const cudaError_t e = bf16 ? norm_bwd_t<__nv_bfloat16>(a, &ctas, s) : norm_bwd_t<float>(a, &ctas, s);
        if (e != cudaSuccess) return e;
    }
    (void)launch_pdl(norm_reduce_kernel, dim3((d + 31) / 32, dbeta ? 2 : 1), dim3(32 * NR_SLICES), 0, s, (const float*)part,
                     (const float*)(part + most * d), ctas, d, dgamma, dbeta);
    return cudaGetLastError();
}

}  // namespace moe
