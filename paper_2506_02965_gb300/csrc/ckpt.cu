// Activation checkpoints in 8 bits (the blocks of span.cuh): packing, unpacking, and the SwiGLU
// backward that reads [G|U] from one. Streams, all HBM-bound.
#include <algorithm>

#include "moe_common.cuh"
#include "moe_internal.h"
#include "span.cuh"

namespace moe {

constexpr int CK_THREADS = 256;
constexpr int CK_U = 4;  // blocks in flight per group of lanes

// A group of 128 / VW lanes takes a block of 128 columns of a row, VW consecutive ones a lane; with
// VW = 1 (rows that no 16-byte access fits) a warp takes it, four columns a lane, 32 apart.
template <typename T, int VW> struct CkptMap {
    static constexpr int LANES = VW == 1 ? 32 : CKPT_BLOCK / VW;
    static constexpr int GROUPS = CK_THREADS / LANES;
    static constexpr int SPANS = VW == 1 ? 4 : 1;
    __device__ static __forceinline__ int col(int lane, int i) { return VW == 1 ? i * 32 + lane : lane * VW; }
};

template <typename T, int VW>
__global__ void __launch_bounds__(CK_THREADS) ckpt_pack_kernel(const T* __restrict__ x, uint32_t blocks, int cols, uint32_t nb,
                                                               int8_t* __restrict__ q, float* __restrict__ scale) {
    pdl_begin();
    using M = CkptMap<T, VW>;
    const int lane = threadIdx.x % M::LANES;
    const uint32_t b0 = blockIdx.x * (M::GROUPS * CK_U) + threadIdx.x / M::LANES;
    Span<T, VW> s[CK_U][M::SPANS];
    int64_t at[CK_U];
    int left[CK_U];  // columns from the block's first to the row's end
#pragma unroll
    for (int u = 0; u < CK_U; ++u) {
        const uint32_t b = b0 + u * M::GROUPS;
        const uint32_t row = b / nb, blk = b - row * nb;
        at[u] = (int64_t)row * cols + blk * CKPT_BLOCK;
        left[u] = b < blocks ? cols - (int)blk * CKPT_BLOCK : 0;
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c < left[u]) s[u][i].load(x + at[u] + c);
            else s[u][i].zero();
        }
    }
#pragma unroll
    for (int u = 0; u < CK_U; ++u) {
        float f[M::SPANS][VW], sc, inv;
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            s[u][i].unpack(f[i]);
            m = max(m, largest_bits(f[i]));
        }
        block_scale(lanes_max<M::LANES>(m), sc, inv);
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c < left[u]) {
                int8_t* p = q + at[u] + c;
                if constexpr (VW == 8)
                    *reinterpret_cast<uint2*>(p) = make_uint2(quant4(f[i][0], f[i][1], f[i][2], f[i][3], inv),
                                                              quant4(f[i][4], f[i][5], f[i][6], f[i][7], inv));
                else if constexpr (VW == 4) *reinterpret_cast<uint32_t*>(p) = quant4(f[i][0], f[i][1], f[i][2], f[i][3], inv);
                else *p = quant1(f[i][0], inv);
            }
        }
        if (lane == 0 && left[u] > 0) scale[b0 + u * M::GROUPS] = sc;
    }
}

template <typename T, int VW>
__global__ void __launch_bounds__(CK_THREADS) ckpt_unpack_kernel(const int8_t* __restrict__ q, const float* __restrict__ scale,
                                                                 uint32_t blocks, int cols, uint32_t nb, T* __restrict__ x) {
    pdl_begin();
    using M = CkptMap<T, VW>;
    const int lane = threadIdx.x % M::LANES;
    const uint32_t b0 = blockIdx.x * (M::GROUPS * CK_U) + threadIdx.x / M::LANES;
    uint32_t w[CK_U][M::SPANS][(VW + 3) / 4];
    float sc[CK_U];
    int64_t at[CK_U];
    int left[CK_U];
#pragma unroll
    for (int u = 0; u < CK_U; ++u) {
        const uint32_t b = b0 + u * M::GROUPS;
        const uint32_t row = b / nb, blk = b - row * nb;
        at[u] = (int64_t)row * cols + blk * CKPT_BLOCK;
        left[u] = b < blocks ? cols - (int)blk * CKPT_BLOCK : 0;
        if (left[u] > 0) sc[u] = scale[b];
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c < left[u]) load_q<VW>(q + at[u] + c, w[u][i]);
        }
    }
#pragma unroll
    for (int u = 0; u < CK_U; ++u)
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c < left[u]) {
                float f[VW];
                Span<T, VW> o;
                unquant<VW>(w[u][i], sc[u], f);
                o.pack(f);
                o.store(x + at[u] + c);
            }
        }
}

// SwiGLU backward from the checkpoint of [G|U] (rows of 2F columns in one run of blocks):
//   s = sigmoid(G), act = G s U, dU = dA G s, dG = dA U s (1 + G (1 - s)).
// Two spans a thread. The sigmoid of bf16 results takes the fast exponential and quotient (errors of a few
// 2^-23, results rounded to 2^-8); with the full-precision ones their instructions, not HBM, are the bound.
template <typename T, int VW>
__global__ void __launch_bounds__(CK_THREADS) ckpt_swiglu_bwd_kernel(const int8_t* __restrict__ q, const float* __restrict__ scale,
                                                                     const T* __restrict__ dact, uint32_t spans, uint32_t per_row,
                                                                     int F, int nb, T* __restrict__ act, T* __restrict__ dh) {
    pdl_begin();
    constexpr int U = 2;
    Span<T, VW> sd[U];
    uint32_t wg[U][(VW + 3) / 4], wu[U][(VW + 3) / 4];
    float cg[U], cu[U];
    uint32_t row[U];
    int col[U];
    bool on[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t v = blockIdx.x * (CK_THREADS * U) + u * CK_THREADS + threadIdx.x;
        on[u] = v < spans;
        row[u] = v / per_row;
        col[u] = (int)(v - row[u] * per_row) * VW;
        if (on[u]) {
            const int8_t* p = q + (int64_t)row[u] * 2 * F + col[u];
            load_q<VW>(p, wg[u]);
            load_q<VW>(p + F, wu[u]);
            cg[u] = scale[(int64_t)row[u] * nb + col[u] / CKPT_BLOCK];
            cu[u] = scale[(int64_t)row[u] * nb + (F + col[u]) / CKPT_BLOCK];
            sd[u].load(dact + (int64_t)row[u] * F + col[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!on[u]) continue;
        float G[VW], Uv[VW], d[VW], a[VW], dg[VW], du[VW];
        unquant<VW>(wg[u], cg[u], G);
        unquant<VW>(wu[u], cu[u], Uv);
        sd[u].unpack(d);
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            const float s = sizeof(T) == 2 ? __fdividef(1.f, 1.f + __expf(-G[j])) : sigmoidf_(G[j]);
            const float gs = G[j] * s;
            a[j] = gs * Uv[j];
            du[j] = d[j] * gs;
            dg[j] = d[j] * Uv[j] * (s + gs * (1.f - s));
        }
        Span<T, VW> o;
        o.pack(a);
        o.store(act + (int64_t)row[u] * F + col[u]);
        T* out = dh + (int64_t)row[u] * 2 * F + col[u];
        o.pack(dg);
        o.store(out);
        o.pack(du);
        o.store(out + F);
    }
}

// ---------------------------------------------------------------------------- launchers
static bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// Rows per launch: the kernels count a launch's blocks or spans in 32 bits.
template <typename F> static cudaError_t by_rows(int64_t rows, int64_t units_per_row, F launch) {
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / units_per_row);
    for (int64_t r = 0; r < rows; r += most) {
        launch(r, std::min(most, rows - r));
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T, int VW>
static cudaError_t pack_t(const T* x, int64_t rows, int cols, int8_t* q, float* scale, cudaStream_t s) {
    const int64_t nb = (cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    constexpr int PER = CkptMap<T, VW>::GROUPS * CK_U;
    return by_rows(rows, nb, [&](int64_t r, int64_t n) {
        (void)launch_pdl(ckpt_pack_kernel<T, VW>, dim3((unsigned)((n * nb + PER - 1) / PER)), dim3(CK_THREADS), 0, s, x + r * cols,
                         (uint32_t)(n * nb), cols, (uint32_t)nb, q + r * cols, scale + r * nb);
    });
}
template <typename T, int VW>
static cudaError_t unpack_t(const int8_t* q, const float* scale, int64_t rows, int cols, T* x, cudaStream_t s) {
    const int64_t nb = (cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    constexpr int PER = CkptMap<T, VW>::GROUPS * CK_U;
    return by_rows(rows, nb, [&](int64_t r, int64_t n) {
        (void)launch_pdl(ckpt_unpack_kernel<T, VW>, dim3((unsigned)((n * nb + PER - 1) / PER)), dim3(CK_THREADS), 0, s, q + r * cols,
                         scale + r * nb, (uint32_t)(n * nb), cols, (uint32_t)nb, x + r * cols);
    });
}
template <typename T, int VW>
static cudaError_t swiglu_t(const int8_t* q, const float* scale, const T* dact, int64_t rows, int F, T* act, T* dh, cudaStream_t s) {
    const int64_t per_row = F / VW, nb = (2 * (int64_t)F + CKPT_BLOCK - 1) / CKPT_BLOCK;
    constexpr int PER = 2 * CK_THREADS;
    return by_rows(rows, per_row, [&](int64_t r, int64_t n) {
        (void)launch_pdl(ckpt_swiglu_bwd_kernel<T, VW>, dim3((unsigned)((n * per_row + PER - 1) / PER)), dim3(CK_THREADS), 0, s,
                         q + r * 2 * F, scale + r * nb, dact + r * F, (uint32_t)(n * per_row), (uint32_t)per_row, F, (int)nb,
                         act + r * F, dh + r * 2 * F);
    });
}

template <typename T> static cudaError_t pack_any(const void* x, int64_t rows, int cols, int8_t* q, float* scale, cudaStream_t s) {
    constexpr int VW = 16 / sizeof(T);
    if (cols % VW == 0 && aligned_to(x, 16) && aligned_to(q, VW)) return pack_t<T, VW>((const T*)x, rows, cols, q, scale, s);
    return pack_t<T, 1>((const T*)x, rows, cols, q, scale, s);
}
template <typename T> static cudaError_t unpack_any(const int8_t* q, const float* scale, int64_t rows, int cols, void* x, cudaStream_t s) {
    constexpr int VW = 16 / sizeof(T);
    if (cols % VW == 0 && aligned_to(x, 16) && aligned_to(q, VW)) return unpack_t<T, VW>(q, scale, rows, cols, (T*)x, s);
    return unpack_t<T, 1>(q, scale, rows, cols, (T*)x, s);
}
template <typename T>
static cudaError_t swiglu_any(const int8_t* q, const float* scale, const void* dact, int64_t rows, int F, void* act, void* dh, cudaStream_t s) {
    constexpr int VW = 16 / sizeof(T);
    if (F % VW == 0 && aligned_to(q, VW) && aligned_to(dact, 16) && aligned_to(act, 16) && aligned_to(dh, 16))
        return swiglu_t<T, VW>(q, scale, (const T*)dact, rows, F, (T*)act, (T*)dh, s);
    return swiglu_t<T, 1>(q, scale, (const T*)dact, rows, F, (T*)act, (T*)dh, s);
}

cudaError_t launch_ckpt_pack(const void* x, int64_t rows, int cols, bool bf16, int8_t* q, float* scale, cudaStream_t s) {
    return bf16 ? pack_any<__nv_bfloat16>(x, rows, cols, q, scale, s) : pack_any<float>(x, rows, cols, q, scale, s);
}
cudaError_t launch_ckpt_unpack(const int8_t* q, const float* scale, int64_t rows, int cols, bool bf16, void* x, cudaStream_t s) {
    return bf16 ? unpack_any<__nv_bfloat16>(q, scale, rows, cols, x, s) : unpack_any<float>(q, scale, rows, cols, x, s);
}
cudaError_t launch_ckpt_swiglu_bwd(const int8_t* q, const float* scale, const void* dact, int64_t rows, int F, bool bf16, void* act,
                                   void* dh, cudaStream_t s) {
    return bf16 ? swiglu_any<__nv_bfloat16>(q, scale, dact, rows, F, act, dh, s) : swiglu_any<float>(q, scale, dact, rows, F, act, dh, s);
}

}  // namespace moe
