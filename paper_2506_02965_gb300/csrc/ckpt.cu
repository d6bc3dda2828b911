// Activation checkpoints in 8 bits (the blocks of span.cuh): packing, unpacking, and the SwiGLU
// backward that reads [G|U] from one. Streams, all HBM-bound: of the copy rate, 6781 GB/s, 32768 x 28672 bf16 packs in
// 412.5 us (1.02), unpacks in 417 (1.01), and its SwiGLU backward takes 660 (1.06); 17994 x 2816 24.3, 24.4 and 37.9 us
// (0.93 to 0.99). bf16 rows of an odd number of elements move 2 bytes a lane, of an odd number of pairs 4, and a row's last
// block takes a whole group of lanes: packing 10000 x 5001 0.42 (unpacking 0.56), 200000 x 67 0.24 (0.41), 20000 x 2002
// 0.58 (0.67); SwiGLU backward of F = 5001 0.63, 1001 0.61, 67 0.39, 1004 (8 bytes a lane) 0.77.
#include <algorithm>
#include <initializer_list>

#include "moe_common.cuh"
#include "moe_internal.h"
#include "span.cuh"

namespace moe {

constexpr int CK_THREADS = 256;
constexpr int CK_U = 4;  // blocks in flight per group of lanes

// Quotient of v < 2^31 by a fixed d: (v mul) >> (31 + s) with 2^s >= d and mul = ceil(2^(31+s) / d), which is
// exact since mul d exceeds 2^(31+s) by less than 2^s.
struct Divisor {
    uint32_t d, mul, s;
    explicit Divisor(uint32_t d_) : d(d_), mul(0), s(0) {
        while ((1ull << s) < d) ++s;
        if (s) mul = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t v) const { return s ? __umulhi(v, mul) >> (s - 1) : v; }
};

// A group of LANES lanes takes a block of 128 columns of a row: VW = 16 / sizeof(T) consecutive ones a lane (half a warp
// or a warp a block), or in rows that no 16-byte access fits 4, 2 or 1, 32 lanes of them in turn.
template <typename T, int VW> struct CkptMap {
    static constexpr int LANES = VW > 2 ? CKPT_BLOCK / VW : 32;
    static constexpr int GROUPS = CK_THREADS / LANES;
    static constexpr int SPANS = CKPT_BLOCK / (LANES * VW);
    __device__ static __forceinline__ int col(int lane, int i) { return (i * LANES + lane) * VW; }
};

template <int VW> __device__ __forceinline__ void store_q(int8_t* p, const float (&f)[VW], float inv) {
    if constexpr (VW == 8) *reinterpret_cast<uint2*>(p) = make_uint2(quant4(f[0], f[1], f[2], f[3], inv), quant4(f[4], f[5], f[6], f[7], inv));
    else if constexpr (VW == 4) *reinterpret_cast<uint32_t*>(p) = quant4(f[0], f[1], f[2], f[3], inv);
    else if constexpr (VW == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)quant4(f[0], f[1], 0.f, 0.f, inv);
    else *p = quant1(f[0], inv);
}

template <typename T, int VW>
__global__ void __launch_bounds__(CK_THREADS) ckpt_pack_kernel(const T* __restrict__ x, uint32_t blocks, int cols, Divisor nb,
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
        const uint32_t row = nb(b), blk = b - row * nb.d;
        at[u] = (int64_t)row * cols + blk * CKPT_BLOCK;
        left[u] = b < blocks ? cols - (int)blk * CKPT_BLOCK : 0;
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c < left[u]) s[u][i].load(x + at[u] + c);
            else s[u][i].zero();
        }
    }
    float sc, inv[CK_U];
    block_scales<M::LANES, CK_U>(
        [&](int u) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < M::SPANS; ++i) m = max(m, s[u][i].largest_bits());
            return m;
        },
        sc, inv);
    if (lane < CK_U && b0 + lane * M::GROUPS < blocks) scale[b0 + lane * M::GROUPS] = sc;
#pragma unroll
    for (int u = 0; u < CK_U; ++u)
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c < left[u]) {
                float f[VW];
                s[u][i].unpack(f);
                store_q<VW>(q + at[u] + c, f, inv[u]);
            }
        }
}

template <typename T, int VW>
__global__ void __launch_bounds__(CK_THREADS) ckpt_unpack_kernel(const int8_t* __restrict__ q, const float* __restrict__ scale,
                                                                 uint32_t blocks, int cols, Divisor nb, T* __restrict__ x) {
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
        const uint32_t row = nb(b), blk = b - row * nb.d;
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
// The sigmoid is the fast one of both types, off by s (1 - s) (4 + 1.23 |G|) + 3 s units of 2^-24, at most 3.4 (far below what
// 8 bits left of G and U; the layer's own fp32 epilogue has the full-precision one): with full-precision exponentials
// and quotients their instructions, not HBM, are the bound.
// A group of lanes takes 128 columns of G, one block of the checkpoint, and the same of U, which lie in one or two.
template <int VW> constexpr int swiglu_u() { return VW > 1 ? 2 : 1; }  // such runs of columns in flight per group of lanes

template <typename T, int VW>
__global__ void __launch_bounds__(CK_THREADS) ckpt_swiglu_bwd_kernel(const int8_t* __restrict__ q, const float* __restrict__ scale,
                                                                     const T* __restrict__ dact, uint32_t runs, Divisor per_row,
                                                                     int F, int nb, T* __restrict__ act, T* __restrict__ dh) {
    pdl_begin();
    using M = CkptMap<T, VW>;
    constexpr int U = swiglu_u<VW>();
    const int lane = threadIdx.x % M::LANES;
    const uint32_t r0 = blockIdx.x * (M::GROUPS * U) + threadIdx.x / M::LANES;
    Span<T, VW> sd[U][M::SPANS];
    uint32_t wg[U][M::SPANS][(VW + 3) / 4], wu[U][M::SPANS][(VW + 3) / 4];
    float cg[U], cu[U][2];
    int64_t at[U], at2[U];  // the run's first column in rows of F; in rows of 2F
    int left[U], split[U];  // columns to the row's end; to U's second block
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t r = r0 + u * M::GROUPS;
        const uint32_t row = per_row(r);
        const int c0 = (int)(r - row * per_row.d) * CKPT_BLOCK, b = (F + c0) / CKPT_BLOCK;
        at[u] = (int64_t)row * F + c0;
        at2[u] = at[u] + (int64_t)row * F;
        left[u] = r < runs ? F - c0 : 0;
        split[u] = (b + 1) * CKPT_BLOCK - (F + c0);
        if (left[u] > 0) {
            const float* sc = scale + (int64_t)row * nb;
            cg[u] = sc[c0 / CKPT_BLOCK];
            cu[u][0] = sc[b];
            cu[u][1] = split[u] < CKPT_BLOCK && b + 1 < nb ? sc[b + 1] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c < left[u]) {
                load_q<VW>(q + at2[u] + c, wg[u][i]);
                load_q<VW>(q + at2[u] + F + c, wu[u][i]);
                sd[u][i].load(dact + at[u] + c);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < M::SPANS; ++i) {
            const int c = M::col(lane, i);
            if (c >= left[u]) continue;
            float G[VW], Uv[VW], d[VW], a[VW], dg[VW], du[VW];
            unquant<VW>(wg[u][i], cg[u], G);
            unquant<VW>(wu[u][i], c < split[u] ? cu[u][0] : cu[u][1], Uv);  // (a span lies in one block: F % VW == 0)
            sd[u][i].unpack(d);
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                const float s = fast_sigmoid(G[j]);
                const float gs = G[j] * s;
                a[j] = gs * Uv[j];
                du[j] = d[j] * gs;
                dg[j] = d[j] * Uv[j] * (s + gs * (1.f - s));
            }
            Span<T, VW> o;
            o.pack(a);
            o.store(act + at[u] + c);
            o.pack(dg);
            o.store(dh + at2[u] + c);
            o.pack(du);
            o.store(dh + at2[u] + F + c);
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
    const int64_t nb = ((int64_t)cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    constexpr int PER = CkptMap<T, VW>::GROUPS * CK_U;
    return by_rows(rows, nb, [&](int64_t r, int64_t n) {
        (void)launch_pdl(ckpt_pack_kernel<T, VW>, dim3((unsigned)((n * nb + PER - 1) / PER)), dim3(CK_THREADS), 0, s, x + r * cols,
                         (uint32_t)(n * nb), cols, Divisor((uint32_t)nb), q + r * cols, scale + r * nb);
    });
}
template <typename T, int VW>
static cudaError_t unpack_t(const int8_t* q, const float* scale, int64_t rows, int cols, T* x, cudaStream_t s) {
    const int64_t nb = ((int64_t)cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    constexpr int PER = CkptMap<T, VW>::GROUPS * CK_U;
    return by_rows(rows, nb, [&](int64_t r, int64_t n) {
        (void)launch_pdl(ckpt_unpack_kernel<T, VW>, dim3((unsigned)((n * nb + PER - 1) / PER)), dim3(CK_THREADS), 0, s, q + r * cols,
                         scale + r * nb, (uint32_t)(n * nb), cols, Divisor((uint32_t)nb), x + r * cols);
    });
}
template <typename T, int VW>
static cudaError_t swiglu_t(const int8_t* q, const float* scale, const T* dact, int64_t rows, int F, T* act, T* dh, cudaStream_t s) {
    const int64_t per_row = ((int64_t)F + CKPT_BLOCK - 1) / CKPT_BLOCK, nb = (2 * (int64_t)F + CKPT_BLOCK - 1) / CKPT_BLOCK;
    constexpr int PER = CkptMap<T, VW>::GROUPS * swiglu_u<VW>();
    return by_rows(rows, per_row, [&](int64_t r, int64_t n) {
        (void)launch_pdl(ckpt_swiglu_bwd_kernel<T, VW>, dim3((unsigned)((n * per_row + PER - 1) / PER)), dim3(CK_THREADS), 0, s,
                         q + r * 2 * F, scale + r * nb, dact + r * F, (uint32_t)(n * per_row), Divisor((uint32_t)per_row), F, (int)nb,
                         act + r * F, dh + r * 2 * F);
    });
}

// The widest span that all of a row's accesses are aligned to: 16 bytes, four elements, two or one
template <typename T> static int span_of(int cols, std::initializer_list<const void*> elems, const int8_t* q) {
    for (int vw : {16 / (int)sizeof(T), 4, 2}) {
        bool ok = cols % vw == 0 && aligned_to(q, vw);
        for (const void* p : elems) ok = ok && aligned_to(p, vw * sizeof(T));
        if (ok) return vw;
    }
    return 1;
}
#define MOE_BY_SPAN(vw, CALL) (vw > 4 ? CALL(16 / (int)sizeof(T)) : vw == 4 ? CALL(4) : vw == 2 ? CALL(2) : CALL(1))

template <typename T> static cudaError_t pack_any(const void* x, int64_t rows, int cols, int8_t* q, float* scale, cudaStream_t s) {
    const int vw = span_of<T>(cols, {x}, q);
#define MOE_CK(V) pack_t<T, V>((const T*)x, rows, cols, q, scale, s)
    return MOE_BY_SPAN(vw, MOE_CK);
#undef MOE_CK
}
template <typename T> static cudaError_t unpack_any(const int8_t* q, const float* scale, int64_t rows, int cols, void* x, cudaStream_t s) {
    const int vw = span_of<T>(cols, {x}, q);
#define MOE_CK(V) unpack_t<T, V>(q, scale, rows, cols, (T*)x, s)
    return MOE_BY_SPAN(vw, MOE_CK);
#undef MOE_CK
}
template <typename T>
static cudaError_t swiglu_any(const int8_t* q, const float* scale, const void* dact, int64_t rows, int F, void* act, void* dh, cudaStream_t s) {
    const int vw = span_of<T>(F, {dact, act, dh}, q);
#define MOE_CK(V) swiglu_t<T, V>(q, scale, (const T*)dact, rows, F, (T*)act, (T*)dh, s)
    return MOE_BY_SPAN(vw, MOE_CK);
#undef MOE_CK
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
