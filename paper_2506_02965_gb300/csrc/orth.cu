// Orthogonalised updates: the momentum in front, and five or so Newton-Schulz products.
//   m' = beta m + g;  u = g + beta m' (nesterov) or m' (g without a momentum);  X = u / |u|_F;
//   per step, on the smaller side:  A = X X^T,  X = a X + (b A + c A A) X;  out = scale X
// with a, b, c = 3.4445, -4.7750, 2.0315 (the published quintic, whose steps take every singular value above about 0.01 of
// the norm into [0.7, 1.2]). For n <= m the sides of a matrix, a step is n^2 m + n^3 + 2 n^2 m operations, of the two
// symmetric products only the tiles on and below the diagonal, the others written as their mirror images: the tensor pipe
// bounds it for n above some hundreds, the launches below.
//
// bf16 matrices run in fp16. Every value is bounded (X's singular values never pass 1.21, so |X| < 1.21, |A| < 1.47,
// |b A + c A A| < 2.81), so powers of two that put them below fp16's largest number keep 11 bits where bf16 would keep
// 8: after five steps, which amplify what small singular directions carry by up to a^5 = 485, bf16 products are 1.2e-2
// off (of the norm, 333 x 1000 to 2048 x 2048 matrices of a gradient's few strong directions over noise). Two more
// things bring that from 1.5e-3 (2.2e-3 for sides of some tens; 8.5e-3 where 16 directions outweigh the rest 30 times) to
// 0.6e-3 (1.4e-3; 1e-3), below the 1.7e-3 of the result's own rounding to bf16:
//   the a X term takes X to 14 bits, its residual as an 8-bit float (e5m2, the upper half of an fp16);
//   from the third step on B = b A + c A A is held as B + t I, and a X + B X taken as (a - t) X + (B + t I) X: most singular
//   values are near 1 by then, B near -2.5 I, and what is left of B + t I is rounded less, as is its product with X.
// Where few directions outweigh the rest the other singular values are not near 1 by then, and the shift costs. Off by, without the
// result's rounding, with and without t (512 x 768, eight directions; after five steps, and after eight, 1e-3 of the norm):
//   directions of the noise    0            3            30           100         1000
//   five steps              0.8 / 1.6    0.65 / 1.2   0.7 / 0.4    1.8 / 1.1    3.2 / 1.9
//   eight                   1.6 / 3.2    1.4 / 2.7    1.3 / 1.8    3.1 / 2.2    11.5 / 7.0
// Without the residual (fp16 X, no t) five steps are 8, 23 and 40 off for the last three.
// The other roundings stay fp16's. All sums are fp32.
//
// A matrix with more rows than columns is not transposed: A = X^T X and X = a X + X (b A + c A A), with the operands'
// other major. fp32 matrices take the fp32 products throughout.
#include <cuda_fp8.h>

#include <cmath>

#include "dense_tc.cuh"
#include "span.cuh"

namespace moe {

namespace {

using namespace dense;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 256.f, kScaleA = 4096.f;  // of the fp16 X, and of A and b A + c A A
constexpr float kResidual = 4096.f;                 // of X's residual, which is 2^-12 of X at most
// t of a step, a number of few bits: about the mean of -B's eigenvalues where a few directions do not outweigh the rest
float shift_of(int step) { return step < 2 ? 0.f : step == 2 ? 1.25f : step == 3 ? 2.25f : 2.5f; }

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// The residuals of X are read and written by the epilogue alone, a box of 32 x 32 at a time, a row a lane: so a box is kept
// as two halves of 16 columns with the lanes' 16 bytes side by side, and a warp moves whole lines.
constexpr int LO_BOX = 32 * 32;
__device__ __forceinline__ int64_t lo_at(int64_t box, int row, int col) { return box * LO_BOX + (col & 16) * 32 + (row & 31) * 16 + (col & 15); }
__device__ __forceinline__ int64_t lo_box(int g, int row, int col, int row_boxes, int col_boxes) {
    return ((int64_t)g * row_boxes + row / 32) * col_boxes + col / 32;
}

// ---------------------------------------------------------------- momentum and norm
// Two passes over the gradient and the momentum, as X needs the norm: 16 x 5632 x 1024 bf16 92 us for the first (6.3 TB/s),
// 195 for the second (5.9 TB/s, m' and X written).
// The sum of squares as three fp32 sums, of x 2^-96, x and x 2^88: one of them neither overflows nor loses what matters,
// from the smallest fp32 numbers to the largest. x itself serves norms of 2^-30 to 2^60; below, a value is at most 2^-30
// and 2^-149 at least, so that the third sum's squares are 2^-122 to 2^116; above, those that matter are over 2^40.
constexpr float kBig = 0x1p-96f, kSmall = 0x1p88f;
struct Squares {
    float big = 0.f, mid = 0.f, small = 0.f;
    __device__ __forceinline__ void add(float x) {
        const float b = x * kBig, s = x * kSmall;
        big = fmaf(b, b, big);
        mid = fmaf(x, x, mid);
        small = fmaf(s, s, small);
    }
};

// N consecutive floats, aligned to them or to 16 bytes
template <int N> __device__ __forceinline__ void load_f32(const float* p, float (&v)[N]) {
    constexpr int W = N < 4 ? N : 4;
#pragma unroll
    for (int i = 0; i < N / W; ++i) {
        Span<float, W> s;
        s.load(p + i * W);
        float f[W];
        s.unpack(f);
#pragma unroll
        for (int j = 0; j < W; ++j) v[i * W + j] = f[j];
    }
}
template <int N> __device__ __forceinline__ void store_f32(float* p, const float (&v)[N]) {
    constexpr int W = N < 4 ? N : 4;
#pragma unroll
    for (int i = 0; i < N / W; ++i) {
        float f[W];
#pragma unroll
        for (int j = 0; j < W; ++j) f[j] = v[i * W + j];
        Span<float, W> s;
        s.pack(f);
        s.store(p + i * W);
    }
}

struct UpdateArgs {
    const void* g;
    const float* mom;      // or null
    float* mom_out;
    const int32_t* counts;
    int64_t elems;         // of a matrix
    int cols;
    int64_t ld, group;     // of X: row stride, and matrix stride
    float beta;
    int nesterov;
    float* part;           // [G][parts][3]
    int parts;
    // fp32: the row offsets of X^T X's parts (see steps_f32), or null
    int32_t* offsets;
    int splits, split_rows, G, ld_rows;
};

// u (and m') of N elements from `at` on
template <typename T, int N>
__device__ __forceinline__ void update_of(const UpdateArgs& a, int64_t at, float (&u)[N], float (&m)[N]) {
    if constexpr (sizeof(T) == 4) {
        load_f32<N>((const float*)a.g + at, u);
    } else {
        constexpr int W = N < 8 ? N : 8;
#pragma unroll
        for (int i = 0; i < N / W; ++i) {
            Span<T, W> s;
            float f[W];
            s.load((const T*)a.g + at + i * W);
            s.unpack(f);
#pragma unroll
            for (int j = 0; j < W; ++j) u[i * W + j] = f[j];
        }
    }
    if (a.mom) {
        load_f32<N>(a.mom + at, m);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            m[j] = fmaf(a.beta, m[j], u[j]);
            u[j] = a.nesterov ? fmaf(a.beta, m[j], u[j]) : m[j];
        }
    }
}

template <typename T, int N> __global__ void __launch_bounds__(256) orth_norm_kernel(const UpdateArgs a) {
    pdl_begin();
    const int g = blockIdx.y;
    if (a.counts && a.counts[g] <= 0) return;
    Squares q;
    // whole spans of the matrix, and the few values before and behind them
    const int64_t first = g * a.elems, base = (first + N - 1) / N * N, end = first + a.elems;
    const int64_t spans = end > base ? (end - base) / N : 0, head = min(base, end) - first, tail = end - (min(base, end) + spans * N);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < spans; i += (int64_t)gridDim.x * 256) {
        float u[N], m[N];
        update_of<T, N>(a, base + i * N, u, m);
#pragma unroll
        for (int j = 0; j < N; ++j) q.add(u[j]);
    }
    if (blockIdx.x == 0 && (int64_t)threadIdx.x < head + tail) {
        const int64_t i = threadIdx.x;
        float u[1], m[1];
        update_of<T, 1>(a, i < head ? first + i : end - tail + (i - head), u, m);
        q.add(u[0]);
    }
    float v[3] = {q.big, q.mid, q.small};
    __shared__ float s_part[8][3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        v[k] = warp_sum(v[k]);
        if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5][k] = v[k];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        float s = 0.f;
        for (int w = 0; w < 8; ++w) s += s_part[w][threadIdx.x];
        a.part[((int64_t)g * a.parts + blockIdx.x) * 3 + threadIdx.x] = s;
    }
}

// What takes u to u / |u|, from the parts, by every CTA for itself (in the same order): a power of two, and a factor after it.
__device__ __forceinline__ float2 inverse_norm(const UpdateArgs& a, int g) {
    __shared__ float s_part[8][3];
    __shared__ float2 s_inv;
    float v[3] = {0.f, 0.f, 0.f};
    for (int i = threadIdx.x; i < a.parts; i += 256)
#pragma unroll
        for (int k = 0; k < 3; ++k) v[k] += a.part[((int64_t)g * a.parts + i) * 3 + k];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        v[k] = warp_sum(v[k]);
        if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5][k] = v[k];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w)
            for (int k = 0; k < 3; ++k) v[k] += s_part[w][k];
        const float inf = __int_as_float(0x7f800000);
        s_inv = !(v[1] < 0x1p120f) ? make_float2(kBig, 1.f / sqrtf(v[0])) : v[1] > 0x1p-60f ? make_float2(1.f, 1.f / sqrtf(v[1]))
                : v[2] > 0.f ? make_float2(kSmall, 1.f / sqrtf(v[2])) : make_float2(1.f, 0.f);  // (nothing: zeros)
        // an infinite or undefined norm leaves nothing but NaN
        if (!(v[0] < inf)) s_inv.y = __int_as_float(0x7fc00000);
    }
    __syncthreads();
    return s_inv;
}

// X = u / |u|: in fp16 with its residual, or in fp32 (a matrix with more columns than rows transposed); and m'
template <typename T, int N, bool HALF>
__global__ void __launch_bounds__(256) orth_start_kernel(const UpdateArgs a, void* hi, uint8_t* lo, int row_boxes, int col_boxes) {
    pdl_begin();
    const int g = blockIdx.y;
    if (!HALF && a.offsets && g == 0 && blockIdx.x == 0)
        for (int i = threadIdx.x; i <= a.G * a.splits; i += 256)
            a.offsets[i] = (int32_t)((int64_t)(i / a.splits) * a.ld_rows + min(a.ld_rows, i % a.splits * a.split_rows));
    const bool called = !a.counts || a.counts[g] > 0;
    if (HALF && !called) return;
    // (the fp32 products take all matrices: one that is left out is zeros there)
    const float2 inv = called ? inverse_norm(a, g) : make_float2(0.f, 0.f);
    const int64_t base = g * a.elems;
    const int rows = (int)(a.elems / a.cols);
    // N = 16: a warp takes blocks of 8 rows by 64 columns, so that X's rows and the residuals' boxes both get whole lines;
    // else of 8 rows by 4 spans of N columns (1, of any alignment: of a row by 32)
    constexpr int ACROSS = N == 1 ? 32 : 4, DOWN = 32 / ACROSS;
    const int blocks = (a.cols + ACROSS * N - 1) / (ACROSS * N);
    const int64_t items = (int64_t)((rows + DOWN - 1) / DOWN) * blocks;
    for (int64_t it = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); it < items; it += (int64_t)gridDim.x * 8) {
        const int rb = (int)((uint32_t)it / (uint32_t)blocks);
        const int row = rb * DOWN + (threadIdx.x & 31) / ACROSS;
        const int col = (((int)it - rb * blocks) * ACROSS + (threadIdx.x & (ACROSS - 1))) * N;
        if (row >= rows || col >= a.cols) continue;
        const int64_t from = base + (int64_t)row * a.cols + col;
        float u[N], m[N];
        if (called) {
            update_of<T, N>(a, from, u, m);
            if (a.mom) store_f32<N>(a.mom_out + from, m);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) u[j] = 0.f;
        }
        const int64_t at = g * a.group + row * a.ld + col;
        if constexpr (HALF) {
            alignas(16) __half h[N];
            alignas(16) uint8_t r[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float x = u[j] * inv.x * inv.y * kScaleX;
                h[j] = __float2half_rn(x);
                r[j] = (uint8_t)__nv_cvt_float_to_fp8((x - __half2float(h[j])) * kResidual, __NV_SATFINITE, __NV_E5M2);
            }
            __half* to = (__half*)hi + at;
            uint8_t* to_lo = lo + lo_at(lo_box(g, row, col, row_boxes, col_boxes), row, col);  // (N columns are in one half)
            if constexpr (N == 16) {
                reinterpret_cast<uint4*>(to)[0] = reinterpret_cast<const uint4*>(h)[0];
                reinterpret_cast<uint4*>(to)[1] = reinterpret_cast<const uint4*>(h)[1];
                *reinterpret_cast<uint4*>(to_lo) = *reinterpret_cast<const uint4*>(r);
            } else if constexpr (N == 8) {
                *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(h);
                *reinterpret_cast<uint2*>(to_lo) = *reinterpret_cast<const uint2*>(r);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    to[j] = h[j];
                    to_lo[j] = r[j];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) u[j] = u[j] * inv.x * inv.y;
            if (rows < a.cols) {
#pragma unroll
                for (int j = 0; j < N; ++j) ((float*)hi)[g * a.elems + (int64_t)(col + j) * rows + row] = u[j];
            } else {
                store_f32<N>((float*)hi + at, u);
            }
        }
    }
}

// ---------------------------------------------------------------- epilogues
// v = alpha acc + beta C for 32 columns of this lane's row, C in fp16 (null: none). All of a warp's chunks of C are on
// their way while the tile's product runs, as whole 64-byte pieces of rows, four lanes each; at its turn a chunk goes
// through the staging box that it will leave from, where every lane finds its row. (One chunk ahead of another, 16 bytes
// of its own row a lane: a step of 16 x 5632 x 1024 180 us; all ahead 166; asynchronous copies into the boxes, for which
// four warps have enough of them, 184: the epilogue's own time a tile, not the memory, sets the pace of a short product.)
struct Term {
    const __half* hi;
    int64_t ld, group;
    float beta;
};
template <int CHUNKS> struct Ahead {
    uint4 h[CHUNKS][4];
    __device__ __forceinline__ void load(const Term& c, const Problem& p, const Tile& ti, const Warp& w) {
        const int row = ti.m0 + w.q * 32 + w.lane / 4;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const int col = ti.n0 + w.c0 + 32 * k;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = c.hi && row + 8 * i < p.M && col < p.N;
                h[k][i] = in ? *reinterpret_cast<const uint4*>(c.hi + ti.g * c.group + (int64_t)(row + 8 * i) * c.ld + col + 8 * (w.lane % 4))
                             : make_uint4(0, 0, 0, 0);
            }
        }
    }
    // this lane's row of chunk k, by way of the box that is next to leave
    template <int NBUF> __device__ __forceinline__ void row(Warp& w, int k, uint32_t (&x)[16]) const {
        if (w.lane == 0) bulk_wait_read<NBUF - 1>();
        __syncwarp();
        uint8_t* box = w.box + w.seq % NBUF * OUT_BOX_BYTES;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + w.lane / 4;
            *reinterpret_cast<uint4*>(box + r * 64 + (((w.lane % 4) ^ ((r >> 1) & 3)) << 4)) = h[k][i];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(box + w.lane * 64 + ((i ^ ((w.lane >> 1) & 3)) << 4));
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
        __syncwarp();
    }
};
__device__ __forceinline__ float2 two_halves(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// The mirror image of 32 columns, from n on, of this lane's row m (two columns a word): of columns j, j + 1 the even lanes
// write rows (m, m + 1) of column j, the odd ones those of column j + 1.
__device__ __forceinline__ void store_mirror(const uint32_t (&u)[16], int lane, int m, int n, int M, __half* out, int64_t ld) {
    __half* to = out + (n + (lane & 1)) * ld + (m & ~1);
    const int rows = (m & ~1) < M ? M - n - (lane & 1) : 0;
#pragma unroll
    for (int i = 0; i < 16; ++i, to += 2 * ld) {
        const uint32_t mine = u[i], other = __shfl_xor_sync(0xffffffffu, mine, 1);
        const uint32_t pair = (lane & 1) ? __byte_perm(other, mine, 0x7632) : __byte_perm(mine, other, 0x5410);
        if (2 * i < rows) *reinterpret_cast<uint32_t*>(to) = pair;
    }
}

// A symmetric product in fp16, its lower tiles and their mirror images. 16 of 1024 x 1024: A over 5632 terms 74 us and 9 for
// the sums of its cut tiles (160 tiles are 2.1 rounds of 76 pairs: 95 us as three), its square 27.5; two of 4096 x 4096 over
// 8192 terms 175, 1.67 PFLOP/s of what is computed.
template <bool CUT_> struct SymEpi {
    static constexpr bool CUT = CUT_;
    Term c;
    float alpha;
    __half* out;
    int64_t ld, group;
    float shift;  // added to the diagonal
    float* parts; // sums of a cut tile's parts, by 32 x 32 chunks as they come from TMEM: [part][chunk][4 columns][row]

    template <int CHUNKS> using Held = Ahead<CHUNKS>;
    template <int NBUF, int CHUNKS>
    __device__ __forceinline__ void fetch(Ahead<CHUNKS>& held, const Problem& p, const Tile& ti, Warp& w) const {
        held.load(c, p, ti, w);
    }
    template <int NBUF, int CHUNKS>
    __device__ __forceinline__ void run(const Ahead<CHUNKS>& held, const Problem& p, const Tile& ti, Warp& w, const CUtensorMap* map) const {
        const int row0 = ti.m0 + w.q * 32, m = row0 + w.lane;
        if (CUT && ti.part >= 0) {
            const int across = p.tn / 32;  // (a tile is a square)
            const int64_t rows = (ti.m0 % p.tn) / 32 + w.q;
#pragma unroll 1
            for (int k = w.c0; k < w.c1; k += 32) {
                float v[32];
                tmem_ld32(w.tmem + k, v);
                float4* to = reinterpret_cast<float4*>(parts + ((ti.part * across + rows) * across + k / 32) * 1024) + w.lane;
#pragma unroll
                for (int i = 0; i < 8; ++i) to[32 * i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
            return;
        }
#pragma unroll
        for (int chunk = 0; chunk < CHUNKS; ++chunk) {
            const int k = w.c0 + 32 * chunk;
            if (ti.n0 + k >= p.N) break;
            float v[32];
            tmem_ld32(w.tmem + k, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= alpha;
            if (c.hi) {
                uint32_t x[16];
                held.template row<NBUF>(w, chunk, x);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 y = two_halves(x[i]);
                    v[2 * i] = fmaf(c.beta, y.x, v[2 * i]);
                    v[2 * i + 1] = fmaf(c.beta, y.y, v[2 * i + 1]);
                }
            }
            if (row0 == ti.n0 + k && shift != 0.f) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] += i == w.lane ? shift : 0.f;
            }
            uint32_t u[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = pack_half(v[2 * i], v[2 * i + 1]);
            store_box<NBUF>(w, map, u, ti.n0 + k, row0, ti.g);
            if (!ti.diag) {
                store_mirror(u, w.lane, m, ti.n0 + k, p.M, out + ti.g * group, ld);
            }
        }
    }
};

// X' = alpha acc + beta X in fp16 with its residual; (LAST) in the matrix's own type, times a scale. 16 x 5632 x 1024 140 us (1.35
// PFLOP/s, 4.1 TB/s of DRAM), 2 x 4096 x 8192 312 (1.76 PFLOP/s).
template <bool LAST> struct StepEpi {
    static constexpr bool CUT = false;
    Term c;
    const uint8_t* lo_in;
    float alpha;
    uint8_t* lo_out;       // LAST: unused
    int row_boxes, col_boxes;
    float scale;           // LAST
    __nv_bfloat16* out;    // LAST: rows of p.N, where the map does not serve them
    int by_map;

    template <int CHUNKS> struct Held {
        Ahead<CHUNKS> x;
        uint4 l[CHUNKS][2];
    };
    template <int NBUF, int CHUNKS>
    __device__ __forceinline__ void fetch(Held<CHUNKS>& held, const Problem& p, const Tile& ti, Warp& w) const {
        held.x.load(c, p, ti, w);
        const int row0 = ti.m0 + w.q * 32;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const int col = ti.n0 + w.c0 + 32 * k;
            const bool in = row0 < p.M && col < p.N;
            const uint4* l = reinterpret_cast<const uint4*>(lo_in + (in ? lo_box(ti.g, row0, col, row_boxes, col_boxes) * LO_BOX : 0));
#pragma unroll
            for (int i = 0; i < 2; ++i) held.l[k][i] = in ? l[32 * i + w.lane] : make_uint4(0, 0, 0, 0);
        }
    }
    template <int NBUF, int CHUNKS>
    __device__ __forceinline__ void run(const Held<CHUNKS>& held, const Problem& p, const Tile& ti, Warp& w, const CUtensorMap* map) const {
        const int row0 = ti.m0 + w.q * 32;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const int col = ti.n0 + w.c0 + 32 * k;
            if (col >= p.N) break;
            float v[32];
            tmem_ld32(w.tmem + w.c0 + 32 * k, v);
            uint32_t x[16];
            held.x.template row<NBUF>(w, k, x);
            const uint32_t* lw = reinterpret_cast<const uint32_t*>(held.l[k]);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                // the residual: two bytes, each the upper one of an fp16
                const float2 h = two_halves(x[i]), y = two_halves(__byte_perm(lw[i / 2], 0, i & 1 ? 0x3424 : 0x1404));
                v[2 * i] = fmaf(c.beta, fmaf(y.x, 1.f / kResidual, h.x), v[2 * i] * alpha);
                v[2 * i + 1] = fmaf(c.beta, fmaf(y.y, 1.f / kResidual, h.y), v[2 * i + 1] * alpha);
            }
            uint32_t u[16];
            if constexpr (LAST) {
#pragma unroll
                for (int i = 0; i < 16; ++i) u[i] = pack_bf16(v[2 * i] * scale, v[2 * i + 1] * scale);
                if (by_map) {
                    store_box<NBUF>(w, map, u, col, row0, ti.g);
                } else {
                    // rows that no map serves (their length is no multiple of 16 bytes): through the box, a row of 32
                    // values a time, a lane each
                    if (w.lane == 0) bulk_wait_read<NBUF - 1>();
                    __syncwarp();
                    uint8_t* box = w.box + w.seq % NBUF * OUT_BOX_BYTES;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<uint4*>(box + w.lane * 64 + ((i ^ ((w.lane >> 1) & 3)) << 4)) =
                            make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
                    __syncwarp();
                    __nv_bfloat16* to = out + ((int64_t)ti.g * p.M + row0) * p.N + col + w.lane;
                    const int rows = min(32, p.M - row0);
                    for (int r = 0; r < rows; ++r) {
                        const int j = w.lane / 8;
                        const __nv_bfloat16 x = *reinterpret_cast<const __nv_bfloat16*>(box + r * 64 + ((j ^ ((r >> 1) & 3)) << 4) + (w.lane % 8) * 2);
                        if (col + w.lane < p.N) to[(int64_t)r * p.N] = x;
                    }
                    __syncwarp();
                }
            } else {
                uint32_t r[8];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    u[i] = pack_half(v[2 * i], v[2 * i + 1]);
                    const float2 h = two_halves(u[i]);
                    const uint32_t e = __nv_cvt_float2_to_fp8x2(make_float2((v[2 * i] - h.x) * kResidual, (v[2 * i + 1] - h.y) * kResidual),
                                                                __NV_SATFINITE, __NV_E5M2);
                    r[i / 2] = i & 1 ? r[i / 2] | (e << 16) : e;
                }
                store_box<NBUF>(w, map, u, col, row0, ti.g);
                if (row0 < p.M) {
                    uint4* to = reinterpret_cast<uint4*>(lo_out + lo_box(ti.g, row0, col, row_boxes, col_boxes) * LO_BOX);
                    to[w.lane] = make_uint4(r[0], r[1], r[2], r[3]);
                    to[32 + w.lane] = make_uint4(r[4], r[5], r[6], r[7]);
                }
            }
        }
    }
};

// A's cut tiles from their parts (dense_tc.cuh: Tail), in order, and their mirror images; a warp a chunk of 32 x 32.
__global__ void __launch_bounds__(128) orth_tail_kernel(const float* __restrict__ sums, const Problem p, float alpha, __half* __restrict__ out,
                                                        int64_t ld, int64_t group) {
    pdl_begin();
    __shared__ unsigned char s_group[MAX_GROUPS];
    __shared__ int s_active;
    if (threadIdx.x < 32) {
        const int run = called_groups(p.counts, p.G, s_group);
        if (threadIdx.x == 0) s_active = run;
    }
    __syncthreads();
    const int mt = (p.M + p.tn - 1) / p.tn, across = p.tn / 32;
    const int per = mt * (mt + 1) / 2;
    const Tail tail = tail_of(s_active * per, p.tail, (p.K + KST - 1) / KST);
    const int lane = threadIdx.x & 31, chunks = across * across;
    const int tile = (int)blockIdx.x * 4 / chunks, chunk = (int)blockIdx.x * 4 % chunks + (threadIdx.x >> 5);
    if (tile >= tail.rest) return;
    const int t = tail.whole + tile, gs = t / per;
    const int2 mn = lower_tile(t - gs * per);
    const int row0 = mn.x * p.tn + chunk / across * 32, n = mn.y * p.tn + chunk % across * 32;
    if (row0 >= p.M || n >= p.N) return;
    const float4* from = reinterpret_cast<const float4*>(sums + ((int64_t)tile * tail.parts * chunks + chunk) * 1024) + lane;
    float v[32] = {};
#pragma unroll 2
    for (int k = 0; k < tail.parts; ++k, from += (int64_t)chunks * 256) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 x = from[32 * i];
            v[4 * i] += x.x;
            v[4 * i + 1] += x.y;
            v[4 * i + 2] += x.z;
            v[4 * i + 3] += x.w;
        }
    }
    uint32_t u[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = pack_half(v[2 * i] * alpha, v[2 * i + 1] * alpha);
    const int m = row0 + lane;
    __half* to = out + s_group[gs] * group;
    if (m < p.M) {  // (rows of A hold whole 64s of columns)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(to + m * ld + n + 8 * i) = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
    }
    if (mn.x != mn.y) store_mirror(u, lane, m, n, p.M, to, ld);
}

// A in fp16 from its parts' sums, in order: [splits][G][n][width] -> rows of ld. A block row of 64 columns by 4 rows.
__global__ void __launch_bounds__(256) orth_square_kernel(const float* __restrict__ sums, int splits, int n, int ld, int width, float alpha,
                                                          __half* __restrict__ out, const int32_t* __restrict__ counts) {
    pdl_begin();
    const int g = blockIdx.y;
    if (counts && counts[g] <= 0) return;
    const int64_t part = (int64_t)gridDim.y * n * width;
    for (int row = (int)blockIdx.x * 4 + (threadIdx.x >> 6); row < n; row += (int)gridDim.x * 4) {
        for (int col = (threadIdx.x & 63) * 2; col < n; col += 128) {
            const float* p = sums + ((int64_t)g * n + row) * width + col;
            float x = 0.f, y = 0.f;
#pragma unroll 8
            for (int k = 0; k < splits; ++k) {
                const float2 v = *reinterpret_cast<const float2*>(p + k * part);
                x += v.x;
                y += v.y;
            }
            *reinterpret_cast<uint32_t*>(out + ((int64_t)g * n + row) * ld + col) = pack_half(x * alpha, y * alpha);
        }
    }
}

// ---------------------------------------------------------------- fp32
// B = a I + b A + c A A, over A's square
__global__ void __launch_bounds__(256) orth_poly_kernel(const float* __restrict__ A, float* __restrict__ sq, int64_t n, int64_t total) {
    pdl_begin();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t at = i % (n * n);
        sq[i] = fmaf(kC, sq[i], fmaf(kB, A[i], at / n == at % n ? kA : 0.f));
    }
}
// the parts' sums, in order
__global__ void __launch_bounds__(256) orth_sum_kernel(const float* __restrict__ parts, float* __restrict__ out, int64_t nn, int64_t total,
                                                       int splits) {
    pdl_begin();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t g = i / nn;
        const float* p = parts + (g * splits - g) * nn + i;
        float s = 0.f;
        for (int k = 0; k < splits; ++k) s += p[k * nn];
        out[i] = s;
    }
}
// scale times X; rows > 0: X is transposed, [cols, rows]
__global__ void __launch_bounds__(256) orth_out_kernel(const float* __restrict__ x, float* __restrict__ out, int64_t elems, int rows, int cols,
                                                       float scale, const int32_t* __restrict__ counts) {
    pdl_begin();
    if (counts && counts[blockIdx.y] <= 0) return;
    const int64_t base = blockIdx.y * elems;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < elems; i += (int64_t)gridDim.x * 256) {
        const int64_t from = rows ? (i % cols) * rows + i / cols : i;
        out[base + i] = x[base + from] * scale;
    }
}

struct Plan {
    int n;              // the smaller side
    int64_t ld, ldn;    // row strides of X and of the squares
    int row_boxes, col_boxes;  // of X's residuals
    int parts;          // CTAs per matrix of the first passes
    Shape gram;              // bf16: tiles and parts of A's product
    int tail;                // its last round of tiles in parts (dense_tc.cuh: Tail), or 0
    int splits, split_rows;  // fp32: parts of X^T X's contraction
    size_t part, offsets, sums, x[2], lo[2], a, b, total;
};

// A's product: the lower tiles, whole or those of the last round in parts, which a pass adds up, or (few tiles, a long side)
// all tiles in parts. In units of a pair's stage as pick_shape; the pass is 12 of them.
Shape pick_gram(int64_t G, int64_t n, int64_t m, int* tail) {
    const int stages = (int)ceil_div(m, KST);
    const Shape parts = pick_shape(n, ceil_div(n, 4) * 4, m, 64, G, false);
    Shape best{true, 1};
    double least = 0;
    auto take = [&](const Shape& s, int places, double cost) {
        if (least != 0 && cost >= least) return;
        least = cost;
        best = s;
        *tail = places;
    };
    for (int pair = 1; pair >= 0; --pair) {
        const int places = pair ? kPairs : 2 * kPairs;
        const int64_t mt = ceil_div(n, pair ? 256 : 128), tiles = std::min<int64_t>(G * mt * (mt + 1) / 2, 0x7fffffff);
        const double each = pair ? 1.0 : 0.92;
        take({pair != 0, 1}, 0, (double)ceil_div(tiles, places) * (stages + 2) * each);
        const Tail t = tail_of((int)tiles, places, stages);
        if (t.rest) take({pair != 0, 1}, places, ((double)(t.whole / places) * (stages + 2) + t.each + 2) * each + 12);
    }
    if (parts.splits > 1) {
        const int64_t mt = ceil_div(n, parts.pair ? 256 : 128);
        take(parts, 0, (double)ceil_div(G * mt * mt * parts.splits, parts.pair ? kPairs : 2 * kPairs) *
                           ((double)stages / parts.splits + 2) * (parts.pair ? 1.0 : 0.92) +
                           8 + (double)parts.splits * G * n * n * 8 / (6.5e6 * 0.7));
    }
    return best;
}

Plan plan(int G, int rows, int cols, bool bf16) {
    Plan p{};
    p.n = std::min(rows, cols);
    p.ld = bf16 ? ceil_div(cols, 64) * 64 : cols;
    p.ldn = bf16 ? ceil_div(p.n, 64) * 64 : p.n;
    p.row_boxes = (int)ceil_div(rows, 32);
    p.col_boxes = (int)ceil_div(cols, 32);
    const int64_t want = ceil_div((int64_t)rows * cols, 8 * 256);
    // (some 48 CTAs a SM: rows of odd lengths are read by single values, whose latency many CTAs hide best; 17 x 5518 x 831 1764 us
    // with 8, 1691 with 16, 1657 with 48, 1664 with 96, whole lines alike), but no more than 8 where a matrix's CTAs, each of
    // which adds up all of its matrix's parts, would read more of those than 12/16 of a byte for each value beside the 13 bytes that
    // the value moves: one step of 1 x 4096 x 4096 249 us, 280 with 48; 2 x 4096 x 4096 470, 487; 4 x 2048 x 2048 179, 196;
    // 1 x 8192 x 8192 1526, 1545 (with 3 bytes a value 252, 472, 183, 1524, with 3/16 249, 465, 185, 1524; the many matrices above keep
    // their 48).
    const int64_t few = (int64_t)std::sqrt((double)rows * cols / 16);
    p.parts = (int)std::max<int64_t>(1, std::min({want, ceil_div(96 * kPairs, G), std::max(ceil_div(16 * kPairs, G), few)}));
    p.splits = 1;
    const int m = std::max(rows, cols);
    if (bf16) {
        p.gram = pick_gram(G, p.n, m, &p.tail);
    } else {
        const int64_t tiles = G * ceil_div(p.n, 128) * ceil_div(p.n, 128);
        int64_t sp = std::min<int64_t>(std::min<int64_t>(256 / G, 2 * kPairs / tiles), m / 128);  // one round of tiles

        sp = std::max<int64_t>(sp, 1);
        p.split_rows = (int)(ceil_div(ceil_div(m, sp), 32) * 32);
        p.splits = (int)ceil_div(m, p.split_rows);
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes);
        return here;
    };
    const size_t xs = (size_t)G * rows * p.ld, as = (size_t)G * p.n * p.ldn, es = bf16 ? 2 : 4;
    p.part = take((size_t)G * p.parts * 12);
    p.offsets = take(p.splits > 1 ? (size_t)(G * p.splits + 1) * 4 : 0);
    for (int i = 0; i < 2; ++i) p.x[i] = take(xs * es);
    for (int i = 0; i < 2; ++i) p.lo[i] = bf16 ? take((size_t)G * p.row_boxes * p.col_boxes * LO_BOX) : 0;
    p.a = take(as * es);
    p.b = take(as * es);
    const size_t cut = p.tail ? (size_t)p.tail * (p.gram.pair ? 256 * 256 : 128 * 128) * 4 : 0;  // (a part a place at most)
    p.sums = take(p.splits > 1 ? as * 4 * p.splits : p.gram.splits > 1 ? (size_t)p.gram.splits * G * p.n * p.ldn * 4 : cut);
    p.total = at;
    return p;
}

#define MOE_TRY(call)                              \
    do {                                           \
        const cudaError_t e_ = (call);             \
        if (e_ != cudaSuccess) return e_;          \
    } while (0)

template <typename T, int N>
cudaError_t start(const UpdateArgs& a, int G, const Plan& pl, void* hi, uint8_t* lo, cudaStream_t s) {
    constexpr bool HALF = sizeof(T) == 2;
    // (A launch of both per matrix, whose second pass then reads from the L2, takes longer: 16 x 36 us for matrices of
    // 5632 x 1024, all in one of each 318.)
    const dim3 grid((unsigned)a.parts, (unsigned)G);
    (void)launch_pdl(orth_norm_kernel<T, 8>, grid, dim3(256), 0, s, a);
    (void)launch_pdl(orth_start_kernel<T, N, HALF>, grid, dim3(256), 0, s, a, hi, lo, pl.row_boxes, pl.col_boxes);
    return cudaGetLastError();
}
template <typename T>
cudaError_t start_n(const UpdateArgs& a, int G, const Plan& pl, void* hi, uint8_t* lo, cudaStream_t s) {
    if (sizeof(T) == 2 && a.cols % 16 == 0) return start<T, sizeof(T) == 2 ? 16 : 8>(a, G, pl, hi, lo, s);
    if (a.cols % 8 == 0) return start<T, 8>(a, G, pl, hi, lo, s);
    if (a.cols % 4 == 0) return start<T, 4>(a, G, pl, hi, lo, s);
    if (a.cols % 2 == 0) return start<T, 2>(a, G, pl, hi, lo, s);
    return start<T, 1>(a, G, pl, hi, lo, s);
}

template <bool A_MN, bool B_MN, typename Epi>
cudaError_t product(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, Problem p, const Epi& e, cudaStream_t s) {
    if (pick_shape(p.M, p.N, p.K, 1, p.G, p.tri).pair) return launch_as<A_MN, B_MN, true, true, 8>(a, b, o, p, e, s);
    return launch_as<A_MN, B_MN, false, true, 8>(a, b, o, p, e, s);
}

template <bool TALL, bool CUT>
cudaError_t launch_lower(bool pair, const CUtensorMap& x, const CUtensorMap& o, const Problem& p, const SymEpi<CUT>& e, cudaStream_t s) {
    if (pair) return launch_as<TALL, TALL, true, true, 8>(x, x, o, p, e, s);
    return launch_as<TALL, TALL, false, true, 8>(x, x, o, p, e, s);
}
template <bool TALL>
cudaError_t launch_gram(bool pair, const CUtensorMap& x, const Problem& p, const SumEpi<false>& e, cudaStream_t s) {
    if (pair) return launch_as<TALL, TALL, true, true, 8>(x, x, x, p, e, s);
    return launch_as<TALL, TALL, false, true, 8>(x, x, x, p, e, s);
}

cudaError_t steps_half(const Plan& pl, const OrthArgs& o, char* ws, cudaStream_t s) {
    const int R = o.rows, C = o.cols, G = o.groups, n = pl.n;
    const bool tall = R > C;
    const int64_t xg = R * pl.ld, ag = n * pl.ldn;
    __half *A = (__half*)(ws + pl.a), *B = (__half*)(ws + pl.b);
    CUtensorMap mx[2], sx[2], ma, sa, mb, sb, mo;
    for (int i = 0; i < 2; ++i)
        if (!make_map3(&mx[i], ws + pl.x[i], C, R, pl.ld, G, xg, false) || !make_map3(&sx[i], ws + pl.x[i], C, R, pl.ld, G, xg, true))
            return cudaErrorInvalidValue;
    if (!make_map3(&ma, A, n, n, pl.ldn, G, ag, false) || !make_map3(&sa, A, n, n, pl.ldn, G, ag, true) ||
        !make_map3(&mb, B, n, n, pl.ldn, G, ag, false) || !make_map3(&sb, B, n, n, pl.ldn, G, ag, true))
        return cudaErrorInvalidValue;
    const bool by_map = C % 8 == 0;
    if (by_map ? !make_map3(&mo, o.out, C, R, C, G, (int64_t)R * C, true) : (mo = sx[0], false)) return cudaErrorInvalidValue;
    Problem sq = problem(n, n, tall ? R : C, G), cube = problem(n, n, n, G), step = problem(R, C, n, G);
    sq.tri = cube.tri = 1;
    sq.counts = cube.counts = step.counts = o.counts;
    Problem lower = sq, parts = sq;
    lower.tail = pl.tail;
    lower.tn = pl.gram.pair ? 256 : 128;
    parts.tri = 0;
    parts.N = (n + 3) / 4 * 4;  // (columns past n: products with zeros)
    split_k(parts, pl.gram.splits);
    for (int i = 0; i < o.steps; ++i) {
        const int x = i & 1, y = x ^ 1;
        const Term none{nullptr, 0, 0, 0.f};
        const SymEpi<false> ea{none, kScaleA / (kScaleX * kScaleX), A, pl.ldn, ag, 0.f, nullptr};
        const SymEpi<true> cut{none, kScaleA / (kScaleX * kScaleX), A, pl.ldn, ag, 0.f, (float*)(ws + pl.sums)};
        if (pl.gram.splits > 1) {
            const SumEpi<false> es{(float*)(ws + pl.sums)};
            if (tall) MOE_TRY((launch_gram<true>(pl.gram.pair, mx[x], parts, es, s)));
            else MOE_TRY((launch_gram<false>(pl.gram.pair, mx[x], parts, es, s)));
            (void)launch_pdl(orth_square_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(n, 4), 16 * kPairs), (unsigned)G), dim3(256), 0, s,
                             (const float*)(ws + pl.sums), parts.splits, n, (int)pl.ldn, parts.N, kScaleA / (kScaleX * kScaleX), A, o.counts);
            MOE_TRY(cudaGetLastError());
        } else {
            // (whole tiles: by the kernel of the square, which is at hand in the instruction caches)
            if (pl.tail) MOE_TRY((tall ? launch_lower<true>(pl.gram.pair, mx[x], sa, lower, cut, s) : launch_lower<false>(pl.gram.pair, mx[x], sa, lower, cut, s)));
            else MOE_TRY((tall ? launch_lower<true>(pl.gram.pair, mx[x], sa, lower, ea, s) : launch_lower<false>(pl.gram.pair, mx[x], sa, lower, ea, s)));
            if (pl.tail) {
                const unsigned chunks = lower.tn * lower.tn / 1024;  // of a tile, four a CTA; half of the places' tiles at most
                (void)launch_pdl(orth_tail_kernel, dim3((unsigned)pl.tail / 2 * chunks / 4), dim3(128), 0, s, (const float*)(ws + pl.sums),
                                 lower, kScaleA / (kScaleX * kScaleX), A, pl.ldn, ag);
                MOE_TRY(cudaGetLastError());
            }
        }
        const float t = shift_of(i);
        const SymEpi<false> eb{{A, pl.ldn, ag, kB}, kC / kScaleA, B, pl.ldn, ag, t * kScaleA, nullptr};
        MOE_TRY((product<false, false>(ma, ma, sb, cube, eb, s)));
        const Term cx{(const __half*)(ws + pl.x[x]), pl.ld, xg, kA - t};
        const uint8_t* lo = (const uint8_t*)(ws + pl.lo[x]);
        if (i + 1 < o.steps) {
            const StepEpi<false> e{cx, lo, 1.f / kScaleA, (uint8_t*)(ws + pl.lo[y]), pl.row_boxes, pl.col_boxes, 1.f, nullptr, 1};
            if (tall) MOE_TRY((product<false, false>(mx[x], mb, sx[y], step, e, s)));
            else MOE_TRY((product<false, true>(mb, mx[x], sx[y], step, e, s)));
        } else {
            const StepEpi<true> e{cx, lo, 1.f / kScaleA, nullptr, pl.row_boxes, pl.col_boxes, o.scale / kScaleX, (__nv_bfloat16*)o.out, by_map};
            if (tall) MOE_TRY((product<false, false>(mx[x], mb, mo, step, e, s)));
            else MOE_TRY((product<false, true>(mb, mx[x], mo, step, e, s)));
        }
    }
    return cudaSuccess;
}

// X is [m, n] here, the longer side outside (transposed on the way in and out where the matrix is wide): A = X^T X is a sum
// over rows, which parts of them share where a matrix has few tiles (8 of 1024 x 256: 64 tiles, 38 us a step as one
// sum).
cudaError_t steps_f32(const Plan& pl, const OrthArgs& o, char* ws, cudaStream_t s) {
    const int G = o.groups, n = pl.n, m = std::max(o.rows, o.cols);
    float *A = (float*)(ws + pl.a), *B = (float*)(ws + pl.b), *sums = (float*)(ws + pl.sums);
    const int64_t nn = (int64_t)n * n;
    const dim3 wide((unsigned)std::min<int64_t>(ceil_div(nn * G, 256), 16 * 2 * kPairs));
    auto rows_by = [&](int rows, const float* a, const float* b, float* out) {  // out = a b, b symmetric [n, n]
        GemmMArgs g{};
        g.G = G;
        g.rows.rows = rows;
        g.rows.a_stride = g.rows.out_stride = rows;
        g.a = a;
        g.b = b;
        g.b_group_elems = nn;
        g.b_kmajor = true;
        g.N = n;
        g.K = n;
        g.epi = EPI_STORE;
        g.out0 = out;
        return launch_gemm_m(g, false, s);
    };
    for (int i = 0; i < o.steps; ++i) {
        float *x = (float*)(ws + pl.x[i & 1]), *y = (float*)(ws + pl.x[(i & 1) ^ 1]);
        GemmKArgs k{};
        k.G = G * pl.splits;
        k.a = k.b = x;
        k.M = k.N = n;
        if (pl.splits > 1) {
            k.rows.offsets = (const int32_t*)(ws + pl.offsets);
            k.rows.rows = G * m;
            k.out = sums;
        } else {
            k.rows.rows = m;
            k.rows.a_stride = k.rows.b_stride = m;
            k.out = A;
        }
        MOE_TRY(launch_gemm_k(k, false, s));
        if (pl.splits > 1) {
            (void)launch_pdl(orth_sum_kernel, wide, dim3(256), 0, s, (const float*)sums, A, nn, nn * G, pl.splits);
            MOE_TRY(cudaGetLastError());
        }
        MOE_TRY(rows_by(n, A, A, B));
        (void)launch_pdl(orth_poly_kernel, wide, dim3(256), 0, s, (const float*)A, B, (int64_t)n, nn * G);
        MOE_TRY(cudaGetLastError());
        MOE_TRY(rows_by(m, x, B, y));
    }
    const int64_t elems = (int64_t)o.rows * o.cols;
    (void)launch_pdl(orth_out_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(elems, 1024), 8 * kPairs), (unsigned)G), dim3(256), 0, s,
                     (const float*)(ws + pl.x[o.steps & 1]), (float*)o.out, elems, o.rows < o.cols ? o.rows : 0, o.cols, o.scale, o.counts);
    return cudaGetLastError();
}

}  // namespace

size_t orth_workspace_bytes(int groups, int rows, int cols, bool bf16) { return plan(groups, rows, cols, bf16).total; }

cudaError_t launch_orthogonalise(const OrthArgs& o, void* workspace, cudaStream_t s) {
    if (o.groups == 0) return cudaSuccess;
    const Plan pl = plan(o.groups, o.rows, o.cols, o.bf16);
    char* ws = (char*)workspace;
    UpdateArgs a{};
    a.g = o.g;
    a.mom = o.momentum;
    a.mom_out = o.momentum_out;
    a.counts = o.counts;
    a.elems = (int64_t)o.rows * o.cols;
    a.cols = o.cols;
    a.ld = pl.ld;
    a.group = o.rows * pl.ld;
    a.beta = o.beta;
    a.nesterov = o.nesterov;
    a.part = (float*)(ws + pl.part);
    a.parts = pl.parts;
    a.G = o.groups;
    a.ld_rows = std::max(o.rows, o.cols);
    a.splits = pl.splits;
    a.split_rows = pl.split_rows;
    if (pl.splits > 1) a.offsets = (int32_t*)(ws + pl.offsets);
    if (o.bf16) {
        MOE_TRY(start_n<__nv_bfloat16>(a, o.groups, pl, ws + pl.x[0], (uint8_t*)(ws + pl.lo[0]), s));
        return steps_half(pl, o, ws, s);
    }
    MOE_TRY(start_n<float>(a, o.groups, pl, ws + pl.x[0], nullptr, s));
    return steps_f32(pl, o, ws, s);
}

cudaError_t orth_status(cudaStream_t s, int* code) { return tu_status_read_clear(s, code); }

}  // namespace moe
