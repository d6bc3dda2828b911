// Softmax cross entropy over a vocabulary, without keeping the logits, and its gradients.
//   z = h W^T;  lse_t = log sum_v exp z_tv;  l_t = lse_t - z_t,y;  loss = sum_t u_t l_t
// lse is never one number: with r the row's largest logit and s = sum_v exp(z - r), l = (r - z_y) + log s, and
// softmax(z) = exp(z - r) / s. As one fp32 number it would round l and every probability to a step of its own size, 8e-6 at
// 100: all of the loss, and of the gradient at the target, of a token that is as sure as that.
//   dz_t = u_t (softmax(z_t) - onehot(y_t));  dh = dz W;  dW = dz^T h
// Three products of 2 T V d operations bound a training step (the tensor pipe), reading W a forward of few tokens.
//
// bf16. The logits stay in the tensor cores' accumulators: the product's epilogue takes a row's largest logit m and
// sum of exp(z - m) over a share of the vocabulary (a tile's columns, or half of them), and a pass over
// these joins them to r and s. A forward keeps nothing else. For the gradients the epilogue also stores exp(z - m), in
// fp16: at most 1, and rounded to 11 bits where bf16 would keep 8, down to 2^-14; below, steps of 2^-24 are left (8 bits at 2^-17, as
// bf16; none from 2^-25 on): a word that far under a neighbour of its share loses its probability, which is lost
// against the neighbour's 1 in dh, but in the word's own row of dW only against other tokens' parts.
// A pass then makes dz = u (exp(z - m) exp(m - r) / s - onehot) in place, in bf16, the
// one rounding of dz that counts, and two products make dh and dW from it. The softmax is not computed again
// for that (a fourth product), which costs a pass over 2 bytes a logit, and room for them: so tokens are taken in
// pieces, as many at once as cost no more room than the fp32 sums of dW over the pieces would.
// u is divided by its largest magnitude before that rounding and multiplied in afterwards, in fp32: weights of
// tokens are mostly all alike, and dz near a token's target would carry the same rounding of u for all of them.
//
// fp32. The logits of a piece are stored transposed, [V, tokens], by the fp32 products, so that the vocabulary is the
// dimension that both gradients' products can cut: dh as sums over parts of the vocabulary, joined afterwards.
#include "dense_tc.cuh"
#include "span.cuh"

namespace moe {

namespace {

using namespace dense;

constexpr int kMaxSplits = 16;      // of the gradients' contractions (dh's of up to 128 tokens four times as many)
constexpr int kShortRows = 256;     // dw of up to so many tokens: eight epilogue warps
constexpr int kF32Splits = 64;
constexpr int kColChunk = 512;      // fp32: vocabulary rows whose statistics one CTA takes
constexpr float kNegInf = -INFINITY;

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// ---------------------------------------------------------------- epilogues
// The logits' tile. Two reads of the accumulator, the largest first: with 1024 and more terms a logit they and the exponentials
// hide behind the next tile's product (4096 x 1024 against 32768 words 158 us, 1.74 PFLOP/s; 2048 x 4096 294, 1.87).
// Statistics of every row's share of columns, the target's logit, and (STORE) exp(z - m) in fp16.
template <bool STORE> struct VocabEpi : Plain {
    const int32_t* target;
    float2* part;  // [M][shares]: largest logit, sum of exp(z - it)
    float* zy;     // [M]
    int shares;

    template <int NBUF, typename H> __device__ __forceinline__ void run(const H&, const Problem& p, const Tile& ti, Warp& w, const CUtensorMap* out) const {
        const int row0 = ti.m0 + w.q * 32, m = row0 + w.lane, cols = w.c1 - w.c0;
        const int base = ti.n0 + w.c0, end = min(p.N, ti.n0 + p.tn);
        if (base >= end) return;
        const int y = m < p.M ? target[m] : -1;
        float mx = kNegInf;
#pragma unroll 1
        for (int c = 0; c < cols && base + c < end; c += 32) {
            float v[32];
            tmem_ld32(w.tmem + w.c0 + c, v);
            const int left = end - (base + c);
            if (left >= 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i) mx = fmaxf(mx, v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i < left) mx = fmaxf(mx, v[i]);
            }
            const bool mine = y >= base + c && y < base + c + 32 && y < end;
            if (__any_sync(0xffffffffu, mine)) {
                float z = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (y == base + c + i) z = v[i];
                if (mine) zy[m] = z;
            }
        }
        const float ref = mx == kNegInf ? 0.f : mx;
        float sum = 0.f;
#pragma unroll 1
        for (int c = 0; c < cols && base + c < end; c += 32) {
            float v[32];
            tmem_ld32(w.tmem + w.c0 + c, v);
            const int left = end - (base + c);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                v[i] = fast_exp(v[i] - ref);
                if (i >= left) v[i] = 0.f;
                sum += v[i];
            }
            if constexpr (STORE) {
                uint32_t u[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) u[i] = pack_half(v[2 * i], v[2 * i + 1]);
                store_box<NBUF>(w, out, u, base + c, row0, 0);
            }
        }
        if (m < p.M) part[(int64_t)m * shares + (ti.n0 / p.tn) * (p.tn > cols ? p.tn / cols : 1) + w.c0 / cols] = make_float2(mx, sum);
    }
};

// A product in bf16, times *alpha; (LAST) with fp32 sums of the pieces before added to it.
template <bool LAST> struct OutEpi : Plain {
    const float* alpha;
    const float* sums;  // [M][N]

    template <int NBUF, typename H> __device__ __forceinline__ void run(const H&, const Problem& p, const Tile& ti, Warp& w, const CUtensorMap* out) const {
        const int row0 = ti.m0 + w.q * 32, m = row0 + w.lane;
        const float a = *alpha;
#pragma unroll 1
        for (int c = w.c0; c < w.c1 && ti.n0 + c < p.N; c += 32) {
            float v[32];
            tmem_ld32(w.tmem + c, v);
            if constexpr (LAST) {
                if (m < p.M) {
                    const float* at = sums + (int64_t)m * p.N + ti.n0 + c;
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 s = *reinterpret_cast<const float4*>(at + i);
                        v[i] += s.x; v[i + 1] += s.y; v[i + 2] += s.z; v[i + 3] += s.w;
                    }
                }
            }
            uint32_t u[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = pack_bf16(a * v[2 * i], a * v[2 * i + 1]);
            store_box<NBUF>(w, out, u, ti.n0 + c, row0, 0);
        }
    }
};

// ---------------------------------------------------------------- passes
__device__ __forceinline__ bool has_target(int y, int V) { return y >= 0 && y < V; }

// scal[0] = the largest |weight| of a token with a target, or 1 / (tokens with a target); scal[1] = 1 / scal[0]. Weights that
// are all 0, too small for that or not finite are taken as they are.
__device__ __forceinline__ float scale_of(bool weighted, float most, int n) {
    return !weighted ? 1.f / (float)max(n, 1) : most > 1e-30f && most < 1e30f ? most : 1.f;
}
// One CTA of whole warps, up to 32.
__device__ __forceinline__ void weights_scale(const int32_t* target, const float* weight, int64_t T, int V, float* scal) {
    __shared__ float s_max[32];
    __shared__ int s_n[32];
    float most = 0.f;
    int n = 0;
    bool bad = false;
    for (int64_t t = threadIdx.x; t < T; t += blockDim.x) {
        const int y = target[t];
        bad |= y >= V;
        if (!has_target(y, V)) continue;
        ++n;
        if (weight) most = weight[t] == weight[t] ? fmaxf(most, fabsf(weight[t])) : INFINITY;
    }
    if (bad) record_status(MOE_ERR_DEVICE_CHECK);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    most = warp_max(most);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
        s_max[warp] = most;
        s_n[warp] = n;
    }
    __syncthreads();
    if (warp == 0) {
        most = warp_max(lane < warps ? s_max[lane] : 0.f);
        n = __reduce_add_sync(0xffffffffu, lane < warps ? s_n[lane] : 0);
        if (lane == 0) {
            const float a = scale_of(weight, most, n);
            scal[0] = a;
            scal[1] = 1.f / a;
        }
    }
    __syncthreads();
}

// loss = sum of u_t l_t by one CTA of whole warps: a fixed order, in 64 bits.
__device__ __forceinline__ void total_loss(const float* token, const int32_t* target, const float* weight, const float* scal, int64_t T, int V,
                                           float* loss) {
    __shared__ double s_part[32];
    double sum = 0.0;
    const float u = scal[0];
    for (int64_t t = threadIdx.x; t < T; t += blockDim.x)
        if (has_target(target[t], V)) sum += (double)token[t] * (weight ? weight[t] : u);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x < 32) {
        sum = threadIdx.x < (blockDim.x >> 5) ? s_part[threadIdx.x] : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (threadIdx.x == 0) *loss = (float)sum;
    }
}
__global__ void __launch_bounds__(1024) vocab_total_kernel(const float* __restrict__ token, const int32_t* __restrict__ target,
                                                           const float* __restrict__ weight, const float* __restrict__ scal, int64_t T,
                                                           int V, float* __restrict__ loss) {
    pdl_begin();
    total_loss(token, target, weight, scal, T, V, loss);
}

struct JoinArgs {
    const float2* part;
    int shares, V, d;
    int64_t rows;
    const int32_t* target;   // of the piece's first token
    const float* zy;         // bf16: the target's logit as the product has it
    const __nv_bfloat16 *h, *w;
    const float* zt;         // fp32: the transposed logits
    float2* stat;            // a token's largest logit r and 1 / s
    float* token;
    // the whole batch
    const int32_t* all_target;
    const float* all_weight;
    int64_t T;
    float* scal;             // null: not in this launch
    float* loss;             // one CTA that holds the whole batch: the loss too
    int32_t* offsets;        // fp32: the vocabulary's parts as row offsets, or null
    int splits, split_rows;
};
// <h, w> of d values in fp32, by a warp
__device__ __forceinline__ float warp_dot(const __nv_bfloat16* h, const __nv_bfloat16* w, int d, int lane) {
    float s = 0.f;
#pragma unroll 4
    for (int i = lane * 8; i < d; i += 256) {
        float a[8], b[8];
        unpack8(ldg_nc(h + i), a);
        unpack8(ldg_nc(w + i), b);
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(a[j], b[j], s);
    }
    return warp_sum(s);
}
// r, s and the token's loss from its shares' statistics: a warp per token, and one more CTA for what the batch needs as a
// whole. In bf16 the target's logit is taken once more as an fp32 dot product: the tensor cores' accumulators truncate,
// which leaves a large logit a few 1e-6 of it short (7 tokens, d = 2048: the losses 1.2e-6 off, and 1e-7 with
// this); its term of s, exp(z_y - r), follows. The probabilities are all of the accumulators' logits, the target's too:
// so they add up to 1, and dz at a sure target is the sum of the others'.
template <bool BF16> __global__ void __launch_bounds__(1024) vocab_join_kernel(const JoinArgs a) {
    pdl_begin();
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (a.scal && !a.loss && blockIdx.x == gridDim.x - 1) {
        weights_scale(a.all_target, a.all_weight, a.T, a.V, a.scal);
        if (a.offsets)
            for (int i = threadIdx.x; i <= a.splits; i += blockDim.x) a.offsets[i] = (int)min64(a.V, (int64_t)i * a.split_rows);
        return;
    }
    const int64_t t = a.loss ? threadIdx.x >> 5 : (int64_t)blockIdx.x * warps + (threadIdx.x >> 5);
    if (t < a.rows) {
        const float2* p = a.part + t * a.shares;
        const int y = a.target[t];
        float m = kNegInf, s = 0.f;
        for (int i0 = lane; i0 < a.shares; i0 += 256) {  // eight shares on their way at once
            float2 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = i0 + 32 * k < a.shares ? p[i0 + 32 * k] : make_float2(kNegInf, 0.f);
            float top = m;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, v[k].x);
            const float ref = top == kNegInf ? 0.f : top;
            s *= expf(m - ref);
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k].y * expf(v[k].x - ref);
            m = top;
        }
        const float top = warp_max(m), ref = top == kNegInf ? 0.f : top;
        s = warp_sum(s * expf(m - ref));
        float l = 0.f;
        if (has_target(y, a.V)) {
            if constexpr (BF16) {
                const float z = a.zy[t];
                float off = z - z == 0.f ? warp_dot(a.h + t * a.d, a.w + (int64_t)y * a.d, a.d, lane) - z : 0.f;
                // (logits above 2^26 are that far off; no infinity from it. The largest logit: of s only what the others add to its
                // 1, so that a small loss keeps its digits)
                off = fminf(fmaxf(off, -64.f), 64.f);
                const bool first = z == ref;
                const float c = expf(first ? -off : off);
                l = (first ? 0.f : (ref - z) - off) + log1pf(first ? (s - 1.f) * c : fmaf(expf(z - ref), c - 1.f, s - 1.f));
            } else {
                l = (ref - a.zt[(int64_t)y * a.rows + t]) + logf(s);
            }
        }
        if (lane == 0) {
            a.stat[t] = make_float2(ref, 1.f / s);
            a.token[t] = l;
        }
    }
    if (!a.loss) return;
    // the whole batch, a lane a token: what weights_scale and total_loss find
    if (a.offsets)
        for (int i = threadIdx.x; i <= a.splits; i += blockDim.x) a.offsets[i] = (int)min64(a.V, (int64_t)i * a.split_rows);
    __syncthreads();
    if (threadIdx.x < 32) {
        const int y = lane < a.rows ? a.target[lane] : -1;
        const bool live = has_target(y, a.V);
        if (y >= a.V) record_status(MOE_ERR_DEVICE_CHECK);
        float u = a.all_weight && live ? a.all_weight[lane] : 0.f;
        const int n = __popc(__ballot_sync(0xffffffffu, live));
        const float most = warp_max(u == u ? fabsf(u) : INFINITY);
        const float scale = scale_of(a.all_weight, most, n);
        if (!a.all_weight) u = scale;
        double sum = live ? (double)a.token[lane] * u : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) {
            a.scal[0] = scale;
            a.scal[1] = 1.f / scale;
            *a.loss = (float)sum;
        }
    }
}

// The hidden states for dW = dz^T h: of tokens without a target zeros, as 0 times what stands there need not be 0. A row's
// CTA of `words` 16-byte words.
__device__ __forceinline__ void live_row(const uint4* h, uint4* to, int64_t t, int words, bool live) {
    for (int i = (int)threadIdx.x; i < words; i += 256) to[t * words + i] = live ? h[t * words + i] : make_uint4(0, 0, 0, 0);
}

struct TotalArgs {  // of the whole batch; loss null: not in this launch
    const float* token;
    const int32_t* target;
    const float* weight;
    int64_t T;
    float* loss;
};
// exp(z - m) in fp16 -> dz / scal[0] in bf16, in place. Rows of ld elements, eight a thread, four times. HBM bounds it: 4096
// tokens, 32768 words: 80 us, 6.5 TB/s.
__global__ void __launch_bounds__(256) vocab_dz_kernel(uint4* __restrict__ e, int64_t ld, const float2* __restrict__ part, int shares,
                                                       int share, const float2* __restrict__ stat, const int32_t* __restrict__ target,
                                                       const float* __restrict__ weight, const float* __restrict__ scal, int V,
                                                       const uint4* __restrict__ h, uint4* __restrict__ h_live, int words,
                                                       const TotalArgs total) {
    pdl_begin();
    constexpr int U = 4;
    const int64_t t = blockIdx.y;
    if (total.loss && blockIdx.x == gridDim.x - 1) {  // one more column of CTAs, of which the first adds up the batch
        if (t == 0) total_loss(total.token, total.target, total.weight, scal, total.T, V, total.loss);
        return;
    }
    const int y = target[t];
    const bool live = has_target(y, V);
    if (blockIdx.x == 0) live_row(h, h_live, t, words, live);
    const float u = !live ? 0.f : weight ? weight[t] * scal[1] : 1.f;
    const float2 st = stat[t];
    uint4* row = e + t * (ld / 8);
    const int first = (int)blockIdx.x * (256 * U) + (int)threadIdx.x;
    uint4 v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int i = first + k * 256;
        v[k] = make_uint4(0, 0, 0, 0);
        if (i * 8 < V) v[k] = row[i];
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int i = first + k * 256;
        if (i * 8 >= V) break;
        // (a token without a target has no gradient, whatever its logits are)
        const float m = live ? part[t * shares + i * 8 / share].x : 0.f;
        const float f = live ? u * (fast_exp(m - st.x) * st.y) : 0.f;
        uint32_t* q = reinterpret_cast<uint32_t*>(&v[k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float2 x = __half22float2(*reinterpret_cast<const __half2*>(&q[j]));
            x.x = live ? x.x * f : 0.f;
            x.y = live ? x.y * f : 0.f;
            if (y == i * 8 + 2 * j) x.x -= u;
            if (y == i * 8 + 2 * j + 1) x.y -= u;
            q[j] = pack_bf16(x.x, x.y);
        }
        row[i] = v[k];
    }
}

// out = alpha * the sum of the splits' fp32 sums, in order. Four elements a thread (1003 x 1152, 7 splits: 8 us).
template <typename T>
__global__ void __launch_bounds__(256) vocab_sum_kernel(const float* __restrict__ sums, int splits, int64_t n, const float* __restrict__ alpha,
                                                        T* __restrict__ out) {
    pdl_begin();
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    const float a = alpha ? *alpha : 1.f;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (n % 4 == 0) {
        for (int s = 0; s < splits; ++s) {
            const float4 x = *reinterpret_cast<const float4*>(sums + s * n + i);
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
        }
    } else {
        for (int s = 0; s < splits; ++s)
            for (int j = 0; j < 4 && i + j < n; ++j) v[j] += sums[s * n + i + j];
    }
    for (int j = 0; j < 4 && i + j < n; ++j) Elem<T>::store(out + i + j, a * v[j]);
}

// ---------------------------------------------------------------- fp32 passes over the transposed logits [V, n]
// Statistics of kColChunk rows of every column: 32 columns by 8 rows of threads.
__global__ void __launch_bounds__(256) vocab_col_kernel(const float* __restrict__ z, int V, int n, float2* __restrict__ part, int shares) {
    pdl_begin();
    __shared__ float2 s_part[8][33];
    const int share = (int)(blockIdx.x % (unsigned)shares);
    const int c = (int)(blockIdx.x / (unsigned)shares) * 32 + (threadIdx.x & 31), lane = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int v0 = share * kColChunk, v1 = min(V, v0 + kColChunk);
    float m = kNegInf, s = 0.f;
    if (c < n) {
        for (int v = v0 + r; v < v1; v += 8) m = fmaxf(m, z[(int64_t)v * n + c]);
        const float ref = m == kNegInf ? 0.f : m;
        for (int v = v0 + r; v < v1; v += 8) s += expf(z[(int64_t)v * n + c] - ref);
    }
    s_part[r][lane] = make_float2(m, s);
    __syncthreads();
    if (r == 0 && c < n) {
        for (int k = 1; k < 8; ++k) m = fmaxf(m, s_part[k][lane].x);
        const float ref = m == kNegInf ? 0.f : m;
        s = 0.f;
        for (int k = 0; k < 8; ++k) s += s_part[k][lane].y * expf(s_part[k][lane].x == kNegInf ? kNegInf : s_part[k][lane].x - ref);
        part[(int64_t)c * shares + share] = make_float2(m, s);
    }
}
__global__ void __launch_bounds__(256) vocab_dz_f32_kernel(float* __restrict__ z, int V, int n, const float2* __restrict__ stat,
                                                           const int32_t* __restrict__ target, const float* __restrict__ weight,
                                                           const float* __restrict__ scal, const float* __restrict__ h,
                                                           float* __restrict__ h_live, int d, int tokens) {
    pdl_begin();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)n * d; i += (int64_t)gridDim.x * 256)
        h_live[i] = has_target(target[i / d], V) ? h[i] : 0.f;
    // a block of 32 tokens by 8 rows of threads, its vocabulary rows eight at a time
    const int t = (int)(blockIdx.x % tokens) * 32 + (threadIdx.x & 31);
    if (t >= n) return;
    const int y = target[t];
    const bool live = has_target(y, V);
    const float u = !live ? 0.f : weight ? weight[t] : scal[0];
    const float2 st = stat[t];
    const int step = (int)(gridDim.x / tokens) * 64;  // (at most 2^18: see kVocabLossMax)
    for (int v0 = (int)(blockIdx.x / tokens) * 64 + (threadIdx.x >> 5); v0 < V; v0 += step) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = v0 + 8 * k < V ? z[(int64_t)(v0 + 8 * k) * n + t] : 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int v = v0 + 8 * k;
            if (v < V) z[(int64_t)v * n + t] = live ? u * (expf(x[k] - st.x) * st.y - (v == y ? 1.f : 0.f)) : 0.f;
        }
    }
}
__global__ void __launch_bounds__(256) vocab_add_kernel(float* __restrict__ to, const float* __restrict__ from, int64_t n) {
    pdl_begin();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] += from[i];
}

// ---------------------------------------------------------------- plan: what a call's sizes decide
struct Plan {
    int64_t rows;  // tokens at once
    int pieces;
    int64_t ld;    // bf16: row stride of the stored exp(z - m)
    int shares, share;
    Shape logits, dh, dw;
    int ew, dw_ew; // epilogue warps of the logits, of dw
    int tn;        // columns of a logits tile
    int f32_splits, f32_rows;
    // workspace: offsets
    size_t scal, token, stat, zy, part, e, live, sums, dwsum, offsets, total;
};

// Products with 32 rows of A (dense_tc.cuh: AR): by the plan's tokens at once, so that a short last piece is laid out as the others.
bool short_a(const Shape& s, int64_t rows) { return !s.pair && rows <= 32; }

Plan plan(int64_t T, int32_t d, int32_t V, bool bf16, bool grads) {
    Plan p{};
    const int64_t t1 = std::max<int64_t>(T, 1);
    if (bf16) {
        // Pieces: with more than one, dW's sums over them are kept in fp32, 4 V d bytes; as many tokens as the stored
        // exponentials' 2 V bytes make of that, and no fewer than 4096 (below, dW's contraction is short).
        // A small vocabulary's exponentials are taken up to half a GB.
        const int64_t most = grads ? std::max<int64_t>(std::max<int64_t>(4096, 2 * (int64_t)d), ((int64_t)1 << 28) / V) : (int64_t)1 << 16;
        p.pieces = (int)ceil_div(t1, most);
        p.rows = p.pieces == 1 ? t1 : ceil_div(ceil_div(t1, p.pieces), 256) * 256;
        p.pieces = (int)ceil_div(t1, p.rows);
        p.ld = ceil_div(V, 64) * 64;
        p.logits = pick_shape(p.rows, V, d, 1);
        p.dh = pick_shape(p.rows, d, V, p.rows <= 128 ? 4 * kMaxSplits : kMaxSplits);
        p.dw = pick_shape(V, d, p.rows, p.pieces == 1 ? kMaxSplits : 1);
        p.ew = d < 1024 ? 8 : 4;  // a short contraction: the epilogue, not the product, sets a tile's time
        p.tn = p.logits.pair ? 256 : 128;
        if (short_a(p.logits, p.rows)) {
            // few tokens stream W: the width by which the rounds of tiles come out fullest (65536: 112 columns, four rounds of
            // 147 tiles; of 128 columns four of 128). Whole staging boxes where the exponentials are stored.
            p.ew = 4;
            int64_t least = 0;
            for (int t = 128; t >= 64; t -= grads ? 32 : 16) {
                const int64_t cost = ceil_div(ceil_div(V, t), 2 * kPairs) * (t + 8);
                if (least == 0 || cost < least) {
                    least = cost;
                    p.tn = t;
                }
            }
        }
        // a contraction of a few stages: the stores set the time
        p.dw_ew = p.rows <= kShortRows ? 8 : 4;
        p.share = p.tn / (p.ew / 4);
        p.shares = (int)ceil_div(V, p.share);
    } else {
        const int64_t most = std::max<int64_t>(128, ((int64_t)1 << 28) / V / 128 * 128);
        p.rows = std::min(t1, most);
        p.pieces = (int)ceil_div(t1, p.rows);
        p.shares = (int)ceil_div(V, kColChunk);
        const int64_t tiles = ceil_div(p.rows, 128) * ceil_div(d, 128);
        const int64_t want = std::min<int64_t>(std::min<int64_t>(kF32Splits, ceil_div(4 * kPairs, tiles)), ceil_div(V, 128));
        p.f32_rows = (int)(ceil_div(ceil_div(V, want), 32) * 32);
        p.f32_splits = (int)ceil_div(V, p.f32_rows);
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes);
        return here;
    };
    p.scal = take(8);
    p.token = take((size_t)t1 * 4);
    p.stat = take((size_t)p.rows * 8);
    p.zy = take((size_t)p.rows * 4);
    p.part = take((size_t)p.rows * p.shares * 8);
    if (bf16) {
        if (grads) {
            p.e = take((size_t)p.rows * p.ld * 2);
            p.live = take((size_t)p.rows * d * 2);
            p.sums = take(std::max(p.dh.splits > 1 ? (size_t)p.dh.splits * p.rows * d * 4 : 0, p.dw.splits > 1 ? (size_t)p.dw.splits * V * d * 4 : 0));
            p.dwsum = take(p.pieces > 1 ? (size_t)V * d * 4 : 0);
        }
    } else {
        p.e = take((size_t)p.rows * V * 4);
        if (grads) {
            p.offsets = take((size_t)(p.f32_splits + 1) * 4);
            p.live = take((size_t)p.rows * d * 4);
            p.sums = take(p.f32_splits > 1 ? (size_t)p.f32_splits * p.rows * d * 4 : 0);
            p.dwsum = take(p.pieces > 1 ? (size_t)V * d * 4 : 0);
        }
    }
    p.total = at;
    return p;
}

template <bool STORE>
cudaError_t logits(const Plan& pl, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, const Problem& p, const VocabEpi<STORE>& e,
                   cudaStream_t s) {
    if (pl.logits.pair) {
        if (pl.ew == 8) return launch_as<false, false, true, false, 8>(a, b, o, p, e, s);
        return launch_as<false, false, true, false, 4>(a, b, o, p, e, s);
    }
    if (short_a(pl.logits, pl.rows)) {
        Problem q = p;
        q.tn = pl.tn;
        return launch_as<false, false, false, false, 4, 32>(a, b, o, q, e, s);
    }
    if (pl.ew == 8) return launch_as<false, false, false, false, 8>(a, b, o, p, e, s);
    return launch_as<false, false, false, false, 4>(a, b, o, p, e, s);
}
template <bool A_MN, typename Epi>
cudaError_t product(bool pair, bool few_rows, int ew, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, const Problem& p, const Epi& e,
                    cudaStream_t s) {
    if constexpr (A_MN) {
        if (ew == 8) {
            if (pair) return launch_as<A_MN, true, true, false, 8>(a, b, o, p, e, s);
            return launch_as<A_MN, true, false, false, 8>(a, b, o, p, e, s);
        }
    } else {
        if (few_rows) return launch_as<A_MN, true, false, false, 4, 32>(a, b, o, p, e, s);
    }
    if (pair) return launch_as<A_MN, true, true, false, 4>(a, b, o, p, e, s);
    return launch_as<A_MN, true, false, false, 4>(a, b, o, p, e, s);
}

#define MOE_TRY(call)                              \
    do {                                           \
        const cudaError_t e_ = (call);             \
        if (e_ != cudaSuccess) return e_;          \
    } while (0)

cudaError_t sum_splits(const float* sums, int splits, int64_t n, const float* alpha, bool bf16, void* out, cudaStream_t s) {
    const dim3 grid((unsigned)ceil_div(n, 1024));
    if (bf16) (void)launch_pdl(vocab_sum_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, sums, splits, n, alpha, (__nv_bfloat16*)out);
    else (void)launch_pdl(vocab_sum_kernel<float>, grid, dim3(256), 0, s, sums, splits, n, alpha, (float*)out);
    return cudaGetLastError();
}

float* token_loss(const Plan& pl, const VocabArgs& a, char* ws) { return a.token_loss ? a.token_loss : (float*)(ws + pl.token); }

// One CTA for a batch of few tokens, which then has the loss too.
bool few(const VocabArgs& a) { return a.T <= 32; }

cudaError_t join(const Plan& pl, const VocabArgs& a, char* ws, int piece, int64_t t0, int64_t n, const float* zt, cudaStream_t s) {
    JoinArgs j{};
    j.part = (const float2*)(ws + pl.part);
    j.shares = pl.shares;
    j.V = a.V;
    j.d = a.d;
    j.rows = n;
    j.target = a.target + t0;
    j.zy = (const float*)(ws + pl.zy);
    j.zt = zt;
    j.stat = (float2*)(ws + pl.stat);
    j.token = token_loss(pl, a, ws) + t0;
    j.all_target = a.target;
    j.all_weight = a.weight;
    j.T = a.T;
    if (piece == 0) j.scal = (float*)(ws + pl.scal);
    if (few(a)) j.loss = a.loss;
    const int warps = few(a) ? (int)a.T : 8;
    const unsigned ctas = few(a) ? 1 : (unsigned)(ceil_div(n, warps) + (piece == 0));
    if (a.bf16) {
        j.h = (const __nv_bfloat16*)a.h + t0 * a.d;
        j.w = (const __nv_bfloat16*)a.w;
        (void)launch_pdl(vocab_join_kernel<true>, dim3(ctas), dim3(32 * warps), 0, s, j);
    } else {
        if (a.dh && piece == 0) j.offsets = (int32_t*)(ws + pl.offsets);
        j.splits = pl.f32_splits;
        j.split_rows = pl.f32_rows;
        (void)launch_pdl(vocab_join_kernel<false>, dim3(ctas), dim3(32 * warps), 0, s, j);
    }
    return cudaGetLastError();
}

cudaError_t piece_bf16(const Plan& pl, const VocabArgs& a, char* ws, int piece, cudaStream_t s) {
    const int64_t t0 = piece * pl.rows, n = std::min(pl.rows, a.T - t0);
    const int d = a.d, V = a.V;
    const __nv_bfloat16* h = (const __nv_bfloat16*)a.h + t0 * d;
    float* scal = (float*)(ws + pl.scal);
    CUtensorMap mh, mw, ml, me;  // (ml: W for the logits)
    if (!make_map3(&mh, h, d, n, d, 1, 0, false, short_a(pl.logits, pl.rows) ? 32 : 128) || !make_map3(&mw, a.w, d, V, d, 1, 0, false) ||
        !make_map3(&ml, a.w, d, V, d, 1, 0, false, short_a(pl.logits, pl.rows) ? pl.tn : 128))
        return cudaErrorInvalidValue;
    Problem p = problem((int)n, V, d);
    if (a.dh) {
        if (!make_map3(&me, ws + pl.e, V, n, pl.ld, 1, 0, true)) return cudaErrorInvalidValue;
        MOE_TRY(logits(pl, mh, ml, me, p, VocabEpi<true>{{}, a.target + t0, (float2*)(ws + pl.part), (float*)(ws + pl.zy), pl.shares}, s));
    } else {
        MOE_TRY(logits(pl, mh, ml, mh, p, VocabEpi<false>{{}, a.target + t0, (float2*)(ws + pl.part), (float*)(ws + pl.zy), pl.shares}, s));
    }
    MOE_TRY(join(pl, a, ws, piece, t0, n, nullptr, s));
    if (!a.dh) return cudaSuccess;
    const float* weight = a.weight ? a.weight + t0 : nullptr;
    for (int64_t r = 0; r < n; r += 65535) {  // (rows of a grid)
        TotalArgs total{token_loss(pl, a, ws), a.target, a.weight, a.T, nullptr};
        if (!few(a) && piece == pl.pieces - 1 && r == 0) total.loss = a.loss;
        (void)launch_pdl(vocab_dz_kernel, dim3((unsigned)(ceil_div(V, 8 * 256 * 4) + (total.loss != nullptr)), (unsigned)std::min<int64_t>(65535, n - r)), dim3(256), 0, s,
                         (uint4*)(ws + pl.e + r * pl.ld * 2), pl.ld, (const float2*)(ws + pl.part) + r * pl.shares, pl.shares, pl.share,
                         (const float2*)(ws + pl.stat) + r, a.target + t0 + r, weight ? weight + r : nullptr, (const float*)scal, V,
                         (const uint4*)(h + r * d), (uint4*)(ws + pl.live + r * d * 2), d / 8, total);
        MOE_TRY(cudaGetLastError());
    }
    CUtensorMap ma, mb, mo;
    // dh = dz W: the vocabulary inside dz's rows, outside W's
    if (!make_map3(&ma, ws + pl.e, V, n, pl.ld, 1, 0, false, short_a(pl.dh, pl.rows) ? 32 : 128)) return cudaErrorInvalidValue;
    if (!make_map3(&mo, (__nv_bfloat16*)a.dh + t0 * d, d, n, d, 1, 0, true)) return cudaErrorInvalidValue;
    p = problem((int)n, d, V);
    split_k(p, pl.dh.splits);
    float* sums = (float*)(ws + pl.sums);
    if (p.splits > 1) {
        MOE_TRY((product<false>(pl.dh.pair, short_a(pl.dh, pl.rows), 4, ma, mw, mo, p, SumEpi<false>{sums}, s)));
        MOE_TRY(sum_splits(sums, p.splits, n * d, scal, true, (__nv_bfloat16*)a.dh + t0 * d, s));
    } else {
        MOE_TRY((product<false>(pl.dh.pair, short_a(pl.dh, pl.rows), 4, ma, mw, mo, p, OutEpi<false>{{}, scal, nullptr}, s)));
    }
    // dW = dz^T h: the tokens outside both
    if (!make_map3(&ma, ws + pl.e, V, n, pl.ld, 1, 0, false) || !make_map3(&mb, ws + pl.live, d, n, d, 1, 0, false) ||
        !make_map3(&mo, a.dw, d, V, d, 1, 0, true)) return cudaErrorInvalidValue;
    p = problem(V, d, (int)n);
    float* acc = (float*)(ws + pl.dwsum);
    if (pl.pieces == 1 && pl.dw.splits > 1) {
        split_k(p, pl.dw.splits);
        MOE_TRY((product<true>(pl.dw.pair, false, pl.dw_ew, ma, mb, mo, p, SumEpi<false>{sums}, s)));
        return sum_splits(sums, p.splits, (int64_t)V * d, scal, true, a.dw, s);
    }
    if (pl.pieces == 1) return product<true>(pl.dw.pair, false, pl.dw_ew, ma, mb, mo, p, OutEpi<false>{{}, scal, nullptr}, s);
    if (piece == 0) return product<true>(pl.dw.pair, false, pl.dw_ew, ma, mb, mo, p, SumEpi<false>{acc}, s);
    if (piece < pl.pieces - 1) return product<true>(pl.dw.pair, false, pl.dw_ew, ma, mb, mo, p, SumEpi<true>{acc}, s);
    return product<true>(pl.dw.pair, false, pl.dw_ew, ma, mb, mo, p, OutEpi<true>{{}, scal, acc}, s);
}

cudaError_t piece_f32(const Plan& pl, const VocabArgs& a, char* ws, int piece, cudaStream_t s) {
    const int64_t t0 = piece * pl.rows, n = std::min(pl.rows, a.T - t0);
    const int d = a.d, V = a.V;
    const float* h = (const float*)a.h + t0 * d;
    float *zt = (float*)(ws + pl.e), *scal = (float*)(ws + pl.scal);
    GemmMArgs m{};
    m.G = 1;
    m.rows.rows = V;
    m.a = a.w;
    m.b = h;
    m.b_group_elems = n * d;
    m.b_kmajor = true;
    m.N = (int)n;
    m.K = d;
    m.epi = EPI_STORE;
    m.out0 = zt;
    MOE_TRY(launch_gemm_m(m, false, s));
    (void)launch_pdl(vocab_col_kernel, dim3((unsigned)(ceil_div(n, 32) * pl.shares)), dim3(256), 0, s, (const float*)zt, V, (int)n,
                     (float2*)(ws + pl.part), pl.shares);
    MOE_TRY(cudaGetLastError());
    MOE_TRY(join(pl, a, ws, piece, t0, n, zt, s));
    if (!a.dh) return cudaSuccess;
    const int tokens = (int)ceil_div(n, 32);  // (columns of blocks)
    const int64_t dz_ctas = tokens * std::min<int64_t>(ceil_div(V, 64), std::max<int64_t>(1, 16 * 2 * kPairs / tokens));
    (void)launch_pdl(vocab_dz_f32_kernel, dim3((unsigned)dz_ctas), dim3(256), 0, s,
                     zt, V, (int)n, (const float2*)(ws + pl.stat), a.target + t0, a.weight ? a.weight + t0 : nullptr, (const float*)scal, h,
                     (float*)(ws + pl.live), d, tokens);
    MOE_TRY(cudaGetLastError());
    // dh: sums over parts of the vocabulary, each a group of rows of both operands
    float *dh = (float*)a.dh + t0 * d, *sums = (float*)(ws + pl.sums);
    GemmKArgs k{};
    k.G = pl.f32_splits;
    k.rows.offsets = (const int32_t*)(ws + pl.offsets);
    k.rows.rows = V;
    k.a = zt;
    k.b = a.w;
    k.M = (int)n;
    k.N = d;
    k.out = pl.f32_splits > 1 ? sums : dh;
    MOE_TRY(launch_gemm_k(k, false, s));
    if (pl.f32_splits > 1) MOE_TRY(sum_splits(sums, pl.f32_splits, n * d, nullptr, false, dh, s));
    m.a = zt;
    m.b = ws + pl.live;
    m.b_kmajor = false;
    m.N = d;
    m.K = (int)n;
    m.out0 = piece == 0 ? a.dw : (void*)(ws + pl.dwsum);
    MOE_TRY(launch_gemm_m(m, false, s));
    if (piece > 0) {
        (void)launch_pdl(vocab_add_kernel, dim3(16 * 2 * kPairs), dim3(256), 0, s, (float*)a.dw, (const float*)(ws + pl.dwsum), (int64_t)V * d);
        MOE_TRY(cudaGetLastError());
    }
    return cudaSuccess;
}

}  // namespace

namespace dense {

bool make_map3(CUtensorMap* m, const void* base, int64_t inner, int64_t outer, int64_t ld, int G, int64_t group, bool store, int box_rows) {
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode fn = [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            ptr = nullptr;
        return (Encode)ptr;
    }();
    if (!fn) return false;
    if (G == 1) group = outer * ld;
    cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)outer, (cuuint64_t)G};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)group * 2};
    cuuint32_t box[3] = {store ? (cuuint32_t)OUT_BOX : 64u, store ? (cuuint32_t)OUT_BOX : (cuuint32_t)box_rows, 1u};
    cuuint32_t estr[3] = {1u, 1u, 1u};
    // (the type only matters to arithmetic that is not done here: fp16 moves as bf16)
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              store ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace dense

size_t vocab_workspace_bytes(int64_t T, int32_t d, int32_t V, bool bf16, bool grads) { return plan(T, d, V, bf16, grads).total; }

cudaError_t launch_vocab_loss(const VocabArgs& a, void* workspace, cudaStream_t s) {
    if (a.T == 0) {
        MOE_TRY(cudaMemsetAsync(a.loss, 0, 4, s));
        return a.dw ? cudaMemsetAsync(a.dw, 0, (size_t)a.V * a.d * (a.bf16 ? 2 : 4), s) : cudaSuccess;
    }
    const Plan pl = plan(a.T, a.d, a.V, a.bf16, a.dh != nullptr);
    char* ws = (char*)workspace;
    float* scal = (float*)(ws + pl.scal);
    for (int i = 0; i < pl.pieces; ++i) MOE_TRY(a.bf16 ? piece_bf16(pl, a, ws, i, s) : piece_f32(pl, a, ws, i, s));
    if (few(a) || (a.bf16 && a.dh)) return cudaSuccess;  // (the loss came with another pass)
    (void)launch_pdl(vocab_total_kernel, dim3(1), dim3(1024), 0, s, (const float*)token_loss(pl, a, ws), a.target, a.weight, (const float*)scal, a.T, a.V,
                     a.loss);
    return cudaGetLastError();
}

cudaError_t vocab_status(cudaStream_t s, int* code) { return tu_status_read_clear(s, code); }

}  // namespace moe
