// Gating rules beyond softmax and top-k: sigmoid or softmax scores, a balance bias that takes part
// in the choice only, expert groups of which some are kept, k picks, renormalised and scaled
// weights; their backward; the balance bias's update.
//
// A token's scores live in the registers of LPT lanes (8, 16 or 32: several tokens a warp for small
// pools), NV per lane. Each group of experts owns an equal, power-of-two share of the token's
// lanes and its experts lie in them in ascending order, so that a group's key is a reduction over
// aligned lanes and, among equal keys, the lowest (lane, place) is the lowest expert.
// The loads are few (a token's row once); what bounds these kernels is instructions per score and, for
// short batches, the launch.
#include <algorithm>

#include "moe_common.cuh"
#include "moe_internal.h"

namespace moe {

constexpr int GT_THREADS = 256;

template <int LPT> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = LPT / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int LPT> __device__ __forceinline__ float lanes_maxf(float v) {
#pragma unroll
    for (int o = LPT / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int LPT> __device__ __forceinline__ uint32_t lanes_maxu(uint32_t v) {
    if constexpr (LPT == 32) {
        return __reduce_max_sync(0xffffffffu, v);
    } else {
#pragma unroll
        for (int o = LPT / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
        return v;
    }
}

// Floats in the order of unsigned integers; -0 counts as +0. The lowest is -inf, above 0.
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t u = __float_as_uint(__fadd_rn(f, 0.f));
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <int NV, int LPT, bool SIG>
__global__ void __launch_bounds__(GT_THREADS) gate_kernel(GateArgs a, int lpg, int nv, int chunk, bool whole) {
    pdl_begin();
    __shared__ int hist[256];
    constexpr float NINF = -INFINITY;
    constexpr int TPW = 32 / LPT, TPC = GT_THREADS / LPT;  // tokens per warp and per CTA at a time
    const int lane = threadIdx.x & 31, l = lane % LPT, base = lane - l;
    const int E = a.E, k = a.k, gs = E / a.groups;
    const int grp = l / lpg, lg = l % lpg, e0 = grp * gs + lg * nv;
    const int cnt = grp < a.groups ? min(max(gs - lg * nv, 0), nv) : 0;
    const int64_t t0 = (int64_t)blockIdx.x * chunk, t1 = min64(t0 + chunk, a.T);
    const int p0 = party_of(a.po, a.P, t0);
    for (int e = threadIdx.x; e < E; e += GT_THREADS) hist[e] = 0;
    __syncthreads();
    // whole warps stay in the loop together: a token past the end computes nothing that is written
    for (int64_t tw = t0 + (threadIdx.x / 32) * TPW; tw < t1; tw += TPC) {
        const int64_t t = tw + lane / LPT;
        const bool on = t < t1;
        const int party = on ? party_of(a.po, a.P, t) : p0;
        float z[NV], s[NV];
        const float* row = a.logits + t * E + e0;
        if (a.vec) {
#pragma unroll
            for (int i = 0; i < NV; i += 4) {
                float4 v = make_float4(NINF, NINF, NINF, NINF);
                if (on && i < cnt) v = *reinterpret_cast<const float4*>(row + i);
                z[i] = v.x;
                if (i + 1 < NV) z[i + 1] = v.y;
                if (i + 2 < NV) z[i + 2] = v.z;
                if (i + 3 < NV) z[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) z[i] = on && i < cnt ? row[i] : NINF;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) z[i] = z[i] == z[i] ? z[i] : NINF;  // NaN: out of reach
        if constexpr (SIG) {
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i] = 1.f / (1.f + expf(-z[i]));
        } else {
            float m = NINF, sum = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) m = fmaxf(m, z[i]);
            m = lanes_maxf<LPT>(m);
            m = m == NINF ? 0.f : m;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s[i] = expf(z[i] - m);
                sum += s[i];
            }
            sum = lanes_sum<LPT>(sum);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i] *= inv;
        }
        if (a.scores && on) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < cnt) a.scores[t * E + e0 + i] = s[i];
        }
        // keys, and the two best of the lane
        float key[NV], b1 = NINF, b2 = NINF;
        const float* bias = a.bias ? a.bias + (int64_t)party * E + e0 : nullptr;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            key[i] = SIG ? s[i] : z[i];
            if (bias && i < cnt) key[i] = __fadd_rn(key[i], bias[i]);
            if (!(z[i] > NINF) || key[i] != key[i]) key[i] = NINF;
            b2 = fmaxf(b2, fminf(b1, key[i]));
            b1 = fmaxf(b1, key[i]);
        }
        bool kept = true;
        if (a.top_groups < a.groups) {
            for (int o = lpg >> 1; o > 0; o >>= 1) {
                const float c1 = __shfl_xor_sync(0xffffffffu, b1, o), c2 = __shfl_xor_sync(0xffffffffu, b2, o);
                b2 = fmaxf(fminf(b1, c1), fmaxf(b2, c2));
                b1 = fmaxf(b1, c1);
            }
            const uint32_t mine = ordered(a.group_top == 2 ? b1 + b2 : b1);
            int rank = 0;
            for (int g = 0; g < a.groups; ++g) {
                const uint32_t other = __shfl_sync(0xffffffffu, mine, base + g * lpg);
                rank += other > mine || (other == mine && g < grp);
            }
            kept = rank < a.top_groups;
        }
        uint32_t u[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) u[i] = kept && i < cnt ? ordered(key[i]) : 0u;  // 0: not to be picked
        // pick j stays in lane j
        int pe = 0;
        float ps = 0.f;
        for (int j = 0; j < k; ++j) {
            uint32_t m = u[0];
#pragma unroll
            for (int i = 1; i < NV; ++i) m = max(m, u[i]);
            const uint32_t best = lanes_maxu<LPT>(m);
            const uint32_t who = __ballot_sync(0xffffffffu, m == best) >> base;
            const int owner = base + __ffs(LPT == 32 ? who : who & ((1u << LPT) - 1)) - 1;
            int e = 0;
            float sv = 0.f;
            if (lane == owner) {
                bool found = false;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (!found && u[i] == best) {
                        found = true;
                        e = e0 + i;
                        sv = s[i];
                        u[i] = 0u;
                    }
            }
            e = __shfl_sync(0xffffffffu, e, owner);
            sv = __shfl_sync(0xffffffffu, sv, owner);
            if (l == j) {
                pe = e;
                ps = sv;
            }
        }
        const float total = a.normalize ? lanes_sum<8>(l < k ? ps : 0.f) : 1.f;  // the picks are in a token's first 8 lanes
        if (on && l < k) {
            a.topk_idx[t * k + l] = pe;
            a.topk_w[t * k + l] = total == 0.f ? 0.f : a.scale * ps / total;
            if (party == p0) atomicAdd(&hist[pe], 1);
            else atomicAdd(&a.counts[party * E + pe], 1);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += GT_THREADS) {
        if (whole) a.counts[e] = hist[e];
        else if (hist[e]) atomicAdd(&a.counts[p0 * E + e], hist[e]);
    }
}

// dlogits of a token by LPT lanes, spans of SP = 4 (or single) scores a lane. The picks' gradients go
// to their places through shared memory, on top of aux_coef.
template <int NV, int LPT, int SP, bool SIG>
__global__ void __launch_bounds__(GT_THREADS) gate_bwd_kernel(GateBwdArgs a, __nv_bfloat16* dz16, int EP, int32_t* chunk_off, int CH,
                                                              int nchunk) {
    pdl_begin();
    constexpr float NINF = -INFINITY;
    constexpr int TPC = GT_THREADS / LPT;
    __shared__ float4 s_dp[GT_THREADS * NV / 4];
    if (chunk_off && blockIdx.x == 0 && threadIdx.x == 0) {  // the chunks of the weight gradient's contraction
        int c = 0;
        for (int q = 0; q < a.P; ++q) {
            const int64_t b = a.po ? a.po[q] : 0, e = a.po ? a.po[q + 1] : a.T;
            for (int64_t r = b; r < e && c < nchunk; r += CH) chunk_off[c++] = (int32_t)r;
        }
        for (; c <= nchunk; ++c) chunk_off[c] = (int32_t)a.T;
    }
    const int E = a.E, k = a.k, l = threadIdx.x % LPT;
    const int64_t t = (int64_t)blockIdx.x * TPC + threadIdx.x / LPT;
    const bool on = t < a.T;
    float* dps = reinterpret_cast<float*>(s_dp) + (threadIdx.x / LPT) * (NV * LPT);
    const int party = on && a.aux_coef ? party_of(a.po, a.P, t) : 0;
    float z[NV];
#pragma unroll
    for (int i = 0; i < NV; i += SP) {
        const int e = i * LPT + l * SP;
        if constexpr (SP == 4) {
            float4 v = make_float4(NINF, NINF, NINF, NINF), c = make_float4(0.f, 0.f, 0.f, 0.f);
            if (on && e < E) v = *reinterpret_cast<const float4*>(a.logits + t * E + e);
            if (on && e < E && a.aux_coef) c = *reinterpret_cast<const float4*>(a.aux_coef + (int64_t)party * E + e);
            z[i] = v.x; z[i + 1] = v.y; z[i + 2] = v.z; z[i + 3] = v.w;
            *reinterpret_cast<float4*>(dps + e) = c;
        } else {
            z[i] = on && e < E ? a.logits[t * E + e] : NINF;
            dps[e] = on && e < E && a.aux_coef ? a.aux_coef[(int64_t)party * E + e] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) z[i] = z[i] == z[i] ? z[i] : NINF;
    // lane j < k holds pick j
    const bool has = on && l < k;
    int pe = has ? a.topk_idx[t * k + l] : 0;
    float g = has ? a.dtopk_w[t * k + l] : 0.f;
    bool ok = has;
    if (has && (pe < 0 || pe >= E)) {
        record_status(MOE_ERR_DEVICE_CHECK);
        ok = false;
        g = 0.f;
        pe = 0;
    }
    float pz = ok ? a.logits[t * E + pe] : NINF;
    pz = pz == pz ? pz : NINF;
    float m = 0.f, inv = 1.f, s[NV], ps;
    if constexpr (SIG) {
        ps = 1.f / (1.f + expf(-pz));
    } else {
        m = NINF;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) m = fmaxf(m, z[i]);
        m = lanes_maxf<LPT>(m);
        m = m == NINF ? 0.f : m;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            s[i] = expf(z[i] - m);
            sum += s[i];
        }
        sum = lanes_sum<LPT>(sum);
        inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < NV; ++i) s[i] *= inv;
        ps = expf(pz - m) * inv;
    }
    float ds = a.scale * g;
    if (a.normalize) {
        const float total = lanes_sum<8>(ok ? ps : 0.f);
        const float inner = lanes_sum<8>(ok ? g * (a.scale * ps / total) : 0.f);
        ds = total == 0.f ? 0.f : (ds - inner) / total;
    }
    __syncwarp();
    if (ok) atomicAdd(&dps[pe], ds);  // the picks of a token differ: one addition per place
    __syncwarp();
    float dp[NV], dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i += SP) {
        const int e = i * LPT + l * SP;
        if constexpr (SP == 4) {
            const float4 v = *reinterpret_cast<const float4*>(dps + e);
            dp[i] = v.x; dp[i + 1] = v.y; dp[i + 2] = v.z; dp[i + 3] = v.w;
        } else {
            dp[i] = dps[e];
        }
    }
    if constexpr (!SIG) {
#pragma unroll
        for (int i = 0; i < NV; ++i) dot = fmaf(dp[i], s[i], dot);
        dot = lanes_sum<LPT>(dot);
    }
#pragma unroll
    for (int i = 0; i < NV; i += SP) {
        const int e = i * LPT + l * SP;
        float o[SP];
#pragma unroll
        for (int j = 0; j < SP; ++j) {
            if constexpr (SIG) {  // s (1 - s) without the difference's cancellation
                const float q = expf(-fabsf(z[i + j]));
                o[j] = dp[i + j] * q / ((1.f + q) * (1.f + q));
            } else {
                o[j] = s[i + j] * (dp[i + j] - dot);
            }
        }
        if (on && e < E) {
            if constexpr (SP == 4) *reinterpret_cast<float4*>(a.dlogits + t * E + e) = make_float4(o[0], o[1], o[2], o[3]);
            else a.dlogits[t * E + e] = o[0];
        }
        if (on && dz16) {
#pragma unroll
            for (int j = 0; j < SP; ++j)
                if (e + j < EP) dz16[t * EP + e + j] = __float2bfloat16_rn(e + j < E ? o[j] : 0.f);
        }
    }
    if (on && dz16)
        for (int e = NV * LPT + l; e < EP; e += LPT) dz16[t * EP + e] = __float2bfloat16_rn(0.f);
}

// out = in + rate * sign(mean - count), the comparison in whole numbers; one CTA per party
__global__ void __launch_bounds__(256) gate_balance_kernel(const int32_t* counts, int E, float rate, const float* in, float* out) {
    pdl_begin();
    __shared__ int64_t part[8];
    const int64_t at = (int64_t)blockIdx.x * E;
    const int e = threadIdx.x;
    const int64_t c = e < E ? counts[at + e] : 0;
    int64_t sum = c;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((e & 31) == 0) part[e >> 5] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += part[i];
    if (e < E) {
        const int64_t diff = sum - c * E;
        out[at + e] = in[at + e] + (diff > 0 ? rate : diff < 0 ? -rate : 0.f);
    }
}

// ---------------------------------------------------------------------------- launchers
static int pow2_ceil(int v) {
    int p = 1;
    while (p < v) p *= 2;
    return p;
}

template <int NV, int LPT>
static cudaError_t launch_gate_t(const GateArgs& a, int lpg, int nv, cudaStream_t s) {
    constexpr int TPC = GT_THREADS / LPT;
    // one pass of a CTA per token while that gives no more than eight CTAs per SM, then several
    int64_t ctas = (a.T + TPC - 1) / TPC;
    const int64_t most = 8 * (int64_t)sm_count();
    const int chunk = (int)(ctas <= most ? TPC : (ctas + most - 1) / most * TPC);
    ctas = (a.T + chunk - 1) / chunk;
    const bool whole = ctas == 1 && a.P == 1;  // the counts are this CTA's: stored, not added
    if (!whole) {
        const cudaError_t e = cudaMemsetAsync(a.counts, 0, sizeof(int32_t) * a.P * a.E, s);
        if (e != cudaSuccess) return e;
    }
    if (a.sigmoid)
        (void)launch_pdl(gate_kernel<NV, LPT, true>, dim3((unsigned)ctas), dim3(GT_THREADS), 0, s, a, lpg, nv, chunk, whole);
    else
        (void)launch_pdl(gate_kernel<NV, LPT, false>, dim3((unsigned)ctas), dim3(GT_THREADS), 0, s, a, lpg, nv, chunk, whole);
    return cudaGetLastError();
}

// Lanes per token: the fewest (8, 16, 32) that give every group a lane and hold the pool with at most
// eight scores a lane; 32 lanes hold up to 16 a lane (groups that are no power of two leave lanes idle).
cudaError_t launch_gate(const GateArgs& a0, cudaStream_t s) {
    GateArgs a = a0;
    if (a.T == 0) return cudaMemsetAsync(a.counts, 0, sizeof(int32_t) * a.P * a.E, s);
    const int Gp = pow2_ceil(a.groups), gs = a.E / a.groups;
    int lpt = 8;
    while (lpt < 32 && (lpt < Gp || (gs + lpt / Gp - 1) / (lpt / Gp) > 8)) lpt *= 2;
    const int lpg = lpt / Gp;
    int nv = (gs + lpg - 1) / lpg;
    if (nv > 2 && gs % 4 == 0) nv = (nv + 3) / 4 * 4;  // whole 16-byte spans (the last lanes of a group hold fewer)
    a.vec = nv % 4 == 0 && gs % 4 == 0 && (uintptr_t)a.logits % 16 == 0;
#define MOE_GATE(NV)                                              \
    (lpt == 8 ? launch_gate_t<NV, 8>(a, lpg, nv, s)               \
              : lpt == 16 ? launch_gate_t<NV, 16>(a, lpg, nv, s) : launch_gate_t<NV, 32>(a, lpg, nv, s))
    if (nv <= 2) return MOE_GATE(2);
    if (nv <= 4) return MOE_GATE(4);
    if (nv <= 8) return MOE_GATE(8);
    return launch_gate_t<16, 32>(a, lpg, nv, s);
#undef MOE_GATE
}

template <int NV, int LPT>
static cudaError_t launch_gate_bwd_t(const GateBwdArgs& a, __nv_bfloat16* dz16, int EP, int32_t* chunk_off, int CH, int nchunk,
                                     cudaStream_t s) {
    const unsigned ctas = (unsigned)((a.T + GT_THREADS / LPT - 1) / (GT_THREADS / LPT));
    const bool vec = a.E % 4 == 0 && (uintptr_t)a.logits % 16 == 0 && (uintptr_t)a.dlogits % 16 == 0 && (uintptr_t)a.aux_coef % 16 == 0;
#define MOE_GB(SP, SIG)                                                                                                        \
    (void)launch_pdl(gate_bwd_kernel<NV, LPT, SP, SIG>, dim3(ctas), dim3(GT_THREADS), 0, s, a, dz16, EP, chunk_off, CH, nchunk)
    if (a.sigmoid) {
        if (vec) MOE_GB(4, true);
        else MOE_GB(1, true);
    } else {
        if (vec) MOE_GB(4, false);
        else MOE_GB(1, false);
    }
#undef MOE_GB
    return cudaGetLastError();
}

cudaError_t launch_gate_bwd(const GateBwdArgs& a, __nv_bfloat16* dz16, int EP, int32_t* chunk_off, int CH, int nchunk, cudaStream_t s) {
    if (a.E <= 32) return launch_gate_bwd_t<4, 8>(a, dz16, EP, chunk_off, CH, nchunk, s);
    if (a.E <= 64) return launch_gate_bwd_t<8, 8>(a, dz16, EP, chunk_off, CH, nchunk, s);
    if (a.E <= 128) return launch_gate_bwd_t<8, 16>(a, dz16, EP, chunk_off, CH, nchunk, s);
    return launch_gate_bwd_t<8, 32>(a, dz16, EP, chunk_off, CH, nchunk, s);
}

cudaError_t launch_gate_balance(const int32_t* counts, int P, int E, float rate, const float* in, float* out, cudaStream_t s) {
    (void)launch_pdl(gate_balance_kernel, dim3(P), dim3(256), 0, s, counts, E, rate, in, out);
    return cudaGetLastError();
}

cudaError_t gate_status(cudaStream_t s, int* code) { return tu_status_read_clear(s, code); }

}  // namespace moe
