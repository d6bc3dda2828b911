// Gating rules beyond softmax and top-k: sigmoid or softmax scores, a balance bias that takes part
// in the choice only, expert groups of which some are kept, k picks, renormalised and scaled
// weights; their backward; the balance bias's update.
//
// Forward. A token's keys live in the registers of LPT lanes (8, 16 or 32: several tokens a warp), up to
// 32 a lane, each group of experts in an equal, power-of-two share of the lanes, so that a group's key
// is a reduction over aligned lanes. The k largest keys come out of sorting networks: every lane sorts its
// own, then lanes merge pairwise, each merge keeping the KT (2, 8) largest of two sorted lists; no
// step waits for the one before it as k rounds of "largest left" would.
// Picks are decided by exact keys. The networks sort approximate ones (scores by two instructions) in 23 bits,
// with the expert in 8 bits below: enough wherever the keys that decide lie further apart than the approximation, which is
// checked. Two groups too close (one token in 1000 of random ones) are decided by exact keys of their warp's
// tokens; experts too close (one in 1000) by the exact keys of those few against each other, or, where they are
// more than 24 (equal keys), by a whole warp, one pick after the other. So the time depends on the keys: where every token
// goes that way (all logits equal, as from a router of zeros, or every key coarser than the networks' units, a bias of 3
// and more beside sigmoid scores), 65536 x 256 takes 292 us with 8 groups and 161 without, not 41.5 and 30.4.
// What bounds the forward is the chain of a token's instructions (370 a token of 256 experts; issue slots half busy with the
// 16 warps an SM that 128 registers leave), not the row's one read: 65536 tokens, 256 experts, 8 groups, bias 41.5 us,
// without groups and bias 30.4 (the read: 10.5); with the scores written too, full-precision ones from a second read of the
// row, 74 and 51.6. Rounds of "largest left" in a warp per token with exact scores took 94.7.
// Also measured: keeping only keys above a floor, the k-th largest of the lanes' largest, and ranking those (16 keys a lane):
// 47 us against 44 of the networks, without groups 33 against 38, 20 against 15 for 64 experts and 11 against 9 for 16;
// the next rows copied ahead to shared memory: 44 (the reads back cost more than the wait).
//
// Backward: one read of the logits, one write of their gradient, HBM-bound (65536 x 256: 24.9 us, 0.82 of the copy rate; softmax
// 26.9, 0.76).
#include <algorithm>

#include "moe_common.cuh"
#include "moe_internal.h"

namespace moe {

constexpr int GT_THREADS = 256;
constexpr int gate_resident(int nv) { return nv > 16 ? 2 : 3; }  // CTAs per SM: 128 or 80 registers a thread (with less they spill)

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

// Floats in the order of unsigned integers; -0 counts as +0. The lowest is -inf, above 0.
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t u = __float_as_uint(__fadd_rn(f, 0.f));
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float unordered(uint32_t u) {
    return __uint_as_float((u & 0x80000000u) ? u ^ 0x80000000u : ~u);
}
constexpr uint32_t KEY_NINF = 0x007fffffu;  // ordered(-inf)

// ---------------------------------------------------------------- sorting networks, descending
__device__ __forceinline__ void cswap(uint32_t& a, uint32_t& b) {
    const uint32_t hi = max(a, b), lo = min(a, b);
    a = hi;
    b = lo;
}
// a bitonic list of N (a power of two)
template <int N> __device__ __forceinline__ void sort_bitonic(uint32_t* v) {
#pragma unroll
    for (int h = N / 2; h > 0; h >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(i & h)) cswap(v[i], v[i + h]);
}
// any list of N, Batcher's odd-even merge sort
template <int N> __device__ __forceinline__ void sort_any(uint32_t* v) {
#pragma unroll
    for (int p = 1; p < N; p <<= 1)
#pragma unroll
        for (int h = p; h > 0; h >>= 1)
#pragma unroll
            for (int j = h % p; j + h < N; j += 2 * h)
#pragma unroll
                for (int i = 0; i < h; ++i)
                    if (i + j + h < N && (i + j) / (2 * p) == (i + j + h) / (2 * p)) cswap(v[i + j], v[i + j + h]);
}
// a <- the N largest of two sorted lists, sorted
template <int N> __device__ __forceinline__ void merge_top(uint32_t* a, const uint32_t* b) {
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = max(a[i], b[N - 1 - i]);
    sort_bitonic<N>(a);
}
// a <- the N largest of two sorted lists, sorted; `rest`: the largest of the others, if that is larger
template <int N> __device__ __forceinline__ void merge_top(uint32_t* a, const uint32_t* b, uint32_t& rest) {
#pragma unroll
    for (int i = 0; i < N; ++i) rest = max(rest, min(a[i], b[N - 1 - i]));
    merge_top<N>(a, b);
}

// Score of one logit: softmax with the row's largest m and 1 / sum, or sigmoid.
template <bool SIG> __device__ __forceinline__ float score_of(float z, float m, float inv) {
    return SIG ? 1.f / (1.f + expf(-z)) : expf(z - m) * inv;
}

// Keys for sorting: the distance of a key below `top` (no key is above it), in units of KEY_RANGE / 2^23 up to
// KEY_RANGE (2 for sigmoid scores and their biases: 2.4e-7, 16 for logits: 1.9e-6), in bits 8 to 30 from
// the top down, and bit 31; an expert's 255 - id below, so that equal ones come in the order of their ids. Two
// keys of the exact order can come out the other way round only within KEY_SURE. In units, for a sigmoid key: the fast
// score is off by s (1 - s) (2^-22 + 1.23 |z| 2^-24) + 1.5 2^-23 s, at most 0.85, the exact one by 0.55, and their sums with the
// bias, below 4, can fall a spacing of at most 1 apart; the three roundings here are 1.25: 3.65 a key, 7.3 for two. Past 4
// sigmoid keys are not sure (fine_top), as they lie on a coarser grid than the units. Logits are exact: the roundings, 1.5 a
// key. (Keys past the range come out equal, and so not sure.) FLOOR: no finite key in the lowest 16 units, which are left
// to those out of reach.
template <bool SIG, bool FLOOR> __device__ __forceinline__ uint32_t sort_key(float key, float top, int id) {
    constexpr float RANGE = SIG ? 2.f : 16.f;
    float t = __saturatef(fmaf(key - top, 1.f / RANGE, 1.f));
    if (FLOOR) t = fmaxf(t, 0x1p-19f);
    return __float_as_uint(fmaf(t, 16777214.f, 16777216.f)) * 256u + (uint32_t)(255 - id);
}
constexpr uint32_t KEY_SURE = 9u << 8;
// Sums of two keys, of groups: 7.3 units for two sigmoid keys and 1 for the exact sum's own rounding below 8, 16.6 for two
// sums; 3 and 4 for two logits below 80, 14.
constexpr int SUM_SURE = 18;
// The top of the sort keys' range, past every key where they are on a coarser grid than that, so that none is sure
template <bool SIG> __device__ __forceinline__ float fine_top(float top, bool sums) {
    return (SIG ? fabsf(top - 1.f) < 3.f : !sums || fabsf(top) < 64.f) ? fmaxf(top, -3e38f) : 3e38f;
}
constexpr uint32_t KEY_OUT = 0x80000000u;  // a key out of reach, with its 255 - id
__device__ __forceinline__ int key_units(uint32_t u) { return (int)(u >> 8) & 0x7fffff; }

// Where a lane's slots lie in its group, in spans of 4 (VEC) or single places, the group's lanes in turn
template <bool VEC> struct Slots {
    int lpg, lg, cnt;  // lanes of the group, this one's place among them, the slots it holds
    __device__ __forceinline__ Slots(int lpg_, int lg_, int size) : lpg(lpg_), lg(lg_) {
        cnt = VEC ? (size / 4 - lg + lpg - 1) / lpg * 4 : (size - lg + lpg - 1) / lpg;
        cnt = size == 0 ? 0 : max(cnt, 0);
    }
    __device__ __forceinline__ int at(int i) const { return VEC ? ((i / 4) * lpg + lg) * 4 + i % 4 : i * lpg + lg; }
    // values of the slots from p (of the group's first expert); `none` past them
    template <int NV> __device__ __forceinline__ void load(const float* p, bool on, float none, float (&z)[NV]) const {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < NV; i += 4) {
                float4 v = make_float4(none, none, none, none);
                if (on && i < cnt) v = *reinterpret_cast<const float4*>(p + at(i));
                z[i] = v.x; z[i + 1] = v.y; z[i + 2] = v.z; z[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) z[i] = on && i < cnt ? p[at(i)] : none;
        }
    }
};

// the two largest of a group's keys, in all its lanes
template <typename V> __device__ __forceinline__ void group_best(V& b1, V& b2, int lpg) {
    for (int o = lpg >> 1; o > 0; o >>= 1) {
        const V c1 = __shfl_xor_sync(0xffffffffu, b1, o), c2 = __shfl_xor_sync(0xffffffffu, b2, o);
        b2 = max(min(b1, c1), max(b2, c2));
        b1 = max(b1, c1);
    }
}

constexpr int GT_CAND = 24;  // keys too close to tell that a token's own lanes decide
struct Candidates {
    int n, id[GT_CAND];
    uint32_t key[GT_CAND];
};

// The picks of one token by exact keys, by a whole warp: one after the other, the lowest id of the largest key
template <bool SIG>
__device__ __noinline__ void exact_token(const GateArgs& a, int64_t t, int* picks) {
    constexpr float NINF = -INFINITY;
    constexpr int NV = 16;  // of 256 experts over 32 lanes, of which a number of groups past a power of two leaves up to half idle
    int groups2 = 1;
    while (groups2 < a.groups) groups2 *= 2;
    const int lane = threadIdx.x & 31, lpg = 32 / groups2, grp = lane / lpg, gs = a.E / a.groups, first = grp * gs;
    const Slots<false> slots(lpg, lane % lpg, grp < a.groups ? gs : 0);
    const float* row = a.logits + t * a.E + first;
    const float* bias = a.bias ? a.bias + (int64_t)party_of(a.po, a.P, t) * a.E + first : nullptr;
    uint32_t u[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const float z = i < slots.cnt ? row[slots.at(i)] : NINF;
        float key = SIG ? score_of<true>(z, 0.f, 1.f) : z;
        if (bias && i < slots.cnt) key = __fadd_rn(key, bias[slots.at(i)]);
        u[i] = i >= slots.cnt ? 0u : z > NINF ? ordered(key) : KEY_NINF;
    }
    if (a.top_groups < a.groups) {
        uint32_t b1 = 0, b2 = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            b2 = max(b2, min(b1, u[i]));
            b1 = max(b1, u[i]);
        }
        group_best(b1, b2, lpg);
        const uint32_t mine = a.group_top == 2 ? ordered(unordered(b1) + unordered(b2)) : b1;
        int rank = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t other = __shfl_sync(0xffffffffu, mine, g * lpg);
            rank += other > mine || (other == mine && g < grp);
        }
        if (rank >= a.top_groups) {
#pragma unroll
            for (int i = 0; i < NV; ++i) u[i] = 0u;
        }
    }
    uint32_t best = 0, id = 0;  // the lane's largest and 256 less its lowest id
    auto scan = [&]() {
        best = id = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (u[i] > best) {
                best = u[i];
                id = (uint32_t)(256 - (first + slots.at(i)));
            }
    };
    scan();
    for (int j = 0; j < a.k; ++j) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, best);
        const uint32_t low = __reduce_max_sync(0xffffffffu, best == top ? id : 0u);
        if (lane == 0) picks[j] = 256 - (int)low;
        if (id == low) {  // one lane: its largest goes
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((uint32_t)(256 - (first + slots.at(i))) == low) u[i] = 0u;
            scan();
        }
    }
    __syncwarp();
}

template <int NV, int LPT, int KT, bool VEC, bool SIG>
__global__ void __launch_bounds__(GT_THREADS, gate_resident(NV)) gate_kernel(const __grid_constant__ GateArgs a, int lpg, int chunk,
                                                                         bool whole) {
    pdl_begin();
    constexpr float NINF = -INFINITY;
    constexpr int TPW = 32 / LPT, TPC = GT_THREADS / LPT;  // tokens per warp and per CTA at a time
    __shared__ int hist[256];
    __shared__ int s_pick[TPC][8];
    __shared__ Candidates s_cand[TPC];
    // the bias of the CTA's first party, four floats of room after each group: the lanes' spans lie in different banks
    __shared__ __align__(16) float s_bias[256 + 4 * 32];
    const int lane = threadIdx.x & 31, l = lane % LPT, base = lane - l;
    const int E = a.E, k = a.k, gs = E / a.groups, grp = l / lpg, first = grp * gs;
    const Slots<VEC> slots(lpg, l % lpg, grp < a.groups ? gs : 0);
    int* picks = s_pick[threadIdx.x / LPT];
    Candidates& cand = s_cand[threadIdx.x / LPT];
    const int64_t t0 = (int64_t)blockIdx.x * chunk, t1 = min64(t0 + chunk, a.T);
    const int p0 = party_of(a.po, a.P, t0);
    const bool one_party = party_of(a.po, a.P, t1 - 1) == p0;
    for (int e = threadIdx.x; e < E; e += GT_THREADS) {
        hist[e] = 0;
        if (a.bias) s_bias[e + e / gs * 4] = a.bias[(int64_t)p0 * E + e];
    }
    __syncthreads();
    int key_party = -1;
    float most_key = 1.f;
    // whole warps stay in the loop together: a token past the end computes nothing that is written
    for (int64_t tw = t0 + (threadIdx.x / 32) * TPW; tw < t1; tw += TPC) {
        const int64_t t = tw + lane / LPT;
        const bool on = t < t1;
        const int party = one_party || !on ? p0 : party_of(a.po, a.P, t);
        const float* row = a.logits + t * E + first;
        const float* bias = a.bias ? a.bias + (int64_t)party * E + first : nullptr;
        float key[NV], m = 0.f, inv = 1.f;
        slots.template load<NV>(row, on, NINF, key);
        // whether every slot of the warp holds an expert within reach: no test of single ones then
        float zero = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) zero = fmaf(key[i], 0.f, zero);  // NaN with an infinity or a NaN
        const bool clean = __all_sync(0xffffffffu, slots.cnt == NV && zero == 0.f);
        if constexpr (!SIG) {
            m = NINF;
#pragma unroll
            for (int i = 0; i < NV; ++i) m = fmaxf(m, key[i]);  // (passes over NaN)
            m = lanes_maxf<LPT>(m);
            m = m == NINF ? 0.f : m;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) sum += fast_exp(fmaxf(key[i] - m, NINF));  // NaN: 0
            sum = lanes_sum<LPT>(sum);
            inv = sum == 0.f ? 0.f : 1.f / sum;
        }
        if (a.scores && on) {  // (rolled loops here and below, which read the row again: the kernel's code stays small)
            float* out = a.scores + t * E + first;
#pragma unroll 1
            for (int i = 0; i < slots.cnt; i += VEC ? 4 : 1) {
                if constexpr (VEC) {
                    const float4 z = *reinterpret_cast<const float4*>(row + slots.at(i));
                    auto of = [&](float x) { return x > NINF ? score_of<SIG>(x, m, inv) : 0.f; };
                    const float4 o = make_float4(of(z.x), of(z.y), of(z.z), of(z.w));
                    if (a.scores_vec) *reinterpret_cast<float4*>(out + slots.at(i)) = o;
                    else out[slots.at(i)] = o.x, out[slots.at(i) + 1] = o.y, out[slots.at(i) + 2] = o.z, out[slots.at(i) + 3] = o.w;
                } else {
                    const float z = row[slots.at(i)];
                    out[slots.at(i)] = z > NINF ? score_of<SIG>(z, m, inv) : 0.f;
                }
            }
        }
        {
            float b[NV];
            if (bias) {
                if (party == p0) slots.template load<NV>(s_bias + grp * (gs + 4), true, NINF, b);
                else slots.template load<NV>(bias, true, NINF, b);
                if (SIG && __any_sync(0xffffffffu, party != key_party)) {  // the most a key of this party can be
                    key_party = party;
                    most_key = b[0];
#pragma unroll
                    for (int i = 1; i < NV; ++i) most_key = fmaxf(most_key, b[i]);
                    most_key = fine_top<true>(1.f + lanes_maxf<LPT>(most_key), true);
                }
            }
            if (clean) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if constexpr (SIG) key[i] = fast_sigmoid(key[i]);
                    if (bias) key[i] += b[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const bool reach = key[i] > NINF;  // (a NaN is out of reach)
                    if constexpr (SIG) key[i] = fast_sigmoid(key[i]);
                    if (bias) key[i] += b[i];
                    key[i] = reach ? key[i] : NINF;
                }
            }
        }
        float top = bias ? most_key : 1.f;
        if constexpr (!SIG) {
            top = key[0];
#pragma unroll
            for (int i = 1; i < NV; ++i) top = fmaxf(top, key[i]);
            top = fine_top<false>(lanes_maxf<LPT>(top), a.top_groups < a.groups);
        }
        // the lane's KT largest, sorted, and the largest of its others; 0 where there is no expert
        uint32_t v[KT], rest = 0;
        {
            uint32_t u[NV];
            if (clean) {
#pragma unroll
                for (int i = 0; i < NV; ++i) u[i] = sort_key<SIG, false>(key[i], top, first + slots.at(i));
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int id = first + slots.at(i);
                    u[i] = key[i] > NINF ? sort_key<SIG, true>(key[i], top, id) : KEY_OUT + (uint32_t)(255 - id);
                    if (i >= slots.cnt) u[i] = 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < KT; ++i) v[i] = i < NV ? u[i] : 0u;
            sort_any<KT>(v);
#pragma unroll
            for (int c = KT; c < NV; c += KT) {
                uint32_t w[KT];
#pragma unroll
                for (int i = 0; i < KT; ++i) w[i] = u[c + i];
                sort_any<KT>(w);
                merge_top<KT>(v, w, rest);
            }
        }
        bool kept = true;
        if (a.top_groups < a.groups) {
            // groups by the units of their best keys, those out of reach below in their order
            uint32_t b1 = v[0], b2 = v[1];
            group_best(b1, b2, lpg);
            constexpr int NEAR = SUM_SURE;
            const int n1 = key_units(b1), n2 = a.group_top == 2 ? key_units(b2) : n1;
            const bool gone = !clean && min(n1, n2) == 0;
            const int mine = gone ? -2 * NEAR * grp : 1 + NEAR + n1 + (a.group_top == 2 ? n2 : 0);
            int rank = 0, close = 0;  // groups ahead of this one; groups too close to tell, itself among them
            for (int g = 0; g < a.groups; ++g) {
                const int d = __shfl_sync(0xffffffffu, mine, base + g * lpg) - mine;
                rank += d > 0;
                close += (uint32_t)(d + NEAR) <= 2u * NEAR;
            }
            const bool sure = close == 1 && (gone || min(n1, n2) >= 32);  // (not at the end of the range)
            if (__any_sync(0xffffffffu, on && !sure && grp < a.groups)) {  // two groups too close: by exact keys
                float c1 = NINF, c2 = NINF;
#pragma unroll 8
                for (int i = 0; i < slots.cnt; ++i) {
                    const float z = on ? row[slots.at(i)] : NINF;
                    float x = SIG ? score_of<true>(z, 0.f, 1.f) : z;
                    if (bias) x = __fadd_rn(x, bias[slots.at(i)]);
                    x = z > NINF ? x : NINF;
                    c2 = fmaxf(c2, fminf(c1, x));
                    c1 = fmaxf(c1, x);
                }
                __syncwarp();
                group_best(c1, c2, lpg);
                const float sum = a.group_top == 2 ? c1 + c2 : c1;
                rank = 0;
                for (int g = 0; g < a.groups; ++g) {
                    const float other = __shfl_sync(0xffffffffu, sum, base + g * lpg);
                    rank += other > sum || (other == sum && g < grp);
                }
            }
            kept = rank < a.top_groups;
#pragma unroll
            for (int i = 0; i < KT; ++i) v[i] = kept ? v[i] : 0u;
            rest = kept ? rest : 0u;
        }
        uint32_t own[KT];  // the lane's, of which the next keeps the token's
#pragma unroll
        for (int i = 0; i < KT; ++i) own[i] = v[i];
#pragma unroll
        for (int o = 1; o < LPT; o <<= 1) {
            uint32_t w[KT];
#pragma unroll
            for (int i = 0; i < KT; ++i) w[i] = __shfl_xor_sync(0xffffffffu, v[i], o);
            merge_top<KT>(v, w);
        }
        // Sure where each of the k largest is clear of the next, and the last of all others, by their count; keys out
        // of reach are equal, and in the order of their ids
        uint32_t mine = v[0], last = v[0];
        bool sure = true;
#pragma unroll
        for (int i = 1; i < KT; ++i) {
            if (i < k) {
                sure &= last - v[i] >= KEY_SURE || (!clean && last < KEY_OUT + 256);
                last = v[i];
                mine = l == i ? v[i] : mine;
            }
        }
        const bool out = !clean && last < KEY_OUT + 256;
        last -= KEY_SURE;
        int n = rest >= last ? 1024 : 0;  // (keys that no list holds)
#pragma unroll
        for (int i = 0; i < KT; ++i) n += own[i] >= last;
#pragma unroll
        for (int o = 1; o < LPT; o <<= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        sure &= n == k || out;
        int pe = 255 - (int)(mine & 0xffu);
        if (__any_sync(0xffffffffu, on && !sure)) {
            // the few that are not clear of the k largest, by exact keys against each other
            if (l == 0) cand.n = 0;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < KT; ++i)
                if (own[i] >= last && !sure && n <= GT_CAND) cand.id[atomicAdd(&cand.n, 1)] = 255 - (int)(own[i] & 0xffu);
            __syncwarp();
            if (on && !sure && n <= GT_CAND) {
                for (int c = l; c < n; c += LPT) {
                    const int e = cand.id[c];
                    const float z = a.logits[t * E + e];
                    float x = SIG ? score_of<true>(z, 0.f, 1.f) : z;
                    if (bias) x = __fadd_rn(x, bias[e - first]);
                    cand.key[c] = z > NINF ? ordered(x) : KEY_NINF;
                }
            }
            __syncwarp();
            if (on && !sure && n <= GT_CAND) {
                for (int c = l; c < n; c += LPT) {
                    int rank = 0;
                    for (int o = 0; o < n; ++o)
                        rank += cand.key[o] > cand.key[c] || (cand.key[o] == cand.key[c] && cand.id[o] < cand.id[c]);
                    if (rank < k) picks[rank] = cand.id[c];
                }
            }
            __syncwarp();
            // many that are not (equal keys): each such token by the whole warp
            const uint32_t many = __ballot_sync(0xffffffffu, on && !sure && n > GT_CAND);
#pragma unroll 1
            for (int j = 0; j < TPW; ++j)
                if ((many >> (j * LPT)) & 1u) exact_token<SIG>(a, tw + j, s_pick[(threadIdx.x / 32) * TPW + j]);
            if (l < k && !sure) pe = picks[l];
            __syncwarp();
        }
        // pick j in lane j
        float ps = 0.f;
        if (on && l < k) {
            const float pz = a.logits[t * E + pe];
            ps = pz > NINF ? score_of<SIG>(pz, m, inv) : 0.f;
        }
        const float total = a.normalize ? lanes_sum<8>(ps) : 1.f;  // the picks are in a token's first 8 lanes
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

__global__ void __launch_bounds__(256) gate_zero_kernel(int32_t* counts, int n) {
    pdl_begin();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) counts[i] = 0;
}

// dlogits of a token by LPT lanes (several tokens a warp), NV scores a lane in spans of SP = 4 (or single ones).
// The picks' gradients touch k places of a row: the row is written as if there were none (but for
// their part in softmax's <ds, s>), then lane j writes pick j's place again (equal picks the same value). One read and one write of a
// row; fast exponentials (2^-22 of the result, as the row's sum).
template <int NV, int LPT, int SP, bool SIG>
__global__ void __launch_bounds__(GT_THREADS) gate_bwd_kernel(const __grid_constant__ GateBwdArgs a, __nv_bfloat16* dz16, int EP,
                                                              int32_t* chunk_off, int CH, int nchunk) {
    pdl_begin();
    constexpr float NINF = -INFINITY;
    constexpr int TPC = GT_THREADS / LPT;
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
    const float* row = a.logits + t * E;
    const float* aux = a.aux_coef && on ? a.aux_coef + (int64_t)party_of(a.po, a.P, t) * E : nullptr;
    float z[NV];
#pragma unroll
    for (int i = 0; i < NV; i += SP) {
        const int e = i * LPT + l * SP;
        if constexpr (SP == 4) {
            float4 v = make_float4(NINF, NINF, NINF, NINF);
            if (on && e < E) v = *reinterpret_cast<const float4*>(row + e);
            z[i] = v.x; z[i + 1] = v.y; z[i + 2] = v.z; z[i + 3] = v.w;
        } else {
            z[i] = on && e < E ? row[e] : NINF;
        }
    }
    // lane j < k holds pick j
    int pe = on && l < k ? a.topk_idx[t * k + l] : 0;
    float g = on && l < k ? a.dtopk_w[t * k + l] : 0.f;
    bool ok = on && l < k;
    if (ok && (pe < 0 || pe >= E)) {
        record_status(MOE_ERR_DEVICE_CHECK);
        ok = false;
    }
    g = ok ? g : 0.f;
    pe = ok ? pe : 0;
    const float pz = ok ? fmaxf(row[pe], NINF) : NINF;
    const float pa = ok && aux ? aux[pe] : 0.f;
    float m = 0.f, inv = 1.f;
    if constexpr (!SIG) {
        m = NINF;
#pragma unroll
        for (int i = 0; i < NV; ++i) m = fmaxf(m, z[i]);  // (passes over NaN)
        m = lanes_maxf<LPT>(m);
        m = m == NINF ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            z[i] = fast_exp(fmaxf(z[i] - m, NINF));  // NaN: 0
            sum += z[i];
        }
        sum = lanes_sum<LPT>(sum);
        inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < NV; ++i) z[i] *= inv;
    }
    const float ps = pz > NINF ? score_of<SIG>(pz, m, inv) : 0.f;
    float ds = a.scale * g;
    if (a.normalize) {
        // a constant added to every pick's g changes nothing, for the weights' sum is the scale: taken from the first
        // pick's on, the terms that cancel are small, and one pick alone has a gradient of exactly 0, not the roundings
        // of two equal terms over a sum that may be small
        const float total = lanes_sum<8>(ok ? ps : 0.f);
        const float g0 = g - __shfl_sync(0xffffffffu, g, 0, 8);
        const float inner = lanes_sum<8>(ok ? g0 * ps : 0.f);
        ds = total == 0.f ? 0.f : a.scale * (g0 - inner / total) / total;
    }
    // Picks that a caller brings may be equal: what all of an expert add to its score's gradient, in their order in each
    // of their lanes. Four steps round the eight lanes meet every pair, and a warp that has none goes on.
    float added = ds;
    const int pid = ok ? pe : -1 - l;
    bool twice = false;
#pragma unroll
    for (int o = 1; o <= 4; ++o) twice |= __shfl_sync(0xffffffffu, pid, (l + o) & 7, 8) == pid;
    if (__any_sync(0xffffffffu, twice)) {
        added = 0.f;
        for (int j = 0; j < k; ++j) {
            const int id = __shfl_sync(0xffffffffu, pid, j, 8);
            const float d = __shfl_sync(0xffffffffu, ds, j, 8);
            added += id == pid ? d : 0.f;
        }
    }
    float dot = 0.f;
    float c[NV];
#pragma unroll
    for (int i = 0; i < NV; i += SP) {
        const int e = i * LPT + l * SP;
        if constexpr (SP == 4) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (aux && e < E) v = *reinterpret_cast<const float4*>(aux + e);
            c[i] = v.x; c[i + 1] = v.y; c[i + 2] = v.z; c[i + 3] = v.w;
        } else {
            c[i] = aux && e < E ? aux[e] : 0.f;
        }
    }
    if constexpr (!SIG) {
        dot = ok ? ds * ps : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) dot = fmaf(c[i], z[i], dot);
        dot = lanes_sum<LPT>(dot);
    }
    // ds s (1 - s), without the difference's cancellation, or s (ds - <ds, s>)
    auto grad = [&](float zs, float d) {
        if constexpr (SIG) {
            const float q = fast_exp2(fmaxf(-fabsf(zs) * LOG2E, NINF));  // NaN: 0
            return d * q * fast_rcp((1.f + q) * (1.f + q));
        } else {
            return zs * (d - dot);
        }
    };
#pragma unroll
    for (int i = 0; i < NV; i += SP) {
        const int e = i * LPT + l * SP;
        float o[SP];
#pragma unroll
        for (int j = 0; j < SP; ++j) o[j] = grad(z[i + j], c[i + j]);
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
    __syncwarp();  // the picks' places are written after the row
    if (ok) {
        const float o = grad(SIG ? pz : ps, pa + added);
        a.dlogits[t * E + pe] = o;
        if (dz16) dz16[t * EP + pe] = __float2bfloat16_rn(o);
    }
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

template <int NV, int LPT, int KT, bool VEC>
static cudaError_t launch_gate_t(const GateArgs& a, int lpg, cudaStream_t s) {
    constexpr int TPC = GT_THREADS / LPT;
    // all CTAs resident at once, each with as many passes as the others
    const int64_t passes = (a.T + TPC - 1) / TPC, most = gate_resident(NV) * (int64_t)sm_count();
    const int chunk = (int)((passes + most - 1) / most * TPC);
    const int64_t ctas = (a.T + chunk - 1) / chunk;
    const bool whole = ctas == 1 && a.P == 1;  // the counts are this CTA's: stored, not added
    if (!whole) {
        (void)launch_pdl(gate_zero_kernel, dim3((a.P * a.E + 255) / 256), dim3(256), 0, s, a.counts, a.P * a.E);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    if (a.sigmoid)
        (void)launch_pdl(gate_kernel<NV, LPT, KT, VEC, true>, dim3((unsigned)ctas), dim3(GT_THREADS), 0, s, a, lpg, chunk, whole);
    else
        (void)launch_pdl(gate_kernel<NV, LPT, KT, VEC, false>, dim3((unsigned)ctas), dim3(GT_THREADS), 0, s, a, lpg, chunk, whole);
    return cudaGetLastError();
}

// Lanes per token: the fewest (8, 16, 32) that give every group a lane and hold the pool with at
// most 32 keys a lane, or 8 while even that leaves every warp resident: fewer lanes a token are fewer
// instructions, more are a shorter chain of them. E = 256, sigmoid, 8 groups, bias: 3000 and 3648 tokens with 8 keys a lane
// 7.2 and 8.1 us, 3649, 4096, 6000 and 9728 with 32 10.1, 11.4, 12.7 and 12.6, the next wave 14.1 (9729) to 17.0 (16384);
// softmax, one group: 6.6, 7.4 | 8.2, 6.4, 8.0, 7.9 | 11.3, 11.4. At 65536 tokens 32 keys a lane measured 39.6, 16 43.8, 8 66
// before the kernel had its present form; 16 between the two is not tried.
cudaError_t launch_gate(const GateArgs& a0, cudaStream_t s) {
    GateArgs a = a0;
    a.scores_vec = (uintptr_t)a.scores % 16 == 0;
    if (a.T == 0) return cudaMemsetAsync(a.counts, 0, sizeof(int32_t) * a.P * a.E, s);
    const int Gp = pow2_ceil(a.groups), gs = a.E / a.groups;
    auto lanes = [&](int keys) {
        int n = 8;
        while (n < 32 && (n < Gp || (gs + n / Gp - 1) / (n / Gp) > keys)) n *= 2;
        return n;
    };
    int lpt = lanes(8);
    if (a.T * lpt / GT_THREADS > gate_resident(8) * (int64_t)sm_count()) lpt = lanes(32);
    const int lpg = lpt / Gp;
    int nv = (gs + lpg - 1) / lpg;
    const bool vec = nv > 2 && gs % 4 == 0 && (uintptr_t)a.logits % 16 == 0 && (uintptr_t)a.bias % 16 == 0;
    if (vec) nv = (gs / 4 + lpg - 1) / lpg * 4;
#define MOE_GATE_K(NV, LPT, VEC) (a.k <= 2 ? launch_gate_t<NV, LPT, 2, VEC>(a, lpg, s) : launch_gate_t<NV, LPT, 8, VEC>(a, lpg, s))
#define MOE_GATE(NV, LPT) (vec ? MOE_GATE_K(NV, LPT, true) : MOE_GATE_K(NV, LPT, false))
    if (lpt == 8) return nv <= 2 ? MOE_GATE_K(2, 8, false) : nv <= 4 ? MOE_GATE(4, 8) : nv <= 8 ? MOE_GATE(8, 8) : nv <= 16 ? MOE_GATE(16, 8) : MOE_GATE(32, 8);
    if (lpt == 16) return nv <= 8 ? MOE_GATE(8, 16) : nv <= 16 ? MOE_GATE(16, 16) : MOE_GATE(32, 16);
    return nv <= 8 ? MOE_GATE(8, 32) : MOE_GATE(16, 32);
#undef MOE_GATE
#undef MOE_GATE_K
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
    if (a.E <= 128) return launch_gate_bwd_t<16, 8>(a, dz16, EP, chunk_off, CH, nchunk, s);
    return launch_gate_bwd_t<16, 16>(a, dz16, EP, chunk_off, CH, nchunk, s);
}

cudaError_t launch_gate_balance(const int32_t* counts, int P, int E, float rate, const float* in, float* out, cudaStream_t s) {
    (void)launch_pdl(gate_balance_kernel, dim3(P), dim3(256), 0, s, counts, E, rate, in, out);
    return cudaGetLastError();
}

cudaError_t gate_status(cudaStream_t s, int* code) { return tu_status_read_clear(s, code); }

}  // namespace moe
