// Embedding lookup with scaling, and its gradient by sorted tokens.
//   out[t] = scale * W[id_t];   dW[v] (+)= scale * sum over t with id_t = v of dout[t]
// Both move rows and add them up, so HBM bounds them: the lookup reads the rows of the distinct ids and
// writes the batch; the gradient reads the batch and writes every row of dW (zeros where no token has the id),
// or reads and writes the tokens' rows when it adds to what is there.
//
// The gradient is a sum of rows in any order of ids, so the tokens are sorted by id first (stable: equal
// ids stay in the order of the batch) and runs of equal ids are added in fp32, in that order, by fixed chunks of
// the sorted tokens: no atomics, the same bits on every call. Three launches:
//   sort    one cluster of 1 to 16 CTAs, a stable radix sort of (id, token) by digits of up to 9 bits; every
//           warp owns a run of keys and counts their digits in shared memory, the CTAs read one another's
//           totals through distributed shared memory; the other SMs zero dW meanwhile;
//   sums    a party of threads per chunk of sorted tokens, a span of columns a thread: runs inside the chunk go
//           to dW, the parts of runs that cross a chunk's ends to the workspace as fp32;
//   joins   runs that crossed: their parts in order of the chunks.
#include <algorithm>
#include <type_traits>

#include "moe_internal.h"
#include "span.cuh"
#include "tc_ptx.cuh"

namespace moe {

namespace {

constexpr int SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_BITS = 9, SORT_BINS = 1 << SORT_BITS;
// Tokens that one CTA sorts; above, up to 16 of them (a cluster of that size has to be allowed, and found room for) with a
// thousand tokens each or more: a CTA takes 8 us and 2.7 more per thousand tokens, a cluster's barriers 4.
constexpr int SORT_MAX_CTAS = 16, SORT_ONE = 2048, SORT_PER_CTA = 1024;
constexpr int PARTY = 256;  // threads of a CTA of the lookup, the sums and the joins

// Sorted tokens per chunk: as many as leave one to two thousand threads an SM, 8 to 64 (a thread has eight rows on their
// way at once; each chunk leaves two rows of partial sums at most).
int chunk_len(int64_t T, int32_t d) {
    int n = 8;
    while (n < 64 && T * d / (8 * n) >= 2 * 152 * 1024) n *= 2;
    return n;
}
int64_t chunks_of(int64_t T, int32_t d) { return (T + chunk_len(T, d) - 1) / chunk_len(T, d); }
size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// ---------------------------------------------------------------- lookup
// A span of 16 bytes (or what the width and the addresses allow) a thread, four of them on their way where the batch is large:
// 16384 rows of 8 KB from 65536 in 31 us, 5.5 TB/s of DRAM; one row in 2.4 us, a launch and two dependent loads.
template <typename T, int N, int U>
__global__ void __launch_bounds__(PARTY) embed_fwd_kernel(const int32_t* __restrict__ ids, int64_t total, uint32_t spr, int32_t V,
                                                          const T* __restrict__ w, float scale, T* __restrict__ out) {
    pdl_begin();
    const int64_t first = (int64_t)blockIdx.x * (PARTY * U);
    const int64_t row0 = first / spr;
    const uint32_t col0 = (uint32_t)(first - row0 * spr);
    Span<T, N> v[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t at = col0 + (uint32_t)(u * PARTY) + threadIdx.x;
        const int64_t row = row0 + at / spr;
        live[u] = false;
        v[u].zero();
        if (first + u * PARTY + threadIdx.x < total) {
            const int32_t id = ids[row];
            live[u] = id >= 0 && id < V;
            if (id >= V) record_status(MOE_ERR_DEVICE_CHECK);
            if (live[u]) v[u].load(w + ((int64_t)id * spr + at % spr) * N);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = first + u * PARTY + threadIdx.x;
        if (i >= total) continue;
        if (live[u]) {
            float f[N];
            v[u].unpack(f);
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] *= scale;
            v[u].pack(f);
        }
        v[u].store(out + i * N);
    }
}

// ---------------------------------------------------------------- sort
struct SortArgs {
    const int32_t* ids;
    int64_t T;
    int32_t V;
    int passes, bits;
    int2* pair[2];             // (id, token) between passes; [0]: the result
    int32_t* runs;             // the sums' list of runs to join: its length, 0 here
    uint8_t* zero;             // dW, or null
    size_t zero_bytes;
};

// Zeros by all threads of the CTAs that do not sort: 16-byte stores but for the ends.
__device__ __forceinline__ void zero_fill(uint8_t* p, size_t bytes, int64_t part, int64_t parts) {
    const size_t head = min((size_t)(-(intptr_t)p & 15), bytes), words = (bytes - head) / 16, tail = head + words * 16;
    uint4* w = reinterpret_cast<uint4*>(p + head);
    for (size_t i = (size_t)part; i < words; i += (size_t)parts) w[i] = make_uint4(0, 0, 0, 0);
    if (part < (int64_t)head) p[part] = 0;
    if (part < (int64_t)(bytes - tail)) p[tail + part] = 0;
}

// The lanes of `there` whose digit is this lane's (a ballot per bit)
__device__ __forceinline__ uint32_t alike(uint32_t there, uint32_t digit, int bits) {
    uint32_t m = there;
#pragma unroll
    for (int b = 0; b < SORT_BITS; ++b) {
        if (b < bits) {
            const uint32_t one = (digit >> b) & 1u, v = __ballot_sync(there, one);
            m &= v ^ (one - 1u);
        }
    }
    return m;
}

// The first cluster sorts, the others zero dW. ONE: a cluster of one CTA, whose keys stay in shared memory between
// passes (T <= SORT_ONE).
template <bool ONE> __global__ void __launch_bounds__(SORT_THREADS) embed_sort_kernel(const SortArgs a, int ctas) {
    pdl_begin();
    if ((int)blockIdx.x >= ctas) {
        zero_fill(a.zero, a.zero_bytes, (int64_t)(blockIdx.x - ctas) * SORT_THREADS + threadIdx.x, (int64_t)(gridDim.x - ctas) * SORT_THREADS);
        return;
    }
    extern __shared__ int32_t s_hist[];  // [SORT_WARPS][bins], and of ONE [2][T] pairs
    __shared__ int32_t s_tot[SORT_BINS], s_base[SORT_BINS], s_sum[SORT_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = (int)blockIdx.x;
    const int bits = a.bits, bins = 1 << bits;
    const int64_t T = a.T, warps = (int64_t)ctas * SORT_WARPS;
    const int64_t per = ((T + warps - 1) / warps + 31) / 32 * 32;
    const int64_t beg = min64(T, (cta * SORT_WARPS + warp) * per), end = min64(T, beg + per);
    int32_t* hist = s_hist + warp * bins;
    int2* held = reinterpret_cast<int2*>(s_hist + SORT_WARPS * bins);

    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * bits, left = a.passes - 1 - p;
        const int2* from = ONE ? held + (left & 1) * T : a.pair[(left + 1) & 1];
        int2* to = ONE ? held + ((left + 1) & 1) * T : a.pair[left & 1];
        auto pair_at = [&](int64_t i) -> int2 {
            if (p > 0) return ONE ? from[i] : __ldcg(from + i);  // (through L2: another SM of the cluster wrote them)
            const int32_t id = a.ids[i];
            if (id >= a.V) record_status(MOE_ERR_DEVICE_CHECK);
            return make_int2(id < 0 || id >= a.V ? a.V : id, (int32_t)i);  // no row: after all others
        };
        for (int i = lane; i < bins; i += 32) hist[i] = 0;
        __syncwarp();
        // KEYS keys a lane at a time; a warp with no more than that keeps them, and who is alike, for the second walk
        constexpr int KEYS = 8;
        int2 k[KEYS];
        uint32_t same[KEYS];
        auto load_keys = [&](int64_t i0) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j) {
                const int64_t i = i0 + 32 * j + lane;
                k[j] = i < end ? pair_at(i) : make_int2(0, 0);
            }
        };
        for (int64_t i0 = beg; i0 < end; i0 += 32 * KEYS) {
            load_keys(i0);
#pragma unroll
            for (int j = 0; j < KEYS; ++j) {
                const int64_t i = i0 + 32 * j + lane;
                if (i - lane >= end) break;
                const uint32_t there = __ballot_sync(0xffffffffu, i < end);
                if (i < end) {
                    const uint32_t d = ((uint32_t)k[j].x >> shift) & (uint32_t)(bins - 1);
                    same[j] = alike(there, d, bits);
                    if ((same[j] & ((1u << lane) - 1)) == 0) hist[d] += __popc(same[j]);
                }
                __syncwarp();
            }
        }
        __syncthreads();
        // digits in front of a warp's in its CTA, and the CTA's totals
        for (int d = threadIdx.x; d < bins; d += SORT_THREADS) {
            int32_t n[SORT_WARPS], run = 0;
#pragma unroll
            for (int w = 0; w < SORT_WARPS; ++w) n[w] = s_hist[w * bins + d];
#pragma unroll
            for (int w = 0; w < SORT_WARPS; ++w) {
                s_hist[w * bins + d] = run;
                run += n[w];
            }
            s_tot[d] = run;
        }
        // where a digit of this CTA begins: smaller digits of all CTAs, then this digit's of the CTAs before
        int32_t all = 0, before = 0;
        if constexpr (ONE) {
            if ((int)threadIdx.x < bins) all = s_tot[threadIdx.x];  // (its own)
        } else {
            tc::cluster_sync_all();
            if ((int)threadIdx.x < bins) {
                const uint32_t mine = tc::smem_u32(&s_tot[threadIdx.x]);
                for (int r = 0; r < ctas; ++r) {
                    const int32_t n = (int32_t)tc::ld_cluster(tc::map_to_rank(mine, (uint32_t)r));
                    if (r < cta) before += n;
                    all += n;
                }
            }
        }
        int32_t inc = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        if (lane == 31) s_sum[warp] = inc;
        __syncthreads();
        if ((int)threadIdx.x < bins) {
            int32_t ahead = 0;
            for (int w = 0; w < warp; ++w) ahead += s_sum[w];
            s_base[threadIdx.x] = ahead + inc - all + before;
        }
        __syncthreads();
        for (int64_t i0 = beg; i0 < end; i0 += 32 * KEYS) {
            const bool again = per > 32 * KEYS;
            if (again) load_keys(i0);
#pragma unroll
            for (int j = 0; j < KEYS; ++j) {
                const int64_t i = i0 + 32 * j + lane;
                if (i - lane >= end) break;
                const uint32_t there = __ballot_sync(0xffffffffu, i < end);
                if (i < end) {
                    const uint32_t d = ((uint32_t)k[j].x >> shift) & (uint32_t)(bins - 1);
                    if (again) same[j] = alike(there, d, bits);
                    const int rank = __popc(same[j] & ((1u << lane) - 1));
                    const int64_t at = s_base[d] + hist[d] + rank;
                    __syncwarp(there);
                    if (rank == 0) hist[d] += __popc(same[j]);
                    to[at] = k[j];
                }
                __syncwarp();
            }
        }
        // the pass is written, and every CTA has read the totals
        if constexpr (ONE) __syncthreads();
        else tc::cluster_sync_all();
    }
    if constexpr (ONE) {  // out in whole lines (scattered stores take a cycle each)
        for (int i = threadIdx.x; i < (int)T; i += SORT_THREADS) a.pair[0][i] = held[T + i];
    }
    if (cta == 0 && threadIdx.x == 0) *a.runs = 0;
}

// ---------------------------------------------------------------- sums
// 16384 x 4096 bf16: 45 us, 4.7 TB/s (the batch's rows read, the distinct ids' written); 4096 x 1024: 7, three dependent loads.
template <typename T> struct EmbedBwd {
    const int2* pair;    // [T] ids in order with their tokens; id V: no row
    int32_t* runs;       // [1 + chunks]: how many runs leave the chunk that they begin in, and those chunks, in any order
    const T* dout;
    T* dw;
    float* part;  // [chunks][2][d]: of the run that came into the chunk, of the one that leaves it
    int64_t n;
    int32_t V;
    uint32_t spr;  // spans per row
    int chunk, party, slabs;
    float scale;
    int accumulate;
};

template <typename T, int N>
__device__ __forceinline__ void embed_put(const EmbedBwd<T>& a, int32_t id, uint32_t col, const float (&acc)[N]) {
    T* at = a.dw + ((int64_t)id * a.spr + col) * N;
    Span<T, N> s;
    float f[N];
    if (a.accumulate) {
        s.load(at);
        s.unpack(f);
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = fmaf(a.scale, acc[j], f[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = a.scale * acc[j];
    }
    s.pack(f);
    s.store(at);
}

template <typename T, int N>
__global__ void __launch_bounds__(PARTY) embed_sum_kernel(const EmbedBwd<T> a) {
    pdl_begin();
    constexpr int U = 8;
    const int parties = PARTY / a.party;
    const int64_t item = (int64_t)blockIdx.x * parties + threadIdx.x / a.party;
    const int64_t chunk = item / a.slabs;
    const uint32_t col = (uint32_t)(item % a.slabs) * a.party + threadIdx.x % a.party;
    const int64_t beg = chunk * a.chunk, end = min64(a.n, beg + a.chunk);
    if (beg >= end || col >= a.spr) return;
    int32_t run = a.pair[beg].x;
    if (run >= a.V) return;
    bool came = beg > 0 && a.pair[beg - 1].x == run;
    float acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
    auto part = [&](int which) {
        float* p = a.part + ((chunk * 2 + which) * a.spr + col) * N;
#pragma unroll
        for (int j = 0; j < N; ++j) p[j] = acc[j];
    };
    for (int64_t p0 = beg; p0 < end; p0 += U) {
        Span<T, N> v[U];
        int32_t k[U], t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int2 e = p0 + u < end ? a.pair[p0 + u] : make_int2(a.V, 0);
            k[u] = e.x;
            t[u] = e.y;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v[u].zero();
            if (k[u] < a.V) v[u].load(a.dout + ((int64_t)t[u] * a.spr + col) * N);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p0 + u < end && k[u] != run) {  // the run ended inside the chunk
                if (came) part(0);
                else embed_put<T, N>(a, run, col, acc);
                came = false;
                run = k[u];
                if (run >= a.V) return;
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] = 0.f;
            }
            float f[N];
            v[u].unpack(f);
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] += f[j];
        }
    }
    const bool leaves = end < a.n && a.pair[end].x == run;
    if (came) part(0);
    else if (leaves) {
        part(1);
        if (col == 0) a.runs[1 + atomicAdd(a.runs, 1)] = (int32_t)chunk;
    } else embed_put<T, N>(a, run, col, acc);
}

template <typename T, int N>
__device__ __forceinline__ void load_part(const EmbedBwd<T>& a, int64_t slot, uint32_t col, float (&v)[N]) {
    constexpr int W = N < 4 ? N : 4;
    const float* p = a.part + (slot * a.spr + col) * N;
#pragma unroll
    for (int i = 0; i < N / W; ++i) {
        Span<float, W> s;
        float f[W];
        s.load(p + i * W);
        s.unpack(f);
#pragma unroll
        for (int j = 0; j < W; ++j) v[i * W + j] = f[j];
    }
}

// A run that begins in a chunk and leaves it: the chunk's part and those of the chunks that it comes into. A CTA per run and
// slab of columns; its parties take equal shares of the run's chunks, each with JOIN parts on their way at once, and
// their sums are added in order: 16384 x 4096, whose most frequent id has 960 tokens, 18 us, 4096 x 1024 8. (The list's
// order is that of the sums' CTAs: it decides who does what, and no sum.)
constexpr int JOIN = 8;
template <typename T, int N>
__global__ void __launch_bounds__(PARTY) embed_join_kernel(const EmbedBwd<T> a) {
    pdl_begin();
    __shared__ float s_sum[PARTY][N];
    const int64_t chunks = (a.n + a.chunk - 1) / a.chunk, items = (int64_t)a.runs[0] * a.slabs;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t chunk = a.runs[1 + item / a.slabs];
        const int32_t run = a.pair[(chunk + 1) * a.chunk].x;
        int64_t more = 0;  // chunks that the run comes into
        for (;;) {
            const int64_t c = chunk + 1 + more + threadIdx.x;
            const int n = __syncthreads_count(c < chunks && a.pair[c * a.chunk].x == run);
            more += n;
            if (n < PARTY) break;
        }
        const int parties = PARTY / a.party, party = threadIdx.x / a.party;
        const uint32_t col = (uint32_t)(item % a.slabs) * a.party + threadIdx.x % a.party;
        const int64_t share = (more + parties - 1) / parties;
        const int64_t c0 = chunk + 1 + min64(more, party * share), c1 = chunk + 1 + min64(more, (party + 1) * share);
        float acc[N];
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] = 0.f;
        if (col < a.spr) {
            if (party == 0) load_part<T, N>(a, chunk * 2 + 1, col, acc);
            for (int64_t c = c0; c < c1; c += JOIN) {
                float v[JOIN][N];
#pragma unroll
                for (int u = 0; u < JOIN; ++u) {
#pragma unroll
                    for (int j = 0; j < N; ++j) v[u][j] = 0.f;
                    if (c + u < c1) load_part<T, N>(a, (c + u) * 2, col, v[u]);
                }
#pragma unroll
                for (int u = 0; u < JOIN; ++u)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] += v[u][j];
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) s_sum[threadIdx.x][j] = acc[j];
        __syncthreads();
        if (party == 0 && col < a.spr) {
            for (int q = 1; q < parties; ++q)
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] += s_sum[threadIdx.x + q * a.party][j];
            embed_put<T, N>(a, run, col, acc);
        }
        __syncthreads();
    }
}

// elements per access that the rows' width and the buffers' addresses allow, up to 16 bytes
int span_of(int32_t d, size_t es, const void* p, const void* q) {
    int n = (int)(16 / es);
    while (n > 1 && (d % n || (uintptr_t)p % (n * es) || (uintptr_t)q % (n * es))) n /= 2;
    return n;
}

template <typename T, int N>
cudaError_t fwd(const int32_t* ids, int64_t T_, int32_t d, int32_t V, const void* w, float scale, void* out, cudaStream_t s) {
    const uint32_t spr = (uint32_t)d / N;
    const int64_t total = T_ * spr;
    // one span a thread while that leaves SMs without work, else four (four loads in flight)
    if (total <= (int64_t)PARTY * 4 * sm_count())
        (void)launch_pdl(embed_fwd_kernel<T, N, 1>, dim3((unsigned)((total + PARTY - 1) / PARTY)), dim3(PARTY), 0, s, ids, total, spr, V,
                         (const T*)w, scale, (T*)out);
    else
        (void)launch_pdl(embed_fwd_kernel<T, N, 4>, dim3((unsigned)((total + 4 * PARTY - 1) / (4 * PARTY))), dim3(PARTY), 0, s, ids,
                         total, spr, V, (const T*)w, scale, (T*)out);
    return cudaGetLastError();
}

template <typename T, int N>
cudaError_t sums(EmbedBwd<T> a, int32_t d, cudaStream_t s) {
    a.spr = (uint32_t)d / N;
    a.party = 32;
    while (a.party < PARTY && (uint32_t)a.party < a.spr) a.party *= 2;
    a.slabs = (int)((a.spr + a.party - 1) / a.party);
    const int64_t items = (a.n + a.chunk - 1) / a.chunk * a.slabs, parties = PARTY / a.party;
    const unsigned ctas = (unsigned)((items + parties - 1) / parties);
    (void)launch_pdl(embed_sum_kernel<T, N>, dim3(ctas), dim3(PARTY), 0, s, a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || a.n <= a.chunk) return e;
    (void)launch_pdl(embed_join_kernel<T, N>, dim3((unsigned)std::min<int64_t>(items, 4 * sm_count())), dim3(PARTY), 0, s, a);
    return cudaGetLastError();
}

}  // namespace

size_t embed_workspace_bytes(int64_t T, int32_t d, int32_t V) {
    return 2 * up((size_t)T * 8) + up((size_t)(chunks_of(T, d) + 1) * 4) + up((size_t)chunks_of(T, d) * 2 * (size_t)d * 4);
}

cudaError_t launch_embed_fwd(const int32_t* ids, int64_t T, int32_t d, int32_t V, bool bf16, const void* w, float scale, void* out,
                             cudaStream_t s) {
    if (T == 0) return cudaSuccess;
    const int n = span_of(d, bf16 ? 2 : 4, w, out);
    if (bf16) {
        if (n == 8) return fwd<__nv_bfloat16, 8>(ids, T, d, V, w, scale, out, s);
        if (n == 4) return fwd<__nv_bfloat16, 4>(ids, T, d, V, w, scale, out, s);
        if (n == 2) return fwd<__nv_bfloat16, 2>(ids, T, d, V, w, scale, out, s);
        return fwd<__nv_bfloat16, 1>(ids, T, d, V, w, scale, out, s);
    }
    if (n == 4) return fwd<float, 4>(ids, T, d, V, w, scale, out, s);
    if (n == 2) return fwd<float, 2>(ids, T, d, V, w, scale, out, s);
    return fwd<float, 1>(ids, T, d, V, w, scale, out, s);
}

cudaError_t launch_embed_bwd(const int32_t* ids, int64_t T, int32_t d, int32_t V, bool bf16, const void* dout, float scale,
                             bool accumulate, void* dw, void* ws, cudaStream_t s) {
    if (T == 0)
        return accumulate ? cudaSuccess : cudaMemsetAsync(dw, 0, (size_t)V * (size_t)d * (bf16 ? 2 : 4), s);
    SortArgs b{};
    char* at = (char*)ws;
    for (int i = 0; i < 2; ++i) {
        b.pair[i] = (int2*)at;
        at += up((size_t)T * 8);
    }
    b.runs = (int32_t*)at;
    at += up((size_t)(chunks_of(T, d) + 1) * 4);
    b.ids = ids;
    b.T = T;
    b.V = V;
    if (!accumulate) {
        b.zero = (uint8_t*)dw;
        b.zero_bytes = (size_t)V * (size_t)d * (bf16 ? 2 : 4);
    }
    // keys are 0 .. V: digits of equal width, as few passes as 9 bits allow
    int all = 1;
    while (((int64_t)V >> all) > 0) ++all;
    b.passes = (all + SORT_BITS - 1) / SORT_BITS;
    b.bits = (all + b.passes - 1) / b.passes;
    const bool one = T <= SORT_ONE;
    int ctas = one ? 1 : 2;
    // (large clusters leave SMs without one, and so without a part in the zeros: four where those take longer than the sort;
    // 16384 tokens, 131072 x 4096: 255 us with four, 290 with 16)
    const int most = b.zero_bytes > (size_t)256 << 20 ? 4 : SORT_MAX_CTAS;
    while (!one && ctas < most && (int64_t)ctas * SORT_PER_CTA < T) ctas *= 2;
    const size_t smem = (size_t)SORT_WARPS * (size_t)(1 << b.bits) * 4 + (one ? (size_t)T * 16 : 0);
    cudaError_t e = allow_dynamic_smem<embed_sort_kernel<true>>((size_t)SORT_WARPS * SORT_BINS * 4 + (size_t)SORT_ONE * 16);
    if (e == cudaSuccess)
        e = once_per_device<embed_sort_kernel<false>>([] {
            const cudaError_t r = cudaFuncSetAttribute((const void*)embed_sort_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                       SORT_WARPS * SORT_BINS * 4);
            return r != cudaSuccess ? r : cudaFuncSetAttribute((const void*)embed_sort_kernel<false>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(SORT_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    // dW is zeroed by the SMs that do not sort, in one round: as many clusters as fit at once (19 of eight CTAs do
    // not: 131072 x 4096 237 us in two rounds, 170 in one)
    static std::atomic<int> resident[kMaxDevices][SORT_MAX_CTAS + 1] = {};  // 1 more than that
    const int dev = current_device();
    int clusters = 0;
    for (;; ctas /= 2) {
        std::atomic<int>* kept = dev >= 0 && dev < kMaxDevices ? &resident[dev][ctas] : nullptr;
        clusters = kept ? kept->load() - 1 : -1;
        if (clusters < 0) {
            cfg.gridDim = dim3((unsigned)(sm_count() / ctas * ctas));
            attr[0].val.clusterDim.x = (unsigned)ctas;
            if ((one ? cudaOccupancyMaxActiveClusters(&clusters, embed_sort_kernel<true>, &cfg)
                     : cudaOccupancyMaxActiveClusters(&clusters, embed_sort_kernel<false>, &cfg)) != cudaSuccess) {
                (void)cudaGetLastError();
                clusters = 0;
            }
            clusters = std::min(clusters, sm_count() / ctas);
            if (kept) *kept = clusters + 1;
        }
        if (clusters >= 2 || ctas <= 2) break;
    }
    attr[0].val.clusterDim.x = (unsigned)ctas;
    clusters = accumulate ? 1 : std::max(clusters, 2);
    cfg.gridDim = dim3((unsigned)(clusters * ctas));
    cfg.numAttrs = 2;
    if ((e = one ? cudaLaunchKernelEx(&cfg, embed_sort_kernel<true>, b, ctas) : cudaLaunchKernelEx(&cfg, embed_sort_kernel<false>, b, ctas)) !=
        cudaSuccess)
        return e;

    auto args = [&](auto* t) {
        using E = std::remove_pointer_t<decltype(t)>;
        EmbedBwd<E> a{};
        a.pair = b.pair[0];
        a.runs = b.runs;
        a.dout = (const E*)dout;
        a.dw = (E*)dw;
        a.part = (float*)at;
        a.n = T;
        a.V = V;
        a.chunk = chunk_len(T, d);
        a.scale = scale;
        a.accumulate = accumulate;
        return a;
    };
    const int n = span_of(d, bf16 ? 2 : 4, dout, dw);
    if (bf16) {
        const auto a = args((__nv_bfloat16*)nullptr);
        if (n == 8) return sums<__nv_bfloat16, 8>(a, d, s);
        if (n == 4) return sums<__nv_bfloat16, 4>(a, d, s);
        if (n == 2) return sums<__nv_bfloat16, 2>(a, d, s);
        return sums<__nv_bfloat16, 1>(a, d, s);
    }
    const auto a = args((float*)nullptr);
    if (n == 4) return sums<float, 4>(a, d, s);
    if (n == 2) return sums<float, 2>(a, d, s);
    return sums<float, 1>(a, d, s);
}

cudaError_t embed_status(cudaStream_t s, int* code) { return tu_status_read_clear(s, code); }

}  // namespace moe
