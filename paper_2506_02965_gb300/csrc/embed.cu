// Embedding lookup with scaling, and its gradient by sorted tokens.
//   out[t] = scale * W[id_t];   dW[v] (+)= scale * sum over t with id_t = v of dout[t]
// Both move rows and add them up, so HBM bounds them: the lookup reads the rows of the distinct ids and
// writes the batch; the gradient reads the batch and writes every row of dW (zeros where no token has the id),
// or reads and writes the tokens' rows when it adds to what is there.
//
// The gradient is a sum of rows in any order of ids, so the tokens are sorted by id first (stable: equal
// ids stay in the order of the batch) and runs of equal ids are added in fp32, in that order, by fixed chunks of
// the sorted tokens: no atomics, the same bits on every call. Three launches:
//   sort    one cluster of 1 to 8 CTAs, a stable radix sort of (id, token) by digits of up to 9 bits; every
//           warp owns a run of keys and counts their digits in shared memory, the CTAs read one another's
//           totals through distributed shared memory;
//   reduce  a party of threads per chunk of sorted tokens, a span of columns a thread: runs inside the chunk go
//           to dW, the parts of runs that cross a chunk's ends to the workspace as fp32; other CTAs zero the
//           rows without tokens meanwhile;
//   join    runs that crossed: their parts in order of the chunks.
#include <algorithm>
#include <type_traits>

#include "moe_internal.h"
#include "span.cuh"
#include "tc_ptx.cuh"

namespace moe {

namespace {

constexpr int SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_BITS = 9, SORT_BINS = 1 << SORT_BITS;
constexpr int SORT_MAX_CTAS = 8;
constexpr int PARTY = 256;  // threads of a CTA of the lookup, the sums and the joins

int chunk_len(int64_t T) { return T <= 8192 ? 32 : 64; }
int64_t chunks_of(int64_t T) { return (T + chunk_len(T) - 1) / chunk_len(T); }
int64_t words_of(int32_t V) { return ((int64_t)V + 31) / 32; }
size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// ---------------------------------------------------------------- lookup
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
struct SortBuf {
    int32_t* key[2];
    int32_t* tok[2];
    uint32_t* used;  // a bit per id, or null
};

// After an even number of passes the sorted tokens are in buffer 0, after an odd one in buffer 1.
__global__ void __launch_bounds__(SORT_THREADS) embed_sort_kernel(const int32_t* __restrict__ ids, int64_t T, int32_t V, int passes,
                                                                  int bits, SortBuf b) {
    pdl_begin();
    extern __shared__ int32_t s_hist[];  // [SORT_WARPS][bins]
    __shared__ int32_t s_tot[SORT_BINS], s_base[SORT_BINS], s_sum[SORT_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ctas = (int)gridDim.x, cta = (int)blockIdx.x;  // (the grid is one cluster)
    const int bins = 1 << bits;
    const int64_t warps = (int64_t)ctas * SORT_WARPS;
    const int64_t per = ((T + warps - 1) / warps + 31) / 32 * 32;
    const int64_t beg = min64(T, (cta * SORT_WARPS + warp) * per), end = min64(T, beg + per);
    int32_t* hist = s_hist + warp * bins;

    if (b.used) {
        const int64_t words = ((int64_t)V + 31) / 32;
        for (int64_t i = (int64_t)cta * SORT_THREADS + threadIdx.x; i < words; i += (int64_t)ctas * SORT_THREADS) b.used[i] = 0;
        tc::cluster_sync_all();
    }
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
        const int32_t *kin = b.key[p & 1], *tin = b.tok[p & 1];
        int32_t *kout = b.key[(p + 1) & 1], *tout = b.tok[(p + 1) & 1];
        // (through L2: another SM of the cluster wrote them)
        auto key_at = [&](int64_t i) -> int32_t {
            if (p > 0) return __ldcg(kin + i);
            const int32_t id = ids[i];
            return id < 0 || id >= V ? V : id;  // no row: after all others
        };
        for (int i = lane; i < bins; i += 32) hist[i] = 0;
        __syncwarp();
        for (int64_t i = beg + lane; i - lane < end; i += 32) {
            const bool in = i < end;
            const uint32_t there = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int32_t k = key_at(i);
                if (p == 0 && ids[i] >= V) record_status(MOE_ERR_DEVICE_CHECK);
                const uint32_t d = ((uint32_t)k >> shift) & (uint32_t)(bins - 1);
                const uint32_t same = __match_any_sync(there, d);
                if ((same & ((1u << lane) - 1)) == 0) hist[d] += __popc(same);
                if (p == 0 && b.used && k < V) atomicOr(b.used + (k >> 5), 1u << (k & 31));
            }
            __syncwarp();
        }
        __syncthreads();
        // digits in front of a warp's in its CTA, and the CTA's totals
        for (int d = threadIdx.x; d < bins; d += SORT_THREADS) {
            int32_t run = 0;
            for (int w = 0; w < SORT_WARPS; ++w) {
                const int32_t n = s_hist[w * bins + d];
                s_hist[w * bins + d] = run;
                run += n;
            }
            s_tot[d] = run;
        }
        tc::cluster_sync_all();
        // where a digit of this CTA begins: smaller digits of all CTAs, then this digit's of the CTAs before
        int32_t all = 0, before = 0;
        if ((int)threadIdx.x < bins) {
            const uint32_t mine = tc::smem_u32(&s_tot[threadIdx.x]);
            for (int r = 0; r < ctas; ++r) {
                const int32_t n = (int32_t)tc::ld_cluster(tc::map_to_rank(mine, (uint32_t)r));
                if (r < cta) before += n;
                all += n;
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
        int32_t ahead = 0;
        for (int w = 0; w < warp; ++w) ahead += s_sum[w];
        if ((int)threadIdx.x < bins) s_base[threadIdx.x] = ahead + inc - all + before;
        __syncthreads();
        for (int64_t i = beg + lane; i - lane < end; i += 32) {
            const bool in = i < end;
            const uint32_t there = __ballot_sync(0xffffffffu, in);
            if (in) {
                const int32_t k = key_at(i);
                const uint32_t d = ((uint32_t)k >> shift) & (uint32_t)(bins - 1);
                const uint32_t same = __match_any_sync(there, d);
                const int rank = __popc(same & ((1u << lane) - 1));
                const int64_t at = s_base[d] + hist[d] + rank;
                __syncwarp(there);
                if (rank == 0) hist[d] += __popc(same);
                kout[at] = k;
                tout[at] = p > 0 ? __ldcg(tin + i) : (int32_t)i;
            }
            __syncwarp();
        }
        tc::cluster_sync_all();  // the pass is written, and every CTA has read the totals
    }
}

// ---------------------------------------------------------------- sums
template <typename T> struct EmbedBwd {
    const int32_t* key;  // [T] sorted ids, V: no row
    const int32_t* tok;  // [T]
    const uint32_t* used;
    const T* dout;
    T* dw;
    float* part;  // [chunks][2][d]: of the run that came into the chunk, of the one that leaves it
    int64_t n;
    int32_t V;
    uint32_t spr;  // spans per row
    int chunk, party, slabs;
    int64_t sum_ctas;
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
    if ((int64_t)blockIdx.x >= a.sum_ctas) {
        // rows without tokens: 32 ids, one word of the bit table, a warp at a time
        const int64_t word = ((int64_t)blockIdx.x - a.sum_ctas) * (PARTY / 32) + (threadIdx.x >> 5);
        if (word * 32 >= a.V) return;
        const uint32_t used = a.used[word];
        const int rows = (int)min64(32, a.V - word * 32);
        Span<T, N> z;
        z.zero();
        for (int r = 0; r < rows; ++r) {
            if ((used >> r) & 1u) continue;
            T* row = a.dw + (word * 32 + r) * (int64_t)a.spr * N;
            for (uint32_t c = threadIdx.x & 31; c < a.spr; c += 32) z.store(row + (int64_t)c * N);
        }
        return;
    }
    const int parties = PARTY / a.party;
    const int64_t item = (int64_t)blockIdx.x * parties + threadIdx.x / a.party;
    const int64_t chunk = item / a.slabs;
    const uint32_t col = (uint32_t)(item % a.slabs) * a.party + threadIdx.x % a.party;
    const int64_t beg = chunk * a.chunk, end = min64(a.n, beg + a.chunk);
    if (beg >= end || col >= a.spr) return;
    int32_t run = a.key[beg];
    if (run >= a.V) return;
    bool came = beg > 0 && a.key[beg - 1] == run;
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
        int32_t k[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u] = p0 + u < end ? a.key[p0 + u] : a.V;
            v[u].zero();
            if (k[u] < a.V) v[u].load(a.dout + ((int64_t)a.tok[p0 + u] * a.spr + col) * N);
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
    const bool leaves = end < a.n && a.key[end] == run;
    if (came) part(0);
    else if (leaves) part(1);
    else embed_put<T, N>(a, run, col, acc);
}

// A run that begins in a chunk and leaves it: the chunk's part, then those of the chunks that it comes into.
template <typename T, int N>
__global__ void __launch_bounds__(PARTY) embed_join_kernel(const EmbedBwd<T> a) {
    pdl_begin();
    const int parties = PARTY / a.party;
    const int64_t item = (int64_t)blockIdx.x * parties + threadIdx.x / a.party;
    const int64_t chunk = item / a.slabs;
    const uint32_t col = (uint32_t)(item % a.slabs) * a.party + threadIdx.x % a.party;
    const int64_t beg = chunk * a.chunk, end = beg + a.chunk;
    if (end >= a.n || col >= a.spr) return;
    const int32_t run = a.key[end - 1];
    if (run >= a.V || a.key[end] != run) return;                       // nothing leaves
    if (a.key[beg] == run && beg > 0 && a.key[beg - 1] == run) return;  // it came in: not its first chunk
    float acc[N];
    const float* p = a.part + ((chunk * 2 + 1) * a.spr + col) * N;
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = p[j];
    for (int64_t c = chunk + 1; c * a.chunk < a.n && a.key[c * a.chunk] == run; ++c) {
        p = a.part + (c * 2 * a.spr + col) * N;
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] += p[j];
    }
    embed_put<T, N>(a, run, col, acc);
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
    a.sum_ctas = (items + parties - 1) / parties;
    const int64_t zero_ctas = a.accumulate ? 0 : (words_of(a.V) + PARTY / 32 - 1) / (PARTY / 32);
    (void)launch_pdl(embed_sum_kernel<T, N>, dim3((unsigned)(a.sum_ctas + zero_ctas)), dim3(PARTY), 0, s, a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || a.n <= a.chunk) return e;
    (void)launch_pdl(embed_join_kernel<T, N>, dim3((unsigned)a.sum_ctas), dim3(PARTY), 0, s, a);
    return cudaGetLastError();
}

}  // namespace

size_t embed_workspace_bytes(int64_t T, int32_t d, int32_t V) {
    return 4 * up((size_t)T * 4) + up((size_t)words_of(V) * 4) + up((size_t)chunks_of(T) * 2 * (size_t)d * 4);
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
    SortBuf b{};
    char* at = (char*)ws;
    for (int i = 0; i < 2; ++i) {
        b.key[i] = (int32_t*)at;
        at += up((size_t)T * 4);
        b.tok[i] = (int32_t*)at;
        at += up((size_t)T * 4);
    }
    uint32_t* used = (uint32_t*)at;
    at += up((size_t)words_of(V) * 4);
    b.used = accumulate ? nullptr : used;
    // keys are 0 .. V: digits of equal width, as few passes as 9 bits allow
    int all = 1;
    while (((int64_t)V >> all) > 0) ++all;
    const int passes = (all + SORT_BITS - 1) / SORT_BITS, bits = (all + passes - 1) / passes;
    int ctas = 1;
    while (ctas < SORT_MAX_CTAS && (int64_t)ctas * 2048 < T) ctas *= 2;
    const size_t smem = (size_t)SORT_WARPS * (size_t)(1 << bits) * 4;
    cudaError_t e = allow_dynamic_smem<embed_sort_kernel>((size_t)SORT_WARPS * SORT_BINS * 4);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
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
    cfg.numAttrs = 2;
    if ((e = cudaLaunchKernelEx(&cfg, embed_sort_kernel, ids, T, V, passes, bits, b)) != cudaSuccess) return e;

    auto args = [&](auto* t) {
        using E = std::remove_pointer_t<decltype(t)>;
        EmbedBwd<E> a{};
        a.key = b.key[passes & 1];
        a.tok = b.tok[passes & 1];
        a.used = used;
        a.dout = (const E*)dout;
        a.dw = (E*)dw;
        a.part = (float*)at;
        a.n = T;
        a.V = V;
        a.chunk = chunk_len(T);
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
