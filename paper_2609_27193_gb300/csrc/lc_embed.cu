// lc_embed.cu -- the embedding lookup and its gradient.
//
// Lookup: y[t] = scale * table[ids[t]].  A copy of rows with one multiply, bound
// by memory (each distinct row read once, each output row written once).  A warp
// moves a segment of one row; a thread has U 16-byte loads in flight.
//
// Gradient: G[v] = scale * sum of dy[t] over the tokens with ids[t] == v.  The
// tokens are sorted by id (stable, so a row's tokens stay in ascending order),
// then the sorted list is cut into chunks of equal length and every chunk sums
// its rows: a word that half of the tokens share costs no more than any other
// chunk.  A row that lies inside one chunk is written by it; a row that crosses
// chunks leaves fp32 partial sums, which a last kernel adds in chunk order.  No
// floating point atomics: the order of every sum is fixed by the sizes.  The rows
// without a token are zeroed from a bitmap of the rows that have one.
#include <cooperative_groups.h>

#include "lc_ops.cuh"

namespace cg = cooperative_groups;

namespace lc {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortCluster = 8;
constexpr int kSortBits = 9;                 // digits of at most 9 bits
constexpr int64_t kSortAlone = 2048;         // up to this many tokens one CTA sorts
constexpr int kSumThreads = 128;
constexpr int64_t kMaxTokens = int64_t(1) << 31;

struct EmbedParams {
    const uint8_t* table;
    const void* ids;
    uint8_t* y;
    int64_t vocab, dim, table_pitch, y_pitch, ntok;   // pitches in bytes
    int64_t items, segs;                              // items = ntok * segs (segments of a row)
    float scale;
};

// V elements an access: a 16-byte vector, or one element where an address or a
// pitch is off 16 bytes.
template <typename T, typename I, int V, int U>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(EmbedParams p) {
    const int lane = threadIdx.x & 31;
    const int64_t step = int64_t(gridDim.x) * (kEmbedThreads / 32);
    for (int64_t item = int64_t(blockIdx.x) * (kEmbedThreads / 32) + (threadIdx.x >> 5); item < p.items; item += step) {
        const int64_t t = item / p.segs;
        const int64_t c0 = (item - t * p.segs) * (32 * V * U) + lane * V;
        const int64_t id = int64_t(static_cast<const I*>(p.ids)[t]);
        const bool row = id >= 0 && id < p.vocab;
        const T* src = reinterpret_cast<const T*>(p.table + (row ? id : 0) * p.table_pitch);
        T* dst = reinterpret_cast<T*>(p.y + t * p.y_pitch);
        const float fill = id < 0 ? 0.0f : __uint_as_float(0x7fffffffu);
        if constexpr (V > 1) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t c = c0 + u * 32 * V;
                if (row && c + V <= p.dim) v[u] = __ldg(reinterpret_cast<const uint4*>(src + c));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t c = c0 + u * 32 * V;
                if (c + V <= p.dim) {
                    float f[V];
                    unpack(v[u], f);
#pragma unroll
                    for (int i = 0; i < V; ++i) f[i] = row ? f[i] * p.scale : fill;
                    st_stream(dst + c, pack(f));
                } else {
                    for (int64_t k = c; k < p.dim; ++k) dst[k] = from_f32<T>(row ? to_f32(src[k]) * p.scale : fill);
                }
            }
        } else {
            T v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t c = c0 + u * 32;
                if (row && c < p.dim) v[u] = src[c];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t c = c0 + u * 32;
                if (c < p.dim) dst[c] = from_f32<T>(row ? to_f32(v[u]) * p.scale : fill);
            }
        }
    }
}

template <typename T, typename I>
cudaError_t launch_embed(EmbedParams p, int sms, cudaStream_t s) {
    constexpr int V = kVec<T>, U = 4;
    const bool vec = aligned16(p.table) && aligned16(p.y) && p.table_pitch % 16 == 0 && p.y_pitch % 16 == 0;
    const int64_t per = vec ? 32 * V * U : 32 * 8;
    p.segs = (p.dim + per - 1) / per;
    p.items = p.ntok * p.segs;
    const int64_t want = (p.items + kEmbedThreads / 32 - 1) / (kEmbedThreads / 32);
    const int64_t most = int64_t(sms) * 256;
    const unsigned grid = unsigned(want < most ? want : most);
    cudaGetLastError();
    if (vec) embed_kernel<T, I, V, U><<<grid, kEmbedThreads, 0, s>>>(p);
    else embed_kernel<T, I, 1, 8><<<grid, kEmbedThreads, 0, s>>>(p);
    return cudaGetLastError();
}

// --- the gradient -----------------------------------------------------------

struct SortParams {
    const void* ids;
    int64_t n, vocab, skip;
    uint32_t* key[2];
    uint32_t* pos[2];
    uint32_t* present;     // bitmap of the rows that have a token (null: not wanted)
    int32_t digit, passes; // bits of a digit, digits
};

// Sorts the tokens by id: least significant digit first, each pass a stable
// counting sort.  One cluster does it all: every warp owns a contiguous range of
// the list, counts its digits (lanes with the same digit find one another by
// match), the counts become offsets by sums over the warps, the cluster's CTAs
// (distributed shared memory) and the digits, and the warp hands its items out in
// order.  Tokens that contribute nothing get the key `vocab` and end up last.
template <typename I>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(SortParams p) {
    extern __shared__ uint32_t sm[];
    __shared__ uint32_t tot[1 << kSortBits];
    __shared__ uint32_t warp_sum[kSortWarps];
    dependents_may_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = int(cluster.block_rank()), nc = int(cluster.num_blocks());
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bins = 1 << p.digit;
    uint32_t* cnt = sm + warp * bins;
    int64_t per = (p.n + int64_t(nc) * kSortWarps - 1) / (int64_t(nc) * kSortWarps);
    per = (per + 31) & ~int64_t(31);
    int64_t lo = (int64_t(rank) * kSortWarps + warp) * per;
    lo = lo < p.n ? lo : p.n;
    const int64_t hi = lo + per < p.n ? lo + per : p.n;
    if (p.present) {
        const int64_t words = (p.vocab + 31) / 32;
        for (int64_t i = int64_t(rank) * kSortThreads + threadIdx.x; i < words; i += int64_t(nc) * kSortThreads)
            p.present[i] = 0;
    }
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * p.digit;
        const uint32_t* ksrc = p.key[(pass & 1) ^ 1];
        const uint32_t* psrc = p.pos[(pass & 1) ^ 1];
        auto key_at = [&](int64_t i) -> uint32_t {
            if (pass) return __ldcg(ksrc + i);
            const int64_t id = int64_t(static_cast<const I*>(p.ids)[i]);
            return uint32_t(id >= 0 && id < p.vocab && id != p.skip ? id : p.vocab);
        };
        for (int b = lane; b < bins; b += 32) cnt[b] = 0;
        __syncwarp();
        for (int64_t i = lo; i < hi; i += 32) {
            const bool in = i + lane < hi;
            const uint32_t d = in ? (key_at(i + lane) >> shift) & uint32_t(bins - 1) : ~0u;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            if (in && lane == __ffs(same) - 1) cnt[d] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        for (int b = threadIdx.x; b < bins; b += kSortThreads) {
            uint32_t s = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = sm[w * bins + b];
                sm[w * bins + b] = s;
                s += c;
            }
            tot[b] = s;
        }
        cluster.sync();
        // bins <= kSortThreads: a thread a digit value
        uint32_t before = 0, all = 0;
        if (int(threadIdx.x) < bins)
            for (int r = 0; r < nc; ++r) {
                const uint32_t t = cluster.map_shared_rank(tot, r)[threadIdx.x];
                if (r < rank) before += t;
                all += t;
            }
        uint32_t scan = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        uint32_t base = before + scan - all;
        for (int w = 0; w < warp; ++w) base += warp_sum[w];
        if (int(threadIdx.x) < bins)
            for (int w = 0; w < kSortWarps; ++w) sm[w * bins + threadIdx.x] += base;
        __syncthreads();
        uint32_t* kdst = p.key[pass & 1];
        uint32_t* pdst = p.pos[pass & 1];
        for (int64_t i = lo; i < hi; i += 32) {
            const bool in = i + lane < hi;
            const uint32_t key = in ? key_at(i + lane) : 0u;
            const uint32_t d = in ? (key >> shift) & uint32_t(bins - 1) : ~0u;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            uint32_t at = 0;
            if (in) at = cnt[d] + __popc(same & ((1u << lane) - 1));
            __syncwarp();
            if (in && lane == __ffs(same) - 1) cnt[d] += __popc(same);
            __syncwarp();
            if (in) {
                kdst[at] = key;
                pdst[at] = pass ? __ldcg(psrc + i + lane) : uint32_t(i + lane);
            }
        }
        cluster.sync();
    }
    if (p.present) {
        const uint32_t* key = p.key[(p.passes - 1) & 1];
        for (int64_t i = lo + lane; i < hi; i += 32) {
            const uint32_t k = __ldcg(key + i);
            if (k < p.vocab && (i == 0 || __ldcg(key + i - 1) != k)) atomicOr(p.present + k / 32, 1u << (k & 31));
        }
    }
}

struct SumParams {
    const uint32_t* key;
    const uint32_t* pos;
    const uint32_t* present;
    const uint8_t* dy;
    uint8_t* grad;
    float* part;          // [chunks][2][slabs][kSumThreads][E]: a chunk's open rows at its start and end
    int64_t n, vocab, dim, dy_pitch, grad_pitch;
    int64_t chunk, chunks, slabs, sum_ctas, zero_rows;
    float scale;
    int32_t accumulate;
};

// The columns of a thread: E consecutive ones (16-byte loads of dy), or E that lie
// kSumThreads apart (single elements).
template <typename TD, bool VEC>
struct Columns {
    static constexpr int E = VEC ? kVec<TD> : 4;
    int64_t c0;
    int64_t dim;
    __device__ Columns(int64_t slab, int64_t d)
        : c0(slab * kSumThreads * E + (VEC ? int(threadIdx.x) * E : int(threadIdx.x))), dim(d) {}
    __device__ int64_t col(int e) const { return VEC ? c0 + e : c0 + int64_t(e) * kSumThreads; }
    __device__ bool whole() const { return VEC && c0 + E <= dim; }
    __device__ void load(const uint8_t* row, float (&f)[E]) const {
        const TD* r = reinterpret_cast<const TD*>(row);
        if constexpr (VEC) {
            if (whole()) {
                unpack(ld_stream(r + c0), f);
                return;
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = col(e) < dim ? to_f32(r[col(e)]) : 0.0f;
    }
    // grad = f (+ grad)
    template <typename TG>
    __device__ void store(uint8_t* row, const float (&f)[E], bool add) const {
        TG* r = reinterpret_cast<TG*>(row);
        if constexpr (VEC) {
            if (whole()) {
                constexpr int B = E * int(sizeof(TG));   // 8, 16 or 32 bytes
                uint32_t w[B / 4];
                if (add) {
#pragma unroll
                    for (int i = 0; i < B / 4; i += 2) {
                        const uint2 o = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint32_t*>(r + c0) + i);
                        w[i] = o.x;
                        w[i + 1] = o.y;
                    }
                }
                if constexpr (sizeof(TG) == 4) {
#pragma unroll
                    for (int e = 0; e < E; ++e) w[e] = __float_as_uint(add ? __uint_as_float(w[e]) + f[e] : f[e]);
                } else {
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        float a = f[2 * i], b = f[2 * i + 1];
                        if (add) {
                            a += __uint_as_float(w[i] << 16);
                            b += __uint_as_float(w[i] & 0xffff0000u);
                        }
                        w[i] = pack_bf16(a, b);
                    }
                }
                uint32_t* dst = reinterpret_cast<uint32_t*>(r + c0);
                if constexpr (B == 8) {
                    *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
                } else {
#pragma unroll
                    for (int i = 0; i < B / 4; i += 4) st_stream(dst + i, make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
                }
                return;
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (col(e) < dim) r[col(e)] = from_f32<TG>(add ? to_f32(r[col(e)]) + f[e] : f[e]);
    }
};

__device__ __forceinline__ int64_t part_at(const SumParams& p, int64_t chunk, int which, int64_t slab, int E) {
    return (((chunk * 2 + which) * p.slabs + slab) * kSumThreads + threadIdx.x) * E;
}

template <typename TD, typename TG, bool VEC>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(SumParams p) {
    using Cols = Columns<TD, VEC>;
    constexpr int E = Cols::E;
    constexpr int U = 8;   // rows in flight
    dependency_wait();
    dependents_may_start();
    if (int64_t(blockIdx.x) >= p.sum_ctas) {
        // rows without a token
        const int64_t r0 = (int64_t(blockIdx.x) - p.sum_ctas) * p.zero_rows;
        const int64_t r1 = r0 + p.zero_rows < p.vocab ? r0 + p.zero_rows : p.vocab;
        const int64_t bytes = p.dim * int64_t(sizeof(TG));
        for (int64_t r = r0; r < r1; ++r) {
            if (p.present[r / 32] >> (r & 31) & 1) continue;
            uint8_t* row = p.grad + r * p.grad_pitch;
            int64_t done = 0;
            if constexpr (VEC) {
                const int64_t nv = bytes / 16;
                for (int64_t i = threadIdx.x; i < nv; i += kSumThreads) st_stream(row + i * 16, make_uint4(0, 0, 0, 0));
                done = nv * 16;
            }
            for (int64_t i = done / int64_t(sizeof(TG)) + threadIdx.x; i < p.dim; i += kSumThreads)
                reinterpret_cast<TG*>(row)[i] = from_f32<TG>(0.0f);
        }
        return;
    }
    const int64_t chunk = blockIdx.x / p.slabs, slab = blockIdx.x % p.slabs;
    const Cols cols(slab, p.dim);
    const int64_t s0 = chunk * p.chunk;
    const int64_t s1 = s0 + p.chunk < p.n ? s0 + p.chunk : p.n;
    const uint32_t none = uint32_t(p.vocab);
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    uint32_t key = p.key[s0];
    bool open = s0 > 0 && p.key[s0 - 1] == key;   // the row began in an earlier chunk
    for (int64_t s = s0; s < s1; s += U) {
        uint32_t k[U + 1];
        float f[U][E];
#pragma unroll
        for (int u = 0; u <= U; ++u) k[u] = s + u < p.n && s + u <= s1 ? p.key[s + u] : none;
        if (k[0] == none) break;   // sorted last: nothing more contributes
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < s1 && k[u] != none) cols.load(p.dy + int64_t(p.pos[s + u]) * p.dy_pitch, f[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s + u >= s1 || k[u] == none) break;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += f[u][e];
            const bool last = s + u + 1 >= s1;
            const uint32_t next = k[u + 1];
            if (next == k[u] && !last) continue;
            if (open || (last && next == k[u])) {
                float* out = p.part + part_at(p, chunk, open ? 0 : 1, slab, E);
#pragma unroll
                for (int e = 0; e < E; ++e) out[e] = acc[e];
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] *= p.scale;
                cols.template store<TG>(p.grad + int64_t(k[u]) * p.grad_pitch, acc, p.accumulate != 0);
            }
            open = false;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = 0.0f;
        }
    }
}

// Rows that cross chunks: the CTA of the chunk in which the row begins adds its
// parts in order.
template <typename TD, typename TG, bool VEC>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(SumParams p) {
    using Cols = Columns<TD, VEC>;
    constexpr int E = Cols::E;
    constexpr int U = 8;
    dependency_wait();
    const int64_t chunk = blockIdx.x / p.slabs, slab = blockIdx.x % p.slabs;
    const int64_t s0 = chunk * p.chunk, s1 = s0 + p.chunk;
    if (s1 >= p.n) return;
    const uint32_t key = p.key[s1];
    if (key == uint32_t(p.vocab) || p.key[s1 - 1] != key) return;              // no row crosses this chunk's end
    if (s0 > 0 && p.key[s0 - 1] == key) return;                                // it began in an earlier chunk
    // chunks c in (chunk, last] begin with this row: the largest one, by bisection
    int64_t lo = chunk + 1, hi = p.chunks - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (p.key[mid * p.chunk] == key) lo = mid;
        else hi = mid - 1;
    }
    const int64_t stride = p.slabs * 2 * kSumThreads * E;
    const float* first = p.part + part_at(p, chunk, 1, slab, E);
    const float* rest = p.part + part_at(p, chunk + 1, 0, slab, E);
    const int64_t m = lo - chunk;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = first[e];
    for (int64_t i = 0; i < m; i += U) {
        float f[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) f[u][e] = i + u < m ? rest[(i + u) * stride + e] : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += f[u][e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= p.scale;
    const Cols cols(slab, p.dim);
    cols.template store<TG>(p.grad + int64_t(key) * p.grad_pitch, acc, p.accumulate != 0);
}

constexpr size_t al256(size_t x) { return (x + 255) & ~size_t(255); }

// Chunks of the sorted list: long enough to fill the device a few times over, at
// most 1024 of them beyond that, so that a row which all tokens share is joined
// from no more parts.
int64_t chunk_of(int64_t n, int64_t slabs) {
    int64_t c = n * slabs / 2432;
    if (c < n / 1024) c = n / 1024;
    c = (c + 7) / 8 * 8;
    return c < 8 ? 8 : c;
}

struct GradLayout {
    size_t key[2], pos[2], present, part, bytes;
};
// E: the columns of a thread; more of them are more partial sums a chunk.
GradLayout grad_layout(int64_t n, int64_t vocab, int64_t part_floats) {
    GradLayout l{};
    size_t at = 0;
    for (int i = 0; i < 2; ++i) {
        l.key[i] = at;
        at += al256(size_t(n) * 4);
        l.pos[i] = at;
        at += al256(size_t(n) * 4);
    }
    l.present = at;
    at += al256(size_t((vocab + 31) / 32) * 4);
    l.part = at;
    l.bytes = at + al256(size_t(part_floats) * 4);
    return l;
}

struct SumShape {
    int64_t slabs, chunk, chunks, part_floats;
};
SumShape sum_shape(int64_t n, int64_t dim, int E) {
    SumShape s;
    s.slabs = (dim + kSumThreads * E - 1) / (kSumThreads * E);
    s.chunk = chunk_of(n, s.slabs);
    s.chunks = (n + s.chunk - 1) / s.chunk;
    s.part_floats = s.chunks * 2 * s.slabs * kSumThreads * E;
    return s;
}

template <typename TD, typename TG, bool VEC>
cudaError_t launch_sum(SumParams p, const SumShape& sh, cudaStream_t s) {
    p.slabs = sh.slabs;
    p.chunk = sh.chunk;
    p.chunks = sh.chunks;
    p.sum_ctas = sh.chunks * sh.slabs;
    int64_t zero = 0;
    if (!p.accumulate) {
        p.zero_rows = 65536 / (p.dim * int64_t(sizeof(TG)));
        p.zero_rows = p.zero_rows < 1 ? 1 : p.zero_rows > 256 ? 256 : p.zero_rows;
        zero = (p.vocab + p.zero_rows - 1) / p.zero_rows;
    }
    cudaError_t e = launch_dependent(embed_sum_kernel<TD, TG, VEC>, int(p.sum_ctas + zero), kSumThreads, 0, s, p);
    if (e == cudaSuccess && p.chunks > 1)
        e = launch_dependent(embed_join_kernel<TD, TG, VEC>, int(p.sum_ctas), kSumThreads, 0, s, p);
    return e;
}

template <typename I>
cudaError_t launch_sort(const SortParams& p, cudaStream_t s) {
    const size_t smem = size_t(kSortWarps) * (size_t(1) << p.digit) * 4;
    static bool ready[kOpsMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(embed_sort_kernel<I>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSortWarps * (1 << kSortBits) * 4);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    const unsigned nc = p.n <= kSortAlone ? 1 : kSortCluster;
    attr.val.clusterDim.x = nc;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(nc);
    c.blockDim = dim3(kSortThreads);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    c.attrs = &attr;
    c.numAttrs = 1;
    cudaGetLastError();
    return cudaLaunchKernelEx(&c, embed_sort_kernel<I>, p);
}

int64_t row_bytes(const lc_rows* r) { return r->stride * elem_size(r->dtype); }

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" lc_status lc_embed(int device, void* cuda_stream, const lc_rows* table, int64_t vocab, int64_t dim,
                              const void* ids, int32_t id_type, int64_t ntok, float scale, const lc_rows* y) {
    const char* call = "lc_embed";
    set_last_error("");
    if (vocab <= 0 || dim <= 0 || ntok < 0 || vocab > kMaxTokens || ntok > kMaxTokens || dim > kMaxTokens)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld tokens, %lld rows of %lld", call, (long long)ntok,
                           (long long)vocab, (long long)dim);
    if (id_type != LC_I32 && id_type != LC_I64)
        return fail_status(LC_ERR_INVALID_ARG, "%s: unknown id type %d", call, int(id_type));
    lc_status st = ops_check_rows(call, "table", table, vocab, dim, false);
    if (st == LC_OK) st = ops_check_rows(call, "y", y, ntok, dim, true);
    if (st != LC_OK) return st;
    if (y->dtype != table->dtype) return fail_status(LC_ERR_INVALID_ARG, "%s: y has another type than the table", call);
    const int isz = id_type == LC_I32 ? 4 : 8;
    if (reinterpret_cast<uintptr_t>(ids) % uintptr_t(isz))
        return fail_status(LC_ERR_INVALID_ARG, "%s: ids is not element-aligned", call);
    OnDevice cur(device);
    const Span2 spans[] = {span_of("table", table, vocab, dim, false), {"ids", ids, 1, ntok * isz, 0, false},
                           span_of("y", y, ntok, dim, true)};
    st = ops_check(call, device, spans, 3);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    if (ntok == 0) return LC_OK;
    EmbedParams p{};
    p.table = static_cast<const uint8_t*>(table->data);
    p.ids = ids;
    p.y = static_cast<uint8_t*>(y->data);
    p.vocab = vocab;
    p.dim = dim;
    p.table_pitch = row_bytes(table);
    p.y_pitch = row_bytes(y);
    p.ntok = ntok;
    p.scale = scale;
    const int sms = ops_sm_count(device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool bf = table->dtype == LC_BF16, i32 = id_type == LC_I32;
    const cudaError_t e = bf ? (i32 ? launch_embed<__nv_bfloat16, int32_t>(p, sms, s) : launch_embed<__nv_bfloat16, int64_t>(p, sms, s))
                             : (i32 ? launch_embed<float, int32_t>(p, sms, s) : launch_embed<float, int64_t>(p, sms, s));
    return ops_launched(call, e);
}

extern "C" uint64_t lc_embed_grad_workspace(int64_t ntok, int64_t vocab, int64_t dim) {
    if (ntok <= 0 || vocab <= 0 || dim <= 0 || ntok > kMaxTokens || vocab > kMaxTokens || dim > kMaxTokens) return 0;
    int64_t floats = 0;
    for (int E = 4; E <= 8; E += 4) {
        const int64_t f = sum_shape(ntok, dim, E).part_floats;
        floats = f > floats ? f : floats;
    }
    return grad_layout(ntok, vocab, floats).bytes;
}

extern "C" lc_status lc_embed_grad(int device, void* cuda_stream, const lc_rows* dy, const void* ids, int32_t id_type,
                                   int64_t ntok, float scale, int64_t skip_id, const lc_rows* grad, int64_t vocab,
                                   int64_t dim, int32_t accumulate, void* workspace, uint64_t workspace_bytes) {
    const char* call = "lc_embed_grad";
    set_last_error("");
    if (vocab <= 0 || dim <= 0 || ntok < 0 || vocab > kMaxTokens - 2 || ntok > kMaxTokens - 2 || dim > kMaxTokens)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld tokens, %lld rows of %lld", call, (long long)ntok,
                           (long long)vocab, (long long)dim);
    if (id_type != LC_I32 && id_type != LC_I64)
        return fail_status(LC_ERR_INVALID_ARG, "%s: unknown id type %d", call, int(id_type));
    lc_status st = ops_check_rows(call, "dy", dy, ntok, dim, false);
    if (st == LC_OK) st = ops_check_rows(call, "grad", grad, vocab, dim, true);
    if (st != LC_OK) return st;
    const int isz = id_type == LC_I32 ? 4 : 8;
    if (reinterpret_cast<uintptr_t>(ids) % uintptr_t(isz))
        return fail_status(LC_ERR_INVALID_ARG, "%s: ids is not element-aligned", call);
    const uint64_t need = lc_embed_grad_workspace(ntok, vocab, dim);
    if (workspace_bytes < need)
        return fail_status(LC_ERR_CAPACITY, "%s: %llu bytes of workspace, %llu needed", call,
                           (unsigned long long)workspace_bytes, (unsigned long long)need);
    if (reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail_status(LC_ERR_INVALID_ARG, "%s: the workspace is not 256-byte aligned", call);
    OnDevice cur(device);
    const Span2 spans[] = {span_of("dy", dy, ntok, dim, false), {"ids", ids, 1, ntok * isz, 0, false},
                           span_of("grad", grad, vocab, dim, true), {"workspace", workspace, 1, int64_t(need), 0, true}};
    st = ops_check(call, device, spans, 4);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const int64_t gp = row_bytes(grad);
    if (ntok == 0) {
        if (accumulate) return LC_OK;
        const size_t width = size_t(dim * elem_size(grad->dtype));
        cudaGetLastError();
        return ops_launched(call, vocab == 1 || size_t(gp) == width
                                      ? cudaMemsetAsync(grad->data, 0, width * size_t(vocab), s)
                                      : cudaMemset2DAsync(grad->data, size_t(gp), 0, width, size_t(vocab), s));
    }
    int bits = 1;
    while (int64_t(1) << bits <= vocab) ++bits;   // keys go up to vocab
    const bool vec = aligned16(dy->data) && aligned16(grad->data) && row_bytes(dy) % 16 == 0 && gp % 16 == 0;
    const bool dbf = dy->dtype == LC_BF16, gbf = grad->dtype == LC_BF16;
    const SumShape sh = sum_shape(ntok, dim, vec && dbf ? 8 : 4);
    const GradLayout l = grad_layout(ntok, vocab, sh.part_floats);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    SortParams q{};
    q.ids = ids;
    q.n = ntok;
    q.vocab = vocab;
    q.skip = skip_id;
    for (int i = 0; i < 2; ++i) {
        q.key[i] = reinterpret_cast<uint32_t*>(ws + l.key[i]);
        q.pos[i] = reinterpret_cast<uint32_t*>(ws + l.pos[i]);
    }
    q.present = accumulate ? nullptr : reinterpret_cast<uint32_t*>(ws + l.present);
    q.passes = (bits + kSortBits - 1) / kSortBits;
    q.digit = (bits + q.passes - 1) / q.passes;
    cudaError_t e = id_type == LC_I32 ? launch_sort<int32_t>(q, s) : launch_sort<int64_t>(q, s);
    if (e != cudaSuccess) return ops_launched(call, e);
    SumParams p{};
    p.key = q.key[(q.passes - 1) & 1];
    p.pos = q.pos[(q.passes - 1) & 1];
    p.present = q.present;
    p.dy = static_cast<const uint8_t*>(dy->data);
    p.grad = static_cast<uint8_t*>(grad->data);
    p.part = reinterpret_cast<float*>(ws + l.part);
    p.n = ntok;
    p.vocab = vocab;
    p.dim = dim;
    p.dy_pitch = row_bytes(dy);
    p.grad_pitch = gp;
    p.scale = scale;
    p.accumulate = accumulate != 0;
    using B = __nv_bfloat16;
    if (vec)
        e = dbf ? (gbf ? launch_sum<B, B, true>(p, sh, s) : launch_sum<B, float, true>(p, sh, s))
                : (gbf ? launch_sum<float, B, true>(p, sh, s) : launch_sum<float, float, true>(p, sh, s));
    else
        e = dbf ? (gbf ? launch_sum<B, B, false>(p, sh, s) : launch_sum<B, float, false>(p, sh, s))
                : (gbf ? launch_sum<float, B, false>(p, sh, s) : launch_sum<float, float, false>(p, sh, s));
    return ops_launched(call, e);
}
