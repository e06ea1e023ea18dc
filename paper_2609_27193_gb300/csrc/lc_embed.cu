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
// floating point atomics: the order of every sum is fixed by the sizes, the types and
// whether rows start on 16-byte boundaries.  The gradient is zeroed by the multiprocessors
// that the sort leaves idle: the rows with a token are written twice, which costs less
// than knowing first which they are.
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
constexpr int64_t kSortPer = 512;            // tokens of a CTA before the cluster grows
constexpr int64_t kSortShared = 65536;       // up to this many tokens the list stays in shared memory
constexpr int kSumThreads = 128;
constexpr int64_t kFew = 64;                 // up to this many tokens one kernel does without a sort
constexpr int64_t kMaxTokens = int64_t(1) << 31;

struct EmbedParams {
    const uint8_t* table;
    const void* ids;
    uint8_t* y;
    int64_t vocab, dim, table_pitch, y_pitch, ntok;   // pitches in bytes
    int64_t items, segs;                              // items = ntok * segs (segments of a row)
    float scale;
};

template <int B>
struct Word;
template <>
struct Word<16> { using type = uint4; };
template <>
struct Word<8> { using type = uint2; };
template <>
struct Word<4> { using type = uint32_t; };
template <>
struct Word<2> { using type = uint16_t; };

// B bytes an access, the most that the addresses and pitches are multiples of.
template <typename T, typename I, int B, int U>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(EmbedParams p) {
    using W = typename Word<B>::type;
    constexpr int V = B / int(sizeof(T));
    const int lane = threadIdx.x & 31;
    const int64_t step = int64_t(gridDim.x) * (kEmbedThreads / 32);
    for (int64_t item = int64_t(blockIdx.x) * (kEmbedThreads / 32) + (threadIdx.x >> 5); item < p.items; item += step) {
        int64_t t, seg;
        split_item(item, p.segs, t, seg);
        const int64_t c0 = seg * (32 * V * U) + lane * V;
        const int64_t id = int64_t(static_cast<const I*>(p.ids)[t]);
        const bool row = id >= 0 && id < p.vocab;
        const T* src = reinterpret_cast<const T*>(p.table + (row ? id : 0) * p.table_pitch);
        T* dst = reinterpret_cast<T*>(p.y + t * p.y_pitch);
        const float fill = id < 0 ? 0.0f : __uint_as_float(0x7fffffffu);
        W v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + u * 32 * V;
            if (row && c + V <= p.dim) v[u] = __ldg(reinterpret_cast<const W*>(src + c));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + u * 32 * V;
            if (c + V <= p.dim) {
                T e[V];
                memcpy(e, &v[u], B);
#pragma unroll
                for (int i = 0; i < V; ++i) e[i] = from_f32<T>(row ? to_f32(e[i]) * p.scale : fill);
                W out;
                memcpy(&out, e, B);
                __stcs(reinterpret_cast<W*>(dst + c), out);
            } else {
                for (int64_t k = c; k < p.dim; ++k) dst[k] = from_f32<T>(row ? to_f32(src[k]) * p.scale : fill);
            }
        }
    }
}

template <typename T, typename I, int B, int U>
cudaError_t launch_embed_bytes(EmbedParams p, int sms, cudaStream_t s) {
    constexpr int64_t per = 32 * (B / int(sizeof(T))) * U;
    p.segs = (p.dim + per - 1) / per;
    p.items = p.ntok * p.segs;
    const int64_t want = (p.items + kEmbedThreads / 32 - 1) / (kEmbedThreads / 32);
    const int64_t most = int64_t(sms) * 256;
    cudaGetLastError();
    embed_kernel<T, I, B, U><<<unsigned(want < most ? want : most), kEmbedThreads, 0, s>>>(p);
    return cudaGetLastError();
}

// Accesses of 16 bytes where addresses and pitches allow them, else of 8, 4 or one
// element (8192 tokens, 32000 rows, bf16: 2048 wide 7.2 us, 2044 8.2, 2046 11.1, 2047 16.4).
template <typename T, typename I>
cudaError_t launch_embed(const EmbedParams& p, int sms, cudaStream_t s) {
    const uintptr_t all = reinterpret_cast<uintptr_t>(p.table) | reinterpret_cast<uintptr_t>(p.y) | uintptr_t(p.table_pitch) |
                          uintptr_t(p.y_pitch);
    if (all % 16 == 0) return launch_embed_bytes<T, I, 16, 4>(p, sms, s);
    if (all % 8 == 0) return launch_embed_bytes<T, I, 8, 8>(p, sms, s);
    if (all % 4 == 0) return launch_embed_bytes<T, I, 4, 8>(p, sms, s);
    return launch_embed_bytes<T, I, sizeof(T), 8>(p, sms, s);
}

// --- the gradient -----------------------------------------------------------

struct SortParams {
    const void* ids;
    int64_t n, vocab, skip;
    uint2* list[2];        // (id, position); [1]: sorted; [0]: between passes (lists that do not stay in shared memory)
    uint8_t* grad;         // zeroed by the CTAs behind the sorting cluster (null: not wanted)
    int64_t rows, width, pitch;   // of grad, in bytes
    int32_t digit, passes; // bits of a digit, digits
    int64_t cap;           // places of a CTA in the list, a multiple of 1024 (SHARED: 1 << cap_log2)
    int32_t cap_log2;
};

// Bytes [from, to) of one row, by the CTA's threads.
__device__ __forceinline__ void zero_span(uint8_t* from, uint8_t* to) {
    uint8_t* v0 = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(from) + 15) & ~uintptr_t(15));
    uint8_t* v1 = reinterpret_cast<uint8_t*>(reinterpret_cast<uintptr_t>(to) & ~uintptr_t(15));
    if (v0 > v1) v0 = v1 = to;
    // elements have 2 or 4 bytes: the ends are whole pairs of bytes
    for (uint8_t* e = from + threadIdx.x * 2; e < v0; e += kSortThreads * 2) *reinterpret_cast<uint16_t*>(e) = 0;
    for (uint8_t* e = v1 + threadIdx.x * 2; e < to; e += kSortThreads * 2) *reinterpret_cast<uint16_t*>(e) = 0;
#pragma unroll 4
    for (uint8_t* v = v0 + threadIdx.x * 16; v < v1; v += kSortThreads * 16) st_stream(v, make_uint4(0, 0, 0, 0));
}
// Share `cta` of `ctas` of the gradient: every ctas-th piece of kZeroPiece bytes where
// rows lie back to back, else every ctas-th row.
constexpr int64_t kZeroPiece = 16 * kSortThreads;
__device__ __forceinline__ void zero_rows(uint8_t* grad, int64_t rows, int64_t width, int64_t pitch, int cta, int ctas) {
    if (pitch == width || rows == 1) {
        const int64_t total = rows * width, head = int64_t(-reinterpret_cast<uintptr_t>(grad) & 15);
        const int64_t pieces = total > head ? (total - head) / kZeroPiece : 0;
        uint8_t* v = grad + head + threadIdx.x * 16;
#pragma unroll 4
        for (int64_t i = cta; i < pieces; i += ctas) st_stream(v + i * kZeroPiece, make_uint4(0, 0, 0, 0));
        if (cta == 0) {
            zero_span(grad, grad + (head < total ? head : total));
            if (total > head) zero_span(grad + head + pieces * kZeroPiece, grad + total);
        }
        return;
    }
    for (int64_t r = cta; r < rows; r += ctas) zero_span(grad + r * pitch, grad + r * pitch + width);
}

// Sorts the tokens by id: least significant digit first, each pass a stable
// counting sort.  One cluster does it all: every warp owns a contiguous range of
// the list, counts its digits, the counts become offsets by sums over the warps, the
// cluster's CTAs (distributed shared memory) and the digits, and the warp hands its
// items out in order (lanes with the same digit find one another by match).  Tokens
// that contribute nothing get the key `vocab` and end up last.
//   SHARED: between passes an item goes straight to its next place in the shared
// memory of the CTA that has it there; a list in global memory costs a trip there
// and a fence of the whole cluster a pass (16381 tokens: 18 us that way, 13 so).
template <typename I, bool SHARED>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(SortParams p) {
    extern __shared__ uint32_t sm[];           // counts [warps][digit values], then (SHARED) lists [2][cap]
    __shared__ uint32_t tot[1 << kSortBits];
    __shared__ uint32_t warp_sum[kSortWarps];
    dependents_may_start();
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = int(cluster.block_rank()), nc = int(cluster.num_blocks());
    if (int(blockIdx.x) >= nc) {
        zero_rows(p.grad, p.rows, p.width, p.pitch, int(blockIdx.x) - nc, int(gridDim.x) - nc);
        return;
    }
    auto meet = [&]() {
        if (nc == 1) __syncthreads();
        else cluster.sync();
    };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bins = 1 << p.digit;
    uint32_t* cnt = sm + warp * bins;
    const int64_t cap = p.cap;
    uint2* list = reinterpret_cast<uint2*>(sm + kSortWarps * bins);
    const int64_t c0 = rank * cap, per = cap / kSortWarps;
    int64_t lo = c0 + warp * per;
    lo = lo < p.n ? lo : p.n;
    const int64_t hi = lo + per < p.n ? lo + per : p.n;
    constexpr int U = 4;                       // items of a lane that are asked for at once
    const bool once = hi - lo <= 32 * U;       // all of the warp's items: they stay in registers
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * p.digit;
        const bool last = pass == p.passes - 1;
        // the list that this pass reads; the one it writes is the other, the last one's always [1]
        const int to_list = (p.passes - pass) & 1, from = to_list ^ 1;
        // (an index into the parameters' arrays would put them on the stack)
        const uint2* far_from = from ? p.list[1] : p.list[0];
        uint2* far_to = from ? p.list[0] : p.list[1];
        uint32_t key[U], pos[U];
        auto load = [&](int64_t at) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = at + u * 32 + lane;
                key[u] = pos[u] = 0;
                if (i >= hi) continue;
                if (pass == 0) {
                    const int64_t id = int64_t(static_cast<const I*>(p.ids)[i]);
                    key[u] = uint32_t(id >= 0 && id < p.vocab && id != p.skip ? id : p.vocab);
                    pos[u] = uint32_t(i);
                } else if constexpr (SHARED) {
                    const uint2 v = list[from * cap + (i - c0)];
                    key[u] = v.x;
                    pos[u] = v.y;
                } else {
                    const uint2 v = __ldcg(far_from + i);
                    key[u] = v.x;
                    pos[u] = v.y;
                }
            }
        };
        for (int b = lane; b < bins; b += 32) cnt[b] = 0;
        __syncwarp();
        for (int64_t at = lo; at < hi; at += 32 * U) {
            load(at);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at + u * 32 + lane < hi) atomicAdd(cnt + ((key[u] >> shift) & uint32_t(bins - 1)), 1u);
        }
        __syncthreads();
        // a thread a digit value (bins <= kSortThreads): its counts over the warps
        const bool mine = int(threadIdx.x) < bins;
        if (mine) {
            uint32_t sum = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) sum += sm[w * bins + threadIdx.x];
            tot[threadIdx.x] = sum;
        }
        meet();
        uint32_t before = 0, all = 0;
        if (mine) {
            uint32_t other[kSortCluster];
#pragma unroll
            for (int r = 0; r < kSortCluster; ++r) other[r] = r < nc ? cluster.map_shared_rank(tot, r)[threadIdx.x] : 0;
#pragma unroll
            for (int r = 0; r < kSortCluster; ++r) {
                if (r < rank) before += other[r];
                all += other[r];
            }
        }
        uint32_t scan = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        uint32_t lower = lane < warp ? warp_sum[lane] : 0;       // the warps with smaller digit values
#pragma unroll
        for (int o = 16; o; o >>= 1) lower += __shfl_xor_sync(0xffffffffu, lower, o);
        if (mine) {
            uint32_t base = before + scan - all + lower;
            // 8 at a time: more would not stay in registers, and local memory is far away here
#pragma unroll 1
            for (int w = 0; w < kSortWarps; w += 8) {
                uint32_t c[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) c[k] = sm[(w + k) * bins + threadIdx.x];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    sm[(w + k) * bins + threadIdx.x] = base;
                    base += c[k];
                }
            }
        }
        __syncthreads();
        for (int64_t at = lo; at < hi; at += 32 * U) {
            if (!once) load(at);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (at + u * 32 >= hi) break;
                const bool in = at + u * 32 + lane < hi;
                const uint32_t d = in ? (key[u] >> shift) & uint32_t(bins - 1) : ~0u;
                const uint32_t same = __match_any_sync(0xffffffffu, d);
                const int first = __ffs(same) - 1;
                uint32_t to = 0;
                if (in && lane == first) to = atomicAdd(cnt + d, uint32_t(__popc(same)));
                __syncwarp();   // the next items' atomics come after these
                to = __shfl_sync(0xffffffffu, to, first) + __popc(same & ((1u << lane) - 1));
                if (!in) continue;
                if (last || !SHARED) {
                    far_to[to] = make_uint2(key[u], pos[u]);
                } else {
                    uint2* there = cluster.map_shared_rank(list, int(to >> p.cap_log2));
                    there[to_list * cap + (to & uint32_t(cap - 1))] = make_uint2(key[u], pos[u]);
                }
            }
        }
        // the next pass reads what this one wrote; after the last, no CTA leaves while another reads its totals
        meet();
    }
}

struct SumParams {
    const uint2* list;    // (id, position), sorted by id
    const uint8_t* dy;
    uint8_t* grad;
    float* part;          // [chunks][2][slabs][G][E]: a chunk's open rows at its start and end
    int64_t n, vocab, dim, dy_pitch, grad_pitch;
    int64_t chunk, chunks, slabs, items;   // items = chunks * slabs
    float scale;
    int32_t accumulate;
};

// The columns of a thread of a group of G: E consecutive ones (16-byte loads of dy),
// or E that lie G apart (single elements).
template <typename TD, bool VEC, int G>
struct Columns {
    static constexpr int E = VEC ? kVec<TD> : 4;
    int64_t c0;
    int64_t dim;
    __device__ Columns(int64_t slab, int64_t d) : c0(slab * G * E + int(threadIdx.x) % G * (VEC ? E : 1)), dim(d) {}
    __device__ int64_t col(int e) const { return VEC ? c0 + e : c0 + int64_t(e) * G; }
    __device__ bool whole() const { return VEC && c0 + E <= dim; }
    // A row's part as it lies in memory, and its values: all rows of a batch are asked for before one is unpacked.
    struct Raw {
        uint4 v;
        TD e[VEC ? 1 : E];
    };
    __device__ __forceinline__ void load(const uint8_t* row, Raw& raw) const {
        const TD* r = reinterpret_cast<const TD*>(row);
        if constexpr (VEC) {
            if (whole()) raw.v = ld_stream(r + c0);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (col(e) < dim) raw.e[e] = r[col(e)];
        }
    }
    __device__ __forceinline__ void add(const uint8_t* row, const Raw& raw, float (&acc)[E]) const {
        if constexpr (VEC) {
            if (whole()) {
                float f[E];
                unpack(raw.v, f);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += f[e];
            } else {
                const TD* r = reinterpret_cast<const TD*>(row);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col(e) < dim) acc[e] += to_f32(r[col(e)]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (col(e) < dim) acc[e] += to_f32(raw.e[e]);
        }
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

template <int G, int E>
__device__ __forceinline__ int64_t part_at(const SumParams& p, int64_t chunk, int which, int64_t slab) {
    return (((chunk * 2 + which) * p.slabs + slab) * G + int(threadIdx.x) % G) * E;
}

// A group of G threads sums one chunk of the sorted list in G * E columns.
template <typename TD, typename TG, bool VEC, int G>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(SumParams p) {
    using Cols = Columns<TD, VEC, G>;
    constexpr int E = Cols::E;
    constexpr int U = 8;   // rows in flight
    dependency_wait();
    dependents_may_start();
    const int lane = threadIdx.x & 31;
    const int64_t item = int64_t(blockIdx.x) * (kSumThreads / G) + int(threadIdx.x) / G;
    if (item >= p.items) return;
    int64_t chunk, slab;
    split_item(item, p.slabs, chunk, slab);
    const Cols cols(slab, p.dim);
    const int64_t s0 = chunk * p.chunk;
    const int64_t s1 = s0 + p.chunk < p.n ? s0 + p.chunk : p.n;
    const uint32_t none = uint32_t(p.vocab);
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    // 32 entries of the list at a time, one a lane; the next ones are asked for early
    auto entry = [&](int64_t s, uint32_t& key, uint32_t& pos) {
        const uint2 v = s < p.n && s <= s1 ? p.list[s] : make_uint2(none, 0);
        key = v.x;
        pos = v.y;
    };
    uint32_t key_next, pos_next;
    entry(s0 + lane, key_next, pos_next);
    const uint32_t before = s0 > 0 ? p.list[s0 - 1].x : none;
    bool open = __shfl_sync(0xffffffffu, key_next, 0) == before;   // the row began in an earlier chunk
    for (int64_t base = s0; base < s1; base += 32) {
        const uint32_t key32 = key_next, pos32 = pos_next;
        if (__shfl_sync(0xffffffffu, key32, 0) == none) break;     // sorted last: nothing more contributes
        entry(base + 32 + lane, key_next, pos_next);
        const uint32_t after = __shfl_sync(0xffffffffu, key_next, 0);
#pragma unroll 1
        for (int part = 0; part < 32; part += U) {
            if (base + part >= s1) break;
            typename Cols::Raw raw[U];
            uint32_t k[U + 1], at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                k[u] = __shfl_sync(0xffffffffu, key32, part + u);
                at[u] = __shfl_sync(0xffffffffu, pos32, part + u);
                if (base + part + u < s1 && k[u] != none) cols.load(p.dy + int64_t(at[u]) * p.dy_pitch, raw[u]);
            }
            k[U] = part + U < 32 ? __shfl_sync(0xffffffffu, key32, (part + U) & 31) : after;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (base + part + u >= s1 || k[u] == none) break;
                cols.add(p.dy + int64_t(at[u]) * p.dy_pitch, raw[u], acc);
                const bool last = base + part + u + 1 >= s1;
                const uint32_t next = k[u + 1];
                if (next == k[u] && !last) continue;
                if (open || next == k[u]) {
                    float* out = p.part + part_at<G, E>(p, chunk, open ? 0 : 1, slab);
#pragma unroll
                    for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(out + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
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
}

// Rows that cross chunks.  The CTA of the chunk in which such a row begins adds its
// parts: its groups take equal runs of them, and the groups' sums are added in order.
constexpr int kJoinThreads = 512;
template <typename TD, typename TG, bool VEC, int G>
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(SumParams p) {
    using Cols = Columns<TD, VEC, G>;
    constexpr int E = Cols::E, R = kJoinThreads / G;
    constexpr int U = 8;
    __shared__ float4 sums[kJoinThreads][E / 4];
    dependency_wait();
    int64_t chunk, slab;
    split_item(blockIdx.x, p.slabs, chunk, slab);
    const int64_t s0 = chunk * p.chunk, s1 = s0 + p.chunk;
    if (s1 >= p.n) return;
    const uint32_t key = p.list[s1].x, last = p.list[s1 - 1].x, before = s0 > 0 ? p.list[s0 - 1].x : uint32_t(p.vocab);
    if (key == uint32_t(p.vocab) || last != key) return;   // no row crosses this chunk's end
    if (s0 > 0 && before == key) return;                   // it began in an earlier chunk
    // chunks c in (chunk, lo] begin with this row: the largest one, by a search that looks at 32 places at a time,
    // first the next ones
    const int lane = threadIdx.x & 31;
    int64_t lo = chunk + 1, hi = p.chunks;                 // key[lo * chunk] == key, hi: beyond
    for (bool near = true; hi - lo > 1; near = false) {
        const int64_t gap = near ? 1 : (hi - lo + 31) / 32, c = lo + gap * (lane + 1);
        const uint32_t same = __ballot_sync(0xffffffffu, c < hi && p.list[c * p.chunk].x == key);
        const int64_t n = __popc(same);                    // sorted: the first n of them
        const int64_t top = lo + gap * (n + 1);
        lo += gap * n;
        if (n < 32 && top < hi) hi = top;
    }
    const int64_t stride = p.slabs * 2 * G * E;
    const int group = threadIdx.x / G;
    const int64_t m = lo - chunk + 1;                      // parts: the chunk's last row, then the others' first
    const int64_t per = (m + R - 1) / R;
    const int64_t i0 = group * per < m ? group * per : m, i1 = i0 + per < m ? i0 + per : m;
    const float* first = p.part + part_at<G, E>(p, chunk, 1, slab);
    const float* rest = p.part + part_at<G, E>(p, chunk, 0, slab);
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    for (int64_t i = i0; i < i1; i += U) {
        float4 f[U][E / 4];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E / 4; ++e)
                f[u][e] = i + u < i1 ? reinterpret_cast<const float4*>(i + u ? rest + (i + u) * stride : first)[e]
                                     : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E / 4; ++e) {
                acc[4 * e] += f[u][e].x;
                acc[4 * e + 1] += f[u][e].y;
                acc[4 * e + 2] += f[u][e].z;
                acc[4 * e + 3] += f[u][e].w;
            }
    }
#pragma unroll
    for (int e = 0; e < E / 4; ++e) sums[threadIdx.x][e] = make_float4(acc[4 * e], acc[4 * e + 1], acc[4 * e + 2], acc[4 * e + 3]);
    __syncthreads();
    if (group) return;
    for (int g = 1; g < R && g * per < m; ++g)
#pragma unroll
        for (int e = 0; e < E / 4; ++e) {
            const float4 f = sums[g * G + threadIdx.x][e];
            acc[4 * e] += f.x;
            acc[4 * e + 1] += f.y;
            acc[4 * e + 2] += f.z;
            acc[4 * e + 3] += f.w;
        }
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= p.scale;
    const Cols cols(slab, p.dim);
    cols.template store<TG>(p.grad + int64_t(key) * p.grad_pitch, acc, p.accumulate != 0);
}

// --- few tokens ---------------------------------------------------------------

struct FewParams {
    const void* ids;
    const uint8_t* dy;
    uint8_t* grad;
    int64_t vocab, skip, dim, dy_pitch, grad_pitch, slabs, sum_ctas, zero_rows;
    float scale;
    int32_t n, accumulate;
};

// Up to kFew tokens: every CTA has all ids in shared memory.  A group of threads takes
// a token and G * E columns; if it is the first with its id it adds up all of them,
// in order.  The CTAs behind these zero the rows that no id names.  One launch instead
// of three (24 tokens of 256 over 8000 rows: 3.7 us instead of 12; at most 8 batches of
// rows one after the other, where every token has the same id).
template <typename TD, typename TG, typename I, bool VEC, int G>
__global__ void __launch_bounds__(kSumThreads) embed_few_kernel(FewParams p) {
    using Cols = Columns<TD, VEC, G>;
    constexpr int E = Cols::E;
    constexpr int U = 8;
    __shared__ uint32_t keys[kFew];
    const uint32_t none = uint32_t(p.vocab);
    if (threadIdx.x < kFew) {
        uint32_t key = none;
        if (int(threadIdx.x) < p.n) {
            const int64_t id = int64_t(static_cast<const I*>(p.ids)[threadIdx.x]);
            if (id >= 0 && id < p.vocab && id != p.skip) key = uint32_t(id);
        }
        keys[threadIdx.x] = key;
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    if (int64_t(blockIdx.x) >= p.sum_ctas) {
        const int64_t r0 = (int64_t(blockIdx.x) - p.sum_ctas) * p.zero_rows;
        const int64_t r1 = r0 + p.zero_rows < p.vocab ? r0 + p.zero_rows : p.vocab;
        const int64_t width = p.dim * int64_t(sizeof(TG));
        const bool vectors = VEC && width % 16 == 0;
        const int warp = threadIdx.x >> 5;
        for (int64_t first = r0; first < r1; first += 32) {
            const int64_t mine = first + lane;
            bool named = false;
            for (int j = 0; j < p.n; ++j) named |= keys[j] == uint32_t(mine);
            uint32_t empty = __ballot_sync(0xffffffffu, mine < r1 && !named);
            if (vectors && width >= 2048) {
                // the CTA a row
                while (empty) {
                    uint8_t* row = p.grad + (first + __ffs(empty) - 1) * p.grad_pitch;
                    empty &= empty - 1;
                    for (int64_t i = threadIdx.x * 16; i < width; i += kSumThreads * 16) st_stream(row + i, make_uint4(0, 0, 0, 0));
                }
                continue;
            }
            // a warp a row
            for (int k = 0; empty; ++k) {
                uint8_t* row = p.grad + (first + __ffs(empty) - 1) * p.grad_pitch;
                empty &= empty - 1;
                if (k % (kSumThreads / 32) != warp) continue;
                if (vectors)
                    for (int64_t i = lane * 16; i < width; i += 512) st_stream(row + i, make_uint4(0, 0, 0, 0));
                else
                    for (int64_t i = lane; i < p.dim; i += 32) reinterpret_cast<TG*>(row)[i] = from_f32<TG>(0.0f);
            }
        }
        return;
    }
    const int64_t item = int64_t(blockIdx.x) * (kSumThreads / G) + int(threadIdx.x) / G;
    const int64_t t = item / p.slabs, slab = item - t * p.slabs;
    if (t >= p.n) return;
    const uint32_t key = keys[t];
    if (key == none) return;
    // the tokens with this id (keys beyond n are `none`)
    uint64_t same = __ballot_sync(0xffffffffu, keys[lane] == key) | uint64_t(__ballot_sync(0xffffffffu, keys[lane + 32] == key)) << 32;
    if (__ffsll((long long)same) - 1 != t) return;
    const Cols cols(slab, p.dim);
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    while (same) {
        typename Cols::Raw raw[U];
        int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at[u] = __ffsll((long long)same) - 1;   // -1: none left
            same &= same - 1;
            if (at[u] >= 0) cols.load(p.dy + at[u] * p.dy_pitch, raw[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at[u] >= 0) cols.add(p.dy + at[u] * p.dy_pitch, raw[u], acc);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= p.scale;
    cols.template store<TG>(p.grad + int64_t(key) * p.grad_pitch, acc, p.accumulate != 0);
}

template <typename TD, typename TG, typename I, bool VEC, int G>
cudaError_t launch_few_group(FewParams p, cudaStream_t s) {
    constexpr int E = Columns<TD, VEC, G>::E;
    p.slabs = (p.dim + G * E - 1) / (G * E);
    p.sum_ctas = (p.n * p.slabs + kSumThreads / G - 1) / (kSumThreads / G);
    int64_t zero = 0;
    if (!p.accumulate) {
        // 16 KB a CTA
        p.zero_rows = 16384 / (p.dim * int64_t(sizeof(TG)));
        p.zero_rows = p.zero_rows < 1 ? 1 : p.zero_rows > 32 ? p.zero_rows / 32 * 32 : p.zero_rows;
        zero = (p.vocab + p.zero_rows - 1) / p.zero_rows;
    }
    if (p.sum_ctas + zero > 0x7fffffff) return cudaErrorInvalidValue;
    cudaGetLastError();
    embed_few_kernel<TD, TG, I, VEC, G><<<unsigned(p.sum_ctas + zero), kSumThreads, 0, s>>>(p);
    return cudaGetLastError();
}
template <typename TD, typename TG, typename I>
cudaError_t launch_few(const FewParams& p, bool vec, cudaStream_t s) {
    if (!vec) return launch_few_group<TD, TG, I, false, kSumThreads>(p, s);
    return p.dim <= 32 * kVec<TD> ? launch_few_group<TD, TG, I, true, 32>(p, s) : launch_few_group<TD, TG, I, true, kSumThreads>(p, s);
}
template <typename TD, typename TG>
cudaError_t launch_few(const FewParams& p, bool vec, bool i32, cudaStream_t s) {
    return i32 ? launch_few<TD, TG, int32_t>(p, vec, s) : launch_few<TD, TG, int64_t>(p, vec, s);
}

constexpr size_t al256(size_t x) { return (x + 255) & ~size_t(255); }

// Chunks of the sorted list: whole batches of 8 rows, long enough to fill the device
// a few times over, and beyond that no more than 512 of them for groups of 128
// threads, 2048 for groups of 32, so that a row which all tokens share is joined from
// no more parts than that (a join has as many more groups as they are smaller).
// 16381 x 768: 35 us; with twice as many 38, with half as many 40.
int64_t chunk_of(int64_t n, int64_t slabs, int64_t group) {
    int64_t c = n * slabs / 4864;
    if (c < n * group / 65536) c = n * group / 65536;
    c = (c + 7) / 8 * 8;
    return c < 8 ? 8 : c;
}

struct GradLayout {
    size_t list[2], part, bytes;
};
// E: the columns of a thread; more of them are more partial sums a chunk.
GradLayout grad_layout(int64_t n, int64_t part_floats) {
    GradLayout l{};
    size_t at = 0;
    for (int i = 0; i < 2; ++i) {
        l.list[i] = at;
        at += al256(size_t(n) * 8);
    }
    l.part = at;
    l.bytes = at + al256(size_t(part_floats) * 4);
    return l;
}

// The group of threads that takes a chunk: as many as a row's columns need, up to
// kSumThreads; wider rows are cut into slabs.
struct SumShape {
    int64_t group, slabs, chunk, chunks, part_floats;
};
SumShape sum_shape(int64_t n, int64_t dim, int E) {
    SumShape s;
    s.group = dim <= 32 * E ? 32 : dim <= 64 * E ? 64 : kSumThreads;
    s.slabs = (dim + s.group * E - 1) / (s.group * E);
    s.chunk = chunk_of(n, s.slabs, s.group);
    s.chunks = (n + s.chunk - 1) / s.chunk;
    s.part_floats = s.chunks * 2 * s.slabs * s.group * E;
    return s;
}

template <typename TD, typename TG, bool VEC, int G>
cudaError_t launch_group(SumParams p, cudaStream_t s) {
    const int64_t grid = (p.items + kSumThreads / G - 1) / (kSumThreads / G);
    cudaError_t e = launch_dependent(embed_sum_kernel<TD, TG, VEC, G>, int(grid), kSumThreads, 0, s, p);
    if (e == cudaSuccess && p.chunks > 1)
        e = launch_dependent(embed_join_kernel<TD, TG, VEC, G>, int(p.items), kJoinThreads, 0, s, p);
    return e;
}

template <typename TD, typename TG, bool VEC>
cudaError_t launch_sum(SumParams p, const SumShape& sh, cudaStream_t s) {
    p.slabs = sh.slabs;
    p.chunk = sh.chunk;
    p.chunks = sh.chunks;
    p.items = sh.chunks * sh.slabs;
    if (sh.group == 32) return launch_group<TD, TG, VEC, 32>(p, s);
    if (sh.group == 64) return launch_group<TD, TG, VEC, 64>(p, s);
    return launch_group<TD, TG, VEC, kSumThreads>(p, s);
}

template <typename I, bool SHARED>
cudaError_t launch_sort(SortParams p, int sms, cudaStream_t s) {
    static bool ready[kOpsMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const size_t counts = size_t(kSortWarps) * 4;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(embed_sort_kernel<I, SHARED>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 int((counts << kSortBits) + (SHARED ? kSortShared / kSortCluster * 16 : 0)));
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    unsigned nc = 1;
    while (nc < kSortCluster && p.n > kSortPer * int64_t(nc)) nc *= 2;
    p.cap_log2 = 10;
    while (int64_t(nc) << p.cap_log2 < p.n) ++p.cap_log2;
    p.cap = SHARED ? int64_t(1) << p.cap_log2 : (p.n + nc * 1024 - 1) / (nc * 1024) * 1024;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = nc;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    // the other multiprocessors zero the gradient meanwhile, from 32 KB a CTA; 512 KB at most, since not every cluster
    // may find a place at once (1 GB in one CTA a multiprocessor: 229 us, with a second wave as long as the first)
    int64_t zero = 0;
    if (p.grad) {
        const int64_t bytes = p.rows * p.width, want = (bytes + 32767) / 32768, most = sms > int(nc) ? sms - int(nc) : 1;
        zero = want < most ? want : most;
        if (zero < bytes / 524288) zero = bytes / 524288;
        if (zero > 1 << 24) zero = 1 << 24;
        zero = (zero + nc - 1) / nc * nc;
    }
    c.gridDim = dim3(nc + unsigned(zero));
    c.blockDim = dim3(kSortThreads);
    c.dynamicSmemBytes = (counts << p.digit) + (SHARED ? size_t(16) << p.cap_log2 : 0);
    c.stream = s;
    c.attrs = &attr;
    c.numAttrs = 1;
    cudaGetLastError();
    return cudaLaunchKernelEx(&c, embed_sort_kernel<I, SHARED>, p);
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
    if (ntok <= kFew || vocab <= 0 || dim <= 0 || ntok > kMaxTokens || vocab > kMaxTokens || dim > kMaxTokens) return 0;
    int64_t floats = 0;
    for (int E = 4; E <= 8; E += 4) {
        const int64_t f = sum_shape(ntok, dim, E).part_floats;
        floats = f > floats ? f : floats;
    }
    return grad_layout(ntok, floats).bytes;
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
    using B = __nv_bfloat16;
    if (ntok <= kFew) {
        FewParams f{};
        f.ids = ids;
        f.dy = static_cast<const uint8_t*>(dy->data);
        f.grad = static_cast<uint8_t*>(grad->data);
        f.vocab = vocab;
        f.skip = skip_id;
        f.dim = dim;
        f.dy_pitch = row_bytes(dy);
        f.grad_pitch = gp;
        f.scale = scale;
        f.n = int32_t(ntok);
        f.accumulate = accumulate != 0;
        const bool i32 = id_type == LC_I32;
        return ops_launched(call, dbf ? (gbf ? launch_few<B, B>(f, vec, i32, s) : launch_few<B, float>(f, vec, i32, s))
                                      : (gbf ? launch_few<float, B>(f, vec, i32, s) : launch_few<float, float>(f, vec, i32, s)));
    }
    const SumShape sh = sum_shape(ntok, dim, vec && dbf ? 8 : 4);
    const GradLayout l = grad_layout(ntok, sh.part_floats);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    SortParams q{};
    q.ids = ids;
    q.n = ntok;
    q.vocab = vocab;
    q.skip = skip_id;
    for (int i = 0; i < 2; ++i) q.list[i] = reinterpret_cast<uint2*>(ws + l.list[i]);
    if (!accumulate) {
        q.grad = static_cast<uint8_t*>(grad->data);
        q.rows = vocab;
        q.width = dim * elem_size(grad->dtype);
        q.pitch = gp;
    }
    q.passes = (bits + kSortBits - 1) / kSortBits;
    q.digit = (bits + q.passes - 1) / q.passes;
    const int sms = ops_sm_count(device);
    cudaError_t e;
    if (ntok <= kSortShared) e = id_type == LC_I32 ? launch_sort<int32_t, true>(q, sms, s) : launch_sort<int64_t, true>(q, sms, s);
    else e = id_type == LC_I32 ? launch_sort<int32_t, false>(q, sms, s) : launch_sort<int64_t, false>(q, sms, s);
    if (e != cudaSuccess) return ops_launched(call, e);
    SumParams p{};
    p.list = q.list[1];
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
    if (vec)
        e = dbf ? (gbf ? launch_sum<B, B, true>(p, sh, s) : launch_sum<B, float, true>(p, sh, s))
                : (gbf ? launch_sum<float, B, true>(p, sh, s) : launch_sum<float, float, true>(p, sh, s));
    else
        e = dbf ? (gbf ? launch_sum<B, B, false>(p, sh, s) : launch_sum<B, float, false>(p, sh, s))
                : (gbf ? launch_sum<float, B, false>(p, sh, s) : launch_sum<float, float, false>(p, sh, s));
    return ops_launched(call, e);
}
