// Rows of a table by id, scaled, and the table's gradient.
//
//   forward:   out[m] = scale * table[ids[m]] + add[m]                      (negative id: no row)
//   backward:  dTable[v] = scale * sum of dOut[k] over the kept rows k with ids[k] = v
//
// The backward sums in a fixed order: the kept rows are sorted by id (a stable radix sort, so that rows of one id stay in
// ascending order), the sorted list is cut into equal pieces, and a piece adds up the rows of each id in it.  An id whose rows
// cross a piece's border leaves partial rows, which a last launch adds in the order of the pieces.  Nothing depends on how
// often an id occurs: the most frequent one is spread over as many pieces as its rows fill.
//
// Bound by memory, in the main by clearing dTable where few of its rows get a gradient (50257 x 768: 154 MB), and for small tables by
// latency.  Up to 131072 rows are sorted by one cluster of blocks in one launch, which exchange their digits' counts through
// distributed shared memory; the other blocks of that launch clear the table meanwhile, and the sums then write over the rows
// that have one.  (Four to six launches of separate counts and scatters: 31 us for 12544 rows and one digit.)  Longer lists take
// two launches a digit.  (At that border the cluster is behind already: 131072 rows into 50257 x 768 146 us, 131073 rows 107;
// 16384 rows 44, 600000 rows 265, floors 27 and 165.)
#include "row_copy.cuh"
#include "row_math.cuh"
#include "tc_ptx.cuh"

namespace sbp {
namespace {

// ---- forward ----
template <typename T, bool kAdd>
__global__ void __launch_bounds__(kCopyThreads)
embedding_forward_kernel(const uint4* __restrict__ table, const RowLength row, int64_t V, const int32_t* __restrict__ ids, int64_t M,
                         float scale, const uint4* add, uint4* out, const int32_t* status_word) {
    pdl_launch_dependents();
    pdl_wait();
    if (block_sees_error(status_word)) return;
    const int64_t begin = (int64_t)blockIdx.x * kCopySpan, total = M * row.n;
    const SpanRows span(begin, row);
    int64_t src[kCopyUnroll];
    uint4 v[kCopyUnroll], a[kCopyUnroll];
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        uint32_t q;
        const int64_t c = span.place(threadIdx.x + u * kCopyThreads, row, &q);
        src[u] = -1;
        if (begin + threadIdx.x + u * kCopyThreads < total) {
            const int64_t id = __ldg(ids + span.first + q);
            if (id >= 0 && id < V) src[u] = id * row.n + c;
        }
    }
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        const int64_t i = begin + threadIdx.x + u * kCopyThreads;
        v[u] = src[u] >= 0 ? __ldg(table + src[u]) : zero;
        if constexpr (kAdd) a[u] = i < total ? __ldcg(add + i) : zero;
    }
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
        const int64_t i = begin + threadIdx.x + u * kCopyThreads;
        if (i >= total) continue;
        constexpr int P = Vec<T>::N / 2;
        f32x2 f[P], g[P];
        Vec<T>::unpack(v[u], f);
        if constexpr (kAdd) Vec<T>::unpack(a[u], g);
        const f32x2 k = pair(scale, scale);
#pragma unroll
        for (int e = 0; e < P; ++e) f[e] = kAdd ? fma(k, f[e], g[e]) : mul(k, f[e]);
        out[i] = src[u] >= 0 ? Vec<T>::pack(f) : kAdd ? a[u] : zero;
    }
}

// Reports ids of V or more among those of the kept rows, as a call's last launch: the kernels before it look whether an earlier call
// left an error in the status word, and would stop at one of their own.  (Only with a status word; it adds 2 us to a call.)
__global__ void __launch_bounds__(256) embedding_report_kernel(const int32_t* ids, const int32_t* keep_rows, const int32_t* M_keep_dev, int64_t M,
                                                               int64_t M_keep_cap, int64_t V, int32_t* status_word) {
    pdl_launch_dependents();
    pdl_wait();
    const int64_t n = load_m_keep(M_keep_dev, M_keep_cap);
    for (int64_t m = (int64_t)blockIdx.x * 256 + threadIdx.x; m < n; m += (int64_t)gridDim.x * 256) {
        const int32_t row = mapped_row(keep_rows, m);
        if (row >= 0 && row < M && __ldg(ids + row) >= V) report_device_error(status_word, SBP_ERR_BAD_INDICES);
    }
}
cudaError_t report_ids(const int32_t* ids, const int32_t* keep_rows, const int32_t* M_keep_dev, int64_t M, int64_t M_keep_cap, int64_t V,
                       int32_t* status_word, cudaStream_t stream) {
    if (status_word == nullptr || M_keep_cap == 0) return cudaSuccess;
    const int64_t blocks = (M_keep_cap + 255) / 256, most = 8 * kNumSMs;
    return launch_pdl(embedding_report_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream, ids, keep_rows, M_keep_dev,
                      M, M_keep_cap, V, status_word);
}

// ---- backward: the sort ----
constexpr int kSortThreads = 512, kSortItems = 8, kSortTile = kSortThreads * kSortItems, kSortWarps = kSortThreads / 32;
constexpr int kDigits = 256, kSortMaxBlocks = 128;
constexpr int kSortCluster = 8;
constexpr int64_t kSortClusterRows = 131072;          // four tiles a block of the cluster

struct SortParams {
    const int32_t *ids, *keep_rows, *M_keep_dev;
    int64_t M, M_keep_cap, V;
    int compact;                                      // dOut is packed: the source row is the place in the list
    uint32_t* keys[2];
    int32_t* rows[2];
    uint32_t* hist;                                   // [blocks][kDigits]
    int64_t span;                                     // rows of a block
    int blocks, passes, bits;                         // sorting blocks; digits of `bits` bits
    uint4* clear;                                     // dTable, or nullptr
    int64_t clear_vecs;
    const int32_t* status_word;
};

// Exclusive sums of one value a digit over the digits, by the first 256 threads; the others pass the barriers.
__device__ __forceinline__ uint32_t digit_scan(uint32_t v, uint32_t* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    if (lane == 31 && warp < kDigits / 32) warp_sums[warp] = s;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < kDigits / 32; ++w) before += w < warp ? warp_sums[w] : 0u;
    __syncthreads();
    return before + s - v;
}

struct SortShared {
    uint32_t base[kDigits];                           // where the next element of a digit goes
    alignas(128) uint32_t count[kSortWarps][kDigits];
    uint32_t warp_sums[kDigits / 32];
};

// Blocks behind the sorting ones clear `part` of `parts` of dTable: one thread copies zeros from shared memory, 16 KB at a time, three
// blocks an SM.  (12288 rows into 50257 x 768, the whole gradient as it was then: 41.4 us, 39.7 now; two blocks an SM 49.7; stores by
// all threads 46 to 48.)
__device__ __forceinline__ void clear_table(const SortParams& p, SortShared& sh, int part, int parts) {
    if (p.clear == nullptr || block_sees_error(p.status_word)) return;
    constexpr int64_t kPiece = sizeof(sh.count) / 16;
    const int64_t pieces = (p.clear_vecs + kPiece - 1) / kPiece, lo = pieces * part / parts, hi = pieces * (part + 1) / parts;
    for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) (&sh.count[0][0])[i] = 0u;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int64_t i = lo + ((int64_t)blockIdx.x - p.blocks); i < hi; i += (int64_t)gridDim.x - p.blocks) {
        const int64_t at = i * kPiece, n = p.clear_vecs - at < kPiece ? p.clear_vecs - at : kPiece;
        ptx::bulk_store(p.clear + at, ptx::smem_addr(&sh.count[0][0]), (uint32_t)n * 16u);
        ptx::bulk_commit();
    }
    ptx::bulk_wait_all();
}

// Counts of the digits of elements [begin, end), left in sh.base.  The first pass makes the keys: the id of the m-th kept row (V:
// none), and where its gradient is; a tile's loads are under way together.
__device__ __forceinline__ void count_digits(const SortParams& p, SortShared& sh, int64_t begin, int64_t end, int pass) {
    if (threadIdx.x < kDigits) sh.base[threadIdx.x] = 0u;
    __syncthreads();
    const uint32_t mask = (1u << p.bits) - 1u;
    for (int64_t tile = begin; tile < end; tile += kSortTile) {
        uint32_t key[kSortItems];
        if (pass == 0) {
            int32_t row[kSortItems], id[kSortItems];
#pragma unroll
            for (int i = 0; i < kSortItems; ++i) {
                const int64_t at = tile + threadIdx.x + i * kSortThreads;
                row[i] = at < end ? mapped_row(p.keep_rows, at) : -1;
            }
#pragma unroll
            for (int i = 0; i < kSortItems; ++i) id[i] = __ldg(p.ids + (row[i] >= 0 && row[i] < p.M ? row[i] : 0));
#pragma unroll
            for (int i = 0; i < kSortItems; ++i) {
                const int64_t at = tile + threadIdx.x + i * kSortThreads;
                const bool ok = row[i] >= 0 && row[i] < p.M;
                key[i] = ok && id[i] >= 0 && id[i] < p.V ? (uint32_t)id[i] : (uint32_t)p.V;
                if (at < end) {
                    p.keys[1][at] = key[i];
                    p.rows[1][at] = p.compact ? (int32_t)at : row[i];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kSortItems; ++i) {
                const int64_t at = tile + threadIdx.x + i * kSortThreads;
                key[i] = at < end ? __ldcg(p.keys[(pass + 1) & 1] + at) : 0u;
            }
        }
#pragma unroll
        for (int i = 0; i < kSortItems; ++i)
            if (tile + threadIdx.x + i * kSortThreads < end) atomicAdd(&sh.base[key[i] >> (pass * p.bits) & mask], 1u);
    }
    __syncthreads();
}

// Elements [begin, begin + kSortTile) of the list, below n: each goes to base[digit] plus the number of elements of its digit
// before it; base moves on.  Warp w has the w-th 256 elements, 32 at a time, so the order of the list is kept.
__device__ __forceinline__ void scatter_tile(const SortParams& p, SortShared& sh, int64_t begin, int64_t n, int pass) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t key[kSortItems], rank[kSortItems];
    int32_t row[kSortItems];
    const int shift = pass * p.bits;
    const uint32_t mask = (1u << p.bits) - 1u;
    const int64_t first = begin + warp * (32 * kSortItems) + lane;
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        const int64_t at = first + 32 * i;
        key[i] = at < n ? __ldcg(p.keys[(pass + 1) & 1] + at) : 0u;
        row[i] = at < n ? __ldcg(p.rows[(pass + 1) & 1] + at) : 0;
    }
    for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) (&sh.count[0][0])[i] = 0u;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        const bool live = first + 32 * i < n;
        const uint32_t d = key[i] >> shift & mask;
        uint32_t peers = __ballot_sync(0xffffffffu, live);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const uint32_t set = __ballot_sync(0xffffffffu, d >> b & 1u);
            peers &= (d >> b & 1u) ? set : ~set;
        }
        const uint32_t before = live ? sh.count[warp][d] : 0u;
        rank[i] = before + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
        if (live && (peers >> lane) == 1u) sh.count[warp][d] = before + __popc(peers);      // the last of them
        __syncwarp();
    }
    __syncthreads();
    if (threadIdx.x < kDigits) {                      // a warp's elements of a digit follow those of the warps before it
        uint32_t at = sh.base[threadIdx.x];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t c = sh.count[w][threadIdx.x];
            sh.count[w][threadIdx.x] = at;
            at += c;
        }
        sh.base[threadIdx.x] = at;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        if (first + 32 * i >= n) continue;
        const uint32_t to = sh.count[warp][key[i] >> shift & mask] + rank[i];
        p.keys[pass & 1][to] = key[i];
        p.rows[pass & 1][to] = row[i];
    }
    __syncthreads();
}

// The whole sort by the first cluster, which the others' clearing hides.  (The sorting blocks write to the workspace alone, and do so
// whatever the status word holds: the sums never see a list that is not sorted.)
__global__ void __launch_bounds__(kSortThreads) embedding_sort_kernel(const SortParams p) {
    __shared__ SortShared sh;
    __shared__ uint32_t counts[kSortCluster][kDigits];               // of every block of the cluster
    pdl_launch_dependents();
    pdl_wait();
    if (blockIdx.x >= (unsigned)p.blocks) return clear_table(p, sh, 0, 1);
    const int64_t n = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const uint32_t rank = ptx::cluster_ctarank();
    const int64_t begin = rank * p.span < n ? rank * p.span : n, end = begin + p.span < n ? begin + p.span : n;
    ptx::cluster_sync_all();                                         // every block has begun
    for (int pass = 0; pass < p.passes; ++pass) {
        count_digits(p, sh, begin, end, pass);
        if (threadIdx.x < kDigits)
            for (uint32_t b = 0; b < kSortCluster; ++b)
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ptx::map_to_cta(ptx::smem_addr(&counts[rank][threadIdx.x]), b)),
                             "r"(sh.base[threadIdx.x]) : "memory");
        ptx::cluster_sync_all();
        uint32_t all = 0u, before = 0u;
        if (threadIdx.x < kDigits) {
#pragma unroll
            for (uint32_t b = 0; b < kSortCluster; ++b) {
                const uint32_t c = counts[b][threadIdx.x];
                all += c;
                before += b < rank ? c : 0u;
            }
        }
        const uint32_t start = digit_scan(all, sh.warp_sums);
        if (threadIdx.x < kDigits) sh.base[threadIdx.x] = start + before;
        __syncthreads();
        for (int64_t at = begin; at < end; at += kSortTile) scatter_tile(p, sh, at, end, pass);
        ptx::cluster_sync_all();                                     // the list is in its new order, and all have read the counts
    }
}

// One pass over more blocks: the digits of every block are counted, then every block adds up the counts in front of its own.
__global__ void __launch_bounds__(kSortThreads) embedding_count_kernel(const SortParams p, int pass) {
    __shared__ SortShared sh;
    pdl_launch_dependents();
    pdl_wait();
    if (blockIdx.x >= (unsigned)p.blocks) return clear_table(p, sh, 2 * pass, 2 * p.passes);
    const int64_t n = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const int64_t begin = blockIdx.x * p.span, end = begin + p.span < n ? begin + p.span : n;
    count_digits(p, sh, begin, end, pass);
    if (threadIdx.x < kDigits) p.hist[blockIdx.x * kDigits + threadIdx.x] = sh.base[threadIdx.x];
}
__global__ void __launch_bounds__(kSortThreads) embedding_scatter_kernel(const SortParams p, int pass) {
    __shared__ SortShared sh;
    pdl_launch_dependents();
    pdl_wait();
    if (blockIdx.x >= (unsigned)p.blocks) return clear_table(p, sh, 2 * pass + 1, 2 * p.passes);
    const int64_t n = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const int64_t begin = blockIdx.x * p.span, end = begin + p.span < n ? begin + p.span : n;
    if (begin >= end) return;
    uint32_t all = 0u, before = 0u;
    if (threadIdx.x < kDigits) {
#pragma unroll 8
        for (int b = 0; b < p.blocks; ++b) {
            const uint32_t c = p.hist[b * kDigits + threadIdx.x];
            all += c;
            before += b < (int)blockIdx.x ? c : 0u;
        }
    }
    const uint32_t start = digit_scan(all, sh.warp_sums);
    if (threadIdx.x < kDigits) sh.base[threadIdx.x] = start + before;
    __syncthreads();
    for (int64_t at = begin; at < end; at += kSortTile) scatter_tile(p, sh, at, end, pass);
}

// ---- backward: the sums ----
struct SumParams {
    const uint4* dOut;
    const uint32_t* keys;                             // sorted; V and above: no id
    const int32_t* rows;
    const int32_t* M_keep_dev;
    int64_t M_keep_cap, V;
    float *dTable, *partial;                          // partial [pieces][2][C]: the id that came in from the left, the one that goes on
    int vecs, strips, piece, accumulate;              // 16-byte vectors of a row, 32-vector strips of it, places of a piece
    float scale;
    const int32_t* status_word;
};

template <int P>
__device__ __forceinline__ void put_sum(float* to, const f32x2 (&f)[P], float scale, bool add_old) {
#pragma unroll
    for (int e = 0; e < P; e += 2) {
        float4* q = reinterpret_cast<float4*>(to + 2 * e);
        const float2 a = both(f[e]), b = both(f[e + 1]);
        float4 s = make_float4(scale * a.x, scale * a.y, scale * b.x, scale * b.y);
        if (add_old) {
            const float4 old = *q;
            s = make_float4(s.x + old.x, s.y + old.y, s.z + old.z, s.w + old.w);
        }
        *q = s;
    }
}

// A warp adds up one strip (32 vectors) of the rows of one piece.
constexpr int kSumUnroll = 8;
template <typename T>
__global__ void __launch_bounds__(256) embedding_sum_kernel(const SumParams p) {
    constexpr int N = Vec<T>::N, P = N / 2;
    pdl_launch_dependents();
    pdl_wait();
    if (block_sees_error(p.status_word)) return;
    const int lane = threadIdx.x & 31;
    const int64_t warp = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t piece = warp / p.strips;
    const int v = (int)(warp % p.strips) * 32 + lane;
    const int64_t n = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const int64_t lo = piece * p.piece, hi = lo + p.piece < n ? lo + p.piece : n;
    if (lo >= hi) return;
    const uint32_t V = (uint32_t)p.V;
    const bool in = v < p.vecs;
    const int64_t C = (int64_t)p.vecs * N;
    const uint32_t left = lo > 0 ? p.keys[lo - 1] : 0xffffffffu, right = hi < n ? p.keys[hi] : 0xffffffffu;
    uint32_t cur = p.keys[lo];
    f32x2 acc[P];
#pragma unroll
    for (int e = 0; e < P; ++e) acc[e] = pair(0.f, 0.f);
    auto put = [&](bool last) {
        if (!in) return;
        if (cur == left) put_sum(p.partial + piece * 2 * C + (int64_t)v * N, acc, 1.f, false);
        else if (last && cur == right) put_sum(p.partial + (piece * 2 + 1) * C + (int64_t)v * N, acc, 1.f, false);
        else put_sum(p.dTable + (int64_t)cur * C + (int64_t)v * N, acc, p.scale, p.accumulate != 0);
    };
    for (int64_t base = lo; base < hi && cur < V; base += 32) {
        const uint32_t my_key = base + lane < hi ? p.keys[base + lane] : V;
        const int32_t my_row = base + lane < hi ? p.rows[base + lane] : 0;
        const int most = hi - base < 32 ? (int)(hi - base) : 32;
        const int count = __popc(__ballot_sync(0xffffffffu, my_key < V && lane < most));       // (sorted: the ones with an id come first)
        for (int j0 = 0; j0 < count; j0 += kSumUnroll) {
            uint4 q[kSumUnroll];
#pragma unroll
            for (int u = 0; u < kSumUnroll; ++u) {
                const int64_t r = __shfl_sync(0xffffffffu, my_row, (j0 + u) & 31);
                q[u] = j0 + u < count && in ? ld_stream(p.dOut + r * p.vecs + v) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int u = 0; u < kSumUnroll; ++u) {
                const uint32_t k = __shfl_sync(0xffffffffu, my_key, (j0 + u) & 31);
                if (j0 + u >= count) break;
                if (k != cur) {
                    put(false);
                    cur = k;
#pragma unroll
                    for (int e = 0; e < P; ++e) acc[e] = pair(0.f, 0.f);
                }
                f32x2 f[P];
                Vec<T>::unpack(q[u], f);
#pragma unroll
                for (int e = 0; e < P; ++e) acc[e] = add(acc[e], f[e]);
            }
        }
        if (count < most) {                           // the rest of the list has no ids
            if (cur < V) put(false);
            return;
        }
    }
    if (cur < V) put(true);
}

// Adds the partial rows of the ids that cross a piece's border.  A warp looks after one strip of the piece in which such an id begins and
// adds up the pieces itself, in their order, where they are kJoinAlone at most; a longer one - of which no two begin in a block's
// eight pieces - is left to all of the block's warps, who take its pieces in turns and whose sums are added in the order of the
// warps.  (A block for each piece: 8 blocks an SM that mostly find nothing to do.)
constexpr int kJoinAlone = 16;
template <typename T>
__global__ void __launch_bounds__(256) embedding_join_kernel(const SumParams p) {
    constexpr int N = Vec<T>::N, P = N / 2;
    __shared__ f32x2 part[8][32][P + 1];
    __shared__ int64_t long_piece, long_end;
    pdl_launch_dependents();
    pdl_wait();
    if (block_sees_error(p.status_word)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) long_piece = -1;
    __syncthreads();
    const int64_t n = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const int64_t piece = blockIdx.x / p.strips * 8 + warp, lo = piece * p.piece, hi = lo + p.piece;
    const int v = (int)(blockIdx.x % p.strips) * 32 + lane;
    const int64_t C = (int64_t)p.vecs * N;
    f32x2 acc[P];
    // pieces from, from + step, ... of the id that begins in piece `first`
    auto add_pieces = [&](int64_t first, int64_t from, int64_t end, int64_t step) {
#pragma unroll
        for (int e = 0; e < P; ++e) acc[e] = pair(0.f, 0.f);
        if (v >= p.vecs) return;
        constexpr int kAhead = 4;                     // loads under way together
        for (int64_t q = from; q < end; q += kAhead * step) {
            f32x2 f[kAhead][P];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t at = q + u * step;
#pragma unroll
                for (int e = 0; e < P; ++e) f[u][e] = pair(0.f, 0.f);
                if (at < end) load_f32<N>(p.partial + (at * 2 + (at == first ? 1 : 0)) * C + (int64_t)v * N, f[u]);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int e = 0; e < P; ++e) acc[e] = add(acc[e], f[u][e]);
        }
    };
    if (hi < n) {
        const uint32_t k = p.keys[hi - 1];
        if (k < (uint32_t)p.V && p.keys[hi] == k && (lo == 0 || p.keys[lo - 1] != k)) {
            const int64_t pieces = (n + p.piece - 1) / p.piece;
            // pieces [piece + 1, end) begin with this id (the list is sorted: 32 probes a step)
            int64_t end = piece + 2, top = pieces;
            while (end < top) {
                const int64_t step = (top - end + 31) / 32, at = end + lane * step;
                const int same = __popc(__ballot_sync(0xffffffffu, at < top && p.keys[(at < top ? at : end) * p.piece] == k));
                if (same == 0) break;
                const int64_t last = end + (same - 1) * step;
                end = last + 1;
                top = last + step < top ? last + step : top;
            }
            if (end - piece <= kJoinAlone) {
                add_pieces(piece, piece, end, 1);
                if (v < p.vecs) put_sum(p.dTable + (int64_t)k * C + (int64_t)v * N, acc, p.scale, p.accumulate != 0);
            } else if (lane == 0) {
                long_piece = piece;
                long_end = end;
            }
        }
    }
    __syncthreads();
    const int64_t first = long_piece;
    if (first < 0) return;
    add_pieces(first, first + warp, long_end, 8);
#pragma unroll
    for (int e = 0; e < P; ++e) part[warp][lane][e] = acc[e];
    __syncthreads();
    if (warp != 0 || v >= p.vecs) return;
#pragma unroll
    for (int w = 1; w < 8; ++w)
#pragma unroll
        for (int e = 0; e < P; ++e) acc[e] = add(acc[e], part[w][lane][e]);
    put_sum(p.dTable + (int64_t)p.keys[(first + 1) * p.piece] * C + (int64_t)v * N, acc, p.scale, p.accumulate != 0);
}

// ---- backward: short lists ----
// Up to kFewRows kept rows there is nothing to sort: one launch, in which block m looks through the list for the id of its m-th row and,
// if no row before it has the same, adds up the rows that have it, in their order.  Eight warps have a strip of the row each, or,
// where an id has many rows, every eighth part of them, which are added in the order of the parts.  The blocks behind clear the rows
// of dTable that no row of the list has.  (250 rows into 2000 x 512 4.2 us, 1000 rows 9.9 and by sorting 20.)  A single block adds up an id's
// rows - 1024 rows of one id, 768 fp32: 56 us, by sorting 17; bf16 34 and 15 - so tables of so few rows that ids must repeat often are
// sorted for.  (Whether they do repeat in a larger table, only the device knows.)
constexpr int kFewRows = 1024;

struct FewParams {
    const uint4* dOut;
    const int32_t *ids, *keep_rows, *M_keep_dev;
    int64_t M, M_keep_cap, V;
    float* dTable;
    int vecs, compact, accumulate;
    float scale;
    const int32_t* status_word;
};

template <typename T>
__global__ void __launch_bounds__(256) embedding_few_kernel(const FewParams p) {
    constexpr int N = Vec<T>::N, P = N / 2;
    __shared__ uint32_t keys[kFewRows];
    __shared__ int32_t rows[kFewRows];                // of the list, then of this block's id
    __shared__ int matches;
    __shared__ f32x2 part[8][32][P + 1];
    pdl_launch_dependents();
    pdl_wait();
    if (block_sees_error(p.status_word)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = (int)load_m_keep(p.M_keep_dev, p.M_keep_cap), mine = (int)blockIdx.x;
    const bool clears = mine >= (int)p.M_keep_cap;
    if (!clears && mine >= n) return;
    const int64_t C = (int64_t)p.vecs * N;
    {
        int32_t row[kFewRows / 256], id[kFewRows / 256];
#pragma unroll
        for (int i = 0; i < kFewRows / 256; ++i) row[i] = (int)threadIdx.x + i * 256 < n ? mapped_row(p.keep_rows, threadIdx.x + i * 256) : -1;
#pragma unroll
        for (int i = 0; i < kFewRows / 256; ++i) id[i] = __ldg(p.ids + (row[i] >= 0 && row[i] < p.M ? row[i] : 0));
#pragma unroll
        for (int i = 0; i < kFewRows / 256; ++i) {
            const int m = (int)threadIdx.x + i * 256;
            const bool ok = row[i] >= 0 && row[i] < p.M;
            keys[m] = ok && id[i] >= 0 && id[i] < p.V ? (uint32_t)id[i] : 0xffffffffu;
            rows[m] = p.compact ? m : row[i];
        }
    }
    __syncthreads();
    if (clears) {
        uint32_t mine_k[kFewRows / 32];
#pragma unroll
        for (int i = 0; i < kFewRows / 32; ++i) mine_k[i] = keys[i * 32 + lane];
        const int64_t warps = ((int64_t)gridDim.x - p.M_keep_cap) * 8, me = ((int64_t)blockIdx.x - p.M_keep_cap) * 8 + warp;
        for (int64_t v = p.V * me / warps; v < p.V * (me + 1) / warps; ++v) {
            bool here = false;
#pragma unroll
            for (int i = 0; i < kFewRows / 32; ++i) here |= mine_k[i] == (uint32_t)v;
            if (__any_sync(0xffffffffu, here)) continue;
            float4* to = reinterpret_cast<float4*>(p.dTable + v * C);
            for (int64_t c = lane; c < C / 4; c += 32) to[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        return;
    }
    const uint32_t key = keys[mine];
    if (key == 0xffffffffu) return;
    if (warp == 0) {                                  // the rows of this id, unless an earlier block has them
        int found = 0;
        for (int c = 0; c < n; c += 32) {
            const bool same = keys[c + lane] == key;
            const uint32_t set = __ballot_sync(0xffffffffu, same);
            if (set && found == 0 && c + __ffs(set) - 1 < mine) {
                found = -1;
                break;
            }
            const int32_t r = rows[c + lane];         // (the list grows behind what is read)
            __syncwarp();
            if (same) rows[found + __popc(set & ((1u << lane) - 1u))] = r;
            found += __popc(set);
            __syncwarp();
        }
        if (lane == 0) matches = found;
    }
    __syncthreads();
    const int count = matches;
    if (count < 0) return;
    const int strips = (p.vecs + 31) / 32;
    auto add_rows = [&](int v, int from, int to, f32x2 (&acc)[P]) {
#pragma unroll
        for (int e = 0; e < P; ++e) acc[e] = pair(0.f, 0.f);
        for (int i = from; i < to; i += 8) {
            uint4 q[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) q[u] = i + u < to && v < p.vecs ? ld_stream(p.dOut + (int64_t)rows[i + u] * p.vecs + v) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (i + u >= to) break;
                f32x2 f[P];
                Vec<T>::unpack(q[u], f);
#pragma unroll
                for (int e = 0; e < P; ++e) acc[e] = add(acc[e], f[e]);
            }
        }
    };
    f32x2 acc[P];
    if (count <= 16) {
        for (int strip = warp; strip < strips; strip += 8) {
            const int v = strip * 32 + lane;
            add_rows(v, 0, count, acc);
            if (v < p.vecs) put_sum(p.dTable + (int64_t)key * C + (int64_t)v * N, acc, p.scale, p.accumulate != 0);
        }
        return;
    }
    for (int strip = 0; strip < strips; ++strip) {
        const int v = strip * 32 + lane;
        add_rows(v, count * warp / 8, count * (warp + 1) / 8, acc);
#pragma unroll
        for (int e = 0; e < P; ++e) part[warp][lane][e] = acc[e];
        __syncthreads();
        if (warp == 0 && v < p.vecs) {
#pragma unroll
            for (int w = 1; w < 8; ++w)
#pragma unroll
                for (int e = 0; e < P; ++e) acc[e] = add(acc[e], part[w][lane][e]);
            put_sum(p.dTable + (int64_t)key * C + (int64_t)v * N, acc, p.scale, p.accumulate != 0);
        }
        __syncthreads();
    }
}

// ---- host ----
struct SumShape {
    int strips, piece;
    int64_t pieces;
};
// pieces: enough warps for the device (16 an SM: more leave more partial rows), and eight places at least, so that a piece's own loads overlap
inline SumShape sum_shape(sbp_dtype dt, int64_t M_keep_cap, int64_t C) {
    SumShape s;
    const int64_t vecs = C / (dt == SBP_BF16 ? 8 : 4);
    s.strips = (int)((vecs + 31) / 32);
    const int64_t want = (int64_t)kNumSMs * 16 / s.strips, p = (M_keep_cap + want) / (want > 0 ? want : 1);
    s.piece = (int)(p < 8 ? 8 : p);
    s.pieces = (M_keep_cap + s.piece - 1) / s.piece;
    return s;
}
struct SortShape {
    int blocks, passes, bits;
    int64_t span;
};
inline SortShape sort_shape(int64_t M_keep_cap, int64_t V) {
    SortShape s;
    int bits = 1;
    while ((V >> bits) != 0) ++bits;                  // keys 0 .. V
    s.passes = (bits + 7) / 8;
    s.bits = (bits + s.passes - 1) / s.passes;
    const int64_t unit = M_keep_cap <= kSortClusterRows ? 32 : kSortTile, most = M_keep_cap <= kSortClusterRows ? kSortCluster : kSortMaxBlocks;
    s.span = (M_keep_cap + unit * most - 1) / (unit * most) * unit;
    s.blocks = M_keep_cap <= kSortClusterRows ? kSortCluster : (int)((M_keep_cap + s.span - 1) / s.span);
    return s;
}
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

cudaError_t launch_embedding_forward(sbp_dtype dt, const void* table, int64_t V, int64_t C, const int32_t* ids, int64_t M, float scale,
                                     const void* add, void* out, int32_t* status_word, cudaStream_t stream) {
    const int64_t vecs = C / (dt == SBP_BF16 ? 8 : 4);
    const RowLength row(vecs);
    const dim3 grid((unsigned)copy_blocks(M * vecs)), block(kCopyThreads);
    auto go = [&](auto kernel) {
        const cudaError_t e = launch_pdl(kernel, grid, block, 0, stream, (const uint4*)table, row, V, ids, M, scale, (const uint4*)add, (uint4*)out, status_word);
        return e == cudaSuccess ? report_ids(ids, nullptr, nullptr, M, M, V, status_word, stream) : e;
    };
    if (dt == SBP_BF16) return add ? go(embedding_forward_kernel<__nv_bfloat16, true>) : go(embedding_forward_kernel<__nv_bfloat16, false>);
    return add ? go(embedding_forward_kernel<float, true>) : go(embedding_forward_kernel<float, false>);
}

size_t embedding_backward_workspace_bytes(sbp_dtype dt, int64_t M_keep_cap, int64_t C) {
    const SumShape s = sum_shape(dt, M_keep_cap, C);
    return 4 * up256((size_t)M_keep_cap * 4) + up256((size_t)kSortMaxBlocks * kDigits * 4) + up256((size_t)s.pieces * 2 * (size_t)C * 4);
}

cudaError_t launch_embedding_backward(sbp_dtype dt, const void* dOut, bool compact, const int32_t* ids, const int32_t* keep_rows,
                                      const int32_t* M_keep_dev, int64_t M, int64_t M_keep_cap, int64_t V, int64_t C, float scale,
                                      float* dTable, bool accumulate, void* workspace, int32_t* status_word, cudaStream_t stream) {
    auto reported = [&](cudaError_t e) { return e == cudaSuccess ? report_ids(ids, keep_rows, M_keep_dev, M, M_keep_cap, V, status_word, stream) : e; };
    if (M_keep_cap <= kFewRows && M_keep_cap <= 32 * V) {
        FewParams f = {};
        f.dOut = (const uint4*)dOut;
        f.ids = ids;
        f.keep_rows = keep_rows;
        f.M_keep_dev = M_keep_dev;
        f.M = M;
        f.M_keep_cap = M_keep_cap;
        f.V = V;
        f.dTable = dTable;
        f.vecs = (int)(C / (dt == SBP_BF16 ? 8 : 4));
        f.compact = compact;
        f.accumulate = accumulate;
        f.scale = scale;
        f.status_word = status_word;
        const int64_t clear = accumulate ? 0 : (V + 7) / 8 < 4 * kNumSMs ? (V + 7) / 8 : 4 * kNumSMs;
        if (M_keep_cap + clear == 0) return cudaSuccess;             // nothing to add, and nothing to clear
        const dim3 grid((unsigned)(M_keep_cap + clear));
        return reported(dt == SBP_BF16 ? launch_pdl(embedding_few_kernel<__nv_bfloat16>, grid, dim3(256), 0, stream, f)
                                       : launch_pdl(embedding_few_kernel<float>, grid, dim3(256), 0, stream, f));
    }
    const SortShape so = sort_shape(M_keep_cap, V);
    const SumShape su = sum_shape(dt, M_keep_cap, C);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const size_t list = up256((size_t)M_keep_cap * 4);
    SortParams p = {};
    p.ids = ids;
    p.keep_rows = keep_rows;
    p.M_keep_dev = M_keep_dev;
    p.M = M;
    p.M_keep_cap = M_keep_cap;
    p.V = V;
    p.compact = compact;
    p.keys[0] = (uint32_t*)ws;
    p.keys[1] = (uint32_t*)(ws + list);
    p.rows[0] = (int32_t*)(ws + 2 * list);
    p.rows[1] = (int32_t*)(ws + 3 * list);
    p.hist = (uint32_t*)(ws + 4 * list);
    p.span = so.span;
    p.blocks = so.blocks;
    p.passes = so.passes;
    p.bits = so.bits;
    p.clear = accumulate ? nullptr : (uint4*)dTable;
    p.clear_vecs = V * (C / 4);
    p.status_word = status_word;
    const int64_t want = (p.clear_vecs + 1023) / 1024;               // (16 KB)
    int clear_blocks = accumulate ? 0 : (int)(want < 3 * kNumSMs ? want : 3 * kNumSMs);
    const dim3 block(kSortThreads);
    cudaError_t e;
    if (M_keep_cap <= kSortClusterRows) {
        clear_blocks = (clear_blocks + kSortCluster - 1) / kSortCluster * kSortCluster;
        e = launch_pdl_cluster(embedding_sort_kernel, dim3((unsigned)(so.blocks + clear_blocks)), block, 0, kSortCluster, stream, p);
        if (e != cudaSuccess) return e;
    } else {
        const dim3 grid((unsigned)(so.blocks + clear_blocks));
        for (int pass = 0; pass < so.passes; ++pass) {
            if ((e = launch_pdl(embedding_count_kernel, grid, block, 0, stream, p, pass)) != cudaSuccess) return e;
            if ((e = launch_pdl(embedding_scatter_kernel, grid, block, 0, stream, p, pass)) != cudaSuccess) return e;
        }
    }
    SumParams s = {};
    s.dOut = (const uint4*)dOut;
    s.keys = p.keys[(so.passes - 1) & 1];
    s.rows = p.rows[(so.passes - 1) & 1];
    s.M_keep_dev = M_keep_dev;
    s.M_keep_cap = M_keep_cap;
    s.V = V;
    s.dTable = dTable;
    s.partial = (float*)(ws + 4 * list + up256((size_t)kSortMaxBlocks * kDigits * 4));
    s.vecs = (int)(C / (dt == SBP_BF16 ? 8 : 4));
    s.strips = su.strips;
    s.piece = su.piece;
    s.accumulate = accumulate;
    s.scale = scale;
    s.status_word = status_word;
    const int64_t warps = su.pieces * su.strips;
    const dim3 sum_grid((unsigned)((warps + 7) / 8)), join_grid((unsigned)((su.pieces + 7) / 8 * su.strips));
    e = dt == SBP_BF16 ? launch_pdl(embedding_sum_kernel<__nv_bfloat16>, sum_grid, dim3(256), 0, stream, s)
                       : launch_pdl(embedding_sum_kernel<float>, sum_grid, dim3(256), 0, stream, s);
    if (e == cudaSuccess && su.pieces >= 2)
        e = dt == SBP_BF16 ? launch_pdl(embedding_join_kernel<__nv_bfloat16>, join_grid, dim3(256), 0, stream, s)
                           : launch_pdl(embedding_join_kernel<float>, join_grid, dim3(256), 0, stream, s);
    return reported(e);
}

}  // namespace sbp
