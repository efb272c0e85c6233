// Norms before and after a block fused with its gate and residual scale, forward and backward.
//
//   u = N(Y) w_post + b_post  (or Y),   R = s H + gate u,   Z = N(R) w_pre + b_pre
//
// N: x -> (x - mean) / sqrt(var + eps) over the C channels of a row (LayerNorm), or x / sqrt(mean(x^2) + eps) (RMSNorm).
// With n = N(x) and q the gradient with respect to n, the gradient with respect to x is
//   rstd (q - mean(q) - n mean(q n))       (without mean(q) for RMSNorm).
//
// Bound by memory: the forward reads H and Y and writes R, Z and the three caches once; the backward reads dR, dZ, R_keep and
// Y_keep and writes dH and dY once.  Nothing but the rows is stored for the backward: a row passes through registers anyway,
// so its statistics are made again there instead of being kept.  Means and variances are taken in two steps (the mean first,
// then the squares of what is left), since the one-step form loses the variance of rows whose mean is large against it.
// All arithmetic is fp32; R is normalised before it is rounded.
#include "row_copy.cuh"
#include "row_math.cuh"
#include "zero_rows.cuh"

#include <type_traits>

namespace sbp {
namespace {

// ---- forward ----
struct NormFwdParams {
    const uint4 *H, *Y;
    const float *post_w, *post_b, *pre_w, *pre_b;
    const uint4* gate;
    uint4 *R, *Z, *Y_keep, *R_keep, *Z_keep;
    const int32_t *keep_rows, *M_keep_dev, *status_word;
    int64_t M, M_keep_cap;
    FastDiv gate_group;
    int vecs, chunk;                                  // 16-byte vectors of a row; rows of a warp (or block)
    float scale, eps, inv_c;
    int caches;
};

// Rows of the caches past M_keep are cleared, and those of entries outside the tensor, the first or the last ones of the list: by worker
// `worker` of `workers`, `threads` threads.  (A function of its own, so that it takes no registers from the rows: inlined it cost up to 4 %.)
__device__ __noinline__ void clear_cache_rows(uint4* Y_keep, uint4* R_keep, uint4* Z_keep, const int32_t* keep_rows, int64_t M, int64_t M_keep,
                                              int64_t M_keep_cap, int vecs, int64_t worker, int64_t workers, int t, int threads) {
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    auto clear = [&](int64_t m) {
        for (int v = t; v < vecs; v += threads) {
            if (Y_keep != nullptr) Y_keep[m * vecs + v] = zero;
            if (R_keep != nullptr) R_keep[m * vecs + v] = zero;
            if (Z_keep != nullptr) Z_keep[m * vecs + v] = zero;
        }
    };
    for (int64_t m = M_keep + worker; m < M_keep_cap; m += workers) clear(m);
    if (keep_rows == nullptr) return;
    if (worker == 0)
        for (int64_t m = 0; m < M_keep && keep_rows[m] < 0; ++m) clear(m);
    if (worker == workers - 1)
        for (int64_t m = M_keep - 1; m >= 0 && keep_rows[m] >= M; --m) clear(m);
}

// kLanes threads of a warp share a row (kLanes 0: a block, for long rows), each with kNV vectors of it, kU rows at a time; the rows of a
// warp, `chunk` <= 32 consecutive ones, are dealt to its groups of lanes in turn.  Which of them are kept, and the place of each in
// the caches, comes from one search of the list.  kFull: the threads' vectors are the row's, none lies behind it (what those
// would hold stays zero otherwise, at the price of a branch a vector, across which nothing is scheduled).
template <typename T, int kNV, int kLanes, bool kFull, bool kLayer, bool kPost>
__global__ void __launch_bounds__(kNV * Vec<T>::N > 8 ? 512 : 256, kNV * Vec<T>::N > 8 ? 1 : 4)
norm_forward_kernel(const NormFwdParams p) {
    constexpr bool kMulti = kLanes == 0;
    constexpr int VN = Vec<T>::N, P = VN / 2, E2 = kNV * P;          // pairs of a vector, pairs a thread holds of a row
    constexpr int kU = E2 > 4 ? 1 : 2;
    constexpr int kGroups = kMulti ? 1 : 32 / (kMulti ? 32 : kLanes);
    __shared__ float4 scratch[kMulti ? 64 : 1];
    pdl_launch_dependents();
    pdl_wait();
    if (block_sees_error(p.status_word)) return;
    const int lane = threadIdx.x & 31;
    const int64_t worker = kMulti ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int64_t workers = kMulti ? (int64_t)gridDim.x : (int64_t)gridDim.x * (blockDim.x >> 5);
    RowThreads<kLanes> row = {kMulti ? (int)threadIdx.x : lane % (kMulti ? 32 : kLanes), (int)blockDim.x, (int)blockDim.x >> 5, 1, 0, scratch};
    const int group = kMulti ? 0 : lane / (kMulti ? 32 : kLanes), threads = row.threads();
    const int64_t M_keep = p.caches ? load_m_keep(p.M_keep_dev, p.M_keep_cap) : 0;
    const int64_t lo = worker * p.chunk;
    const int count = lo < p.M ? (p.M - lo < p.chunk ? (int)(p.M - lo) : p.chunk) : 0;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    bool in[kNV];
#pragma unroll
    for (int j = 0; j < kNV; ++j) in[j] = kFull || row.t + j * threads < p.vecs;

    if (count > 0) {
        uint32_t kept = 0u;                           // bit d: row lo + d is in the list
        int64_t place = 0;                            // of the first of them
        for (int d0 = 0; d0 < count; d0 += kU * kGroups) {
            f32x2 x[kU][E2];
            uint4 yq[kU][kNV], hq[kU][kNV];
            int64_t at[kU];
            bool live[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int d = d0 + u * kGroups + group;
                live[u] = d < count;
                at[u] = (lo + d) * p.vecs + row.t;
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    yq[u][j] = in[j] && live[u] && p.Y != nullptr ? __ldcg(p.Y + at[u] + j * threads) : zero;
                    hq[u][j] = in[j] && live[u] && p.H != nullptr ? __ldcg(p.H + at[u] + j * threads) : zero;
                }
            }
            if (d0 == 0 && p.caches) {                // (under the first rows' loads)
                if (p.keep_rows == nullptr) {
                    const int64_t n = M_keep - lo;
                    kept = n >= 32 ? 0xffffffffu : n > 0 ? (1u << n) - 1u : 0u;
                    place = lo;
                } else {
                    place = warp_lower_bound(p.keep_rows, M_keep, lo, lane);
                    const int64_t d = place + lane < M_keep ? (int64_t)__ldg(p.keep_rows + place + lane) - lo : 32;
                    kept = __reduce_or_sync(0xffffffffu, d >= 0 && d < 32 ? 1u << d : 0u);
                }
            }
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < kNV; ++j) Vec<T>::unpack(yq[u][j], &x[u][j * P]);
            auto normalise = [&](const float* w, const float* b) {
                float s[kU];
                if constexpr (kLayer) {
#pragma unroll
                    for (int u = 0; u < kU; ++u) {
                        f32x2 a = x[u][0];
#pragma unroll
                        for (int e = 1; e < E2; ++e) a = add(a, x[u][e]);
                        s[u] = both(a).x + both(a).y;
                    }
                    row.sums(s);
#pragma unroll
                    for (int u = 0; u < kU; ++u)
#pragma unroll
                        for (int j = 0; j < kNV; ++j) {
                            const float m = in[j] ? -s[u] * p.inv_c : 0.f;          // threads past the row hold zeros
#pragma unroll
                            for (int e = 0; e < P; ++e) x[u][j * P + e] = add(x[u][j * P + e], pair(m, m));
                        }
                }
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    f32x2 a = mul(x[u][0], x[u][0]);
#pragma unroll
                    for (int e = 1; e < E2; ++e) a = fma(x[u][e], x[u][e], a);
                    s[u] = both(a).x + both(a).y;
                }
                row.sums(s);
#pragma unroll
                for (int u = 0; u < kU; ++u) s[u] = rsqrtf(fmaf(s[u], p.inv_c, p.eps));
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    if (!in[j]) continue;
                    f32x2 wf[P], bf[P];
                    load_f32<VN>(w + (row.t + j * threads) * VN, wf);
                    if (b != nullptr) {
                        load_f32<VN>(b + (row.t + j * threads) * VN, bf);
                    } else {
#pragma unroll
                        for (int e = 0; e < P; ++e) bf[e] = pair(-0.f, -0.f);
                    }
#pragma unroll
                    for (int u = 0; u < kU; ++u)
#pragma unroll
                        for (int e = 0; e < P; ++e) x[u][j * P + e] = fma(mul(x[u][j * P + e], pair(s[u], s[u])), wf[e], bf[e]);
                }
            };
            if constexpr (kPost) normalise(p.post_w, p.post_b);
            int64_t slot[kU];
            bool keep[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int d = (d0 + u * kGroups + group) & 31;
                keep[u] = live[u] && (kept >> d & 1u);
                slot[u] = (place + __popc(kept & ((1u << d) - 1u))) * p.vecs + row.t;
                if (p.gate != nullptr && live[u]) {
                    const uint4* gate = p.gate + (int64_t)p.gate_group((uint32_t)(lo + d0 + u * kGroups + group)) * p.vecs + row.t;
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        if (!in[j]) continue;
                        f32x2 g[P];
                        Vec<T>::unpack(__ldg(gate + j * threads), g);
#pragma unroll
                        for (int e = 0; e < P; ++e) x[u][j * P + e] = mul(x[u][j * P + e], g[e]);
                    }
                }
                uint4 r[kNV];
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    f32x2 h[P];
                    Vec<T>::unpack(hq[u][j], h);
#pragma unroll
                    for (int e = 0; e < P; ++e) x[u][j * P + e] = p.H != nullptr ? fma(pair(p.scale, p.scale), h[e], x[u][j * P + e]) : x[u][j * P + e];
                    r[j] = Vec<T>::pack(&x[u][j * P]);
                }
                if (p.R != nullptr && live[u]) {
#pragma unroll
                    for (int j = 0; j < kNV; ++j)
                        if (in[j]) p.R[at[u] + j * threads] = r[j];
                }
                if (keep[u]) {
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        if (!in[j]) continue;
                        if (p.R_keep != nullptr) p.R_keep[slot[u] + j * threads] = r[j];
                        if (p.Y_keep != nullptr) p.Y_keep[slot[u] + j * threads] = yq[u][j];
                    }
                }
            }
            if (p.pre_w != nullptr) {
                __syncwarp();
                normalise(p.pre_w, p.pre_b);
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    if (!live[u]) continue;
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        if (!in[j]) continue;
                        const uint4 z = Vec<T>::pack(&x[u][j * P]);
                        if (p.Z != nullptr) p.Z[at[u] + j * threads] = z;
                        if (keep[u] && p.Z_keep != nullptr) p.Z_keep[slot[u] + j * threads] = z;
                    }
                }
            }
            __syncwarp();
        }
    }
    // (kLanes 0: the threads of the block)
    if (p.caches) clear_cache_rows(p.Y_keep, p.R_keep, p.Z_keep, p.keep_rows, p.M, M_keep, p.M_keep_cap, p.vecs, worker, workers,
                                   kMulti ? (int)threadIdx.x : lane, kMulti ? (int)blockDim.x : 32);
}

// ---- backward ----
constexpr int kNormMaxC = 8192;
constexpr int kNormSums = 5;                          // dpost_w, dpost_b, dpre_w, dpre_b, dgate
constexpr int kNormMostWorkers = 15;                  // of a block, where each has a barrier of its own
struct NormBwdParams {
    const uint4 *dR, *dZ, *R_keep, *Y_keep;
    const float *post_w, *post_b, *pre_w;
    const uint4* gate;
    uint4 *dH, *dY;
    const int32_t *keep_rows, *M_keep_dev, *status_word;
    int64_t M, M_keep_cap;
    FastDiv gate_group;
    float* dgate;                                     // (where it has more than one row: its sums leave a row at a time)
    float* sums;                                      // [kNormSums][blocks][C]
    float* gate_sums;                                 // [workers][2][C]: first and last gate row of each worker
    int64_t workers;
    int want;                                         // bit k: sum k is wanted
    int one_gate;                                     // the gate has one row: its gradient is a sum like the others
    int vecs, warps, per_block, accumulate, copy_rest;               // warps of a worker (kLanes 0), workers of a block
    int blocks;                                       // with workers; those behind them only copy
    float scale, eps, inv_c;
};

__device__ __forceinline__ int64_t norm_chunk(int64_t M_keep, int64_t workers) { return (M_keep + workers - 1) / workers; }

// Rows that a worker has at a time, and threads of a block (one an SM), by the numbers a thread has of a row: two rows share what a row
// costs besides its numbers, and give a warp something to do while it waits for the sums of either.
__host__ __device__ constexpr int norm_backward_rows(int numbers, bool many_warps) { return numbers <= 8 && !many_warps ? 2 : 1; }
__host__ __device__ constexpr int norm_backward_threads(int numbers, bool many_warps) { return numbers <= 8 && !many_warps ? 384 : 512; }

// A worker - kLanes threads of a warp, or, kLanes 0, some warps - takes consecutive kept rows, two at a time where they fit in the
// registers; a thread has the same kNV vectors of each, so that its share of the weights' gradients stays there too: the sums of
// dZ n_R and dZ, and, for the rows of one gate row, S1 = sum G n_Y and S0 = sum G, of which the other three are made when the gate
// row changes (dgate = post_w S1 + post_b S0, dpost_w += gate S1, dpost_b += gate S0).  At the end the block's workers are added up
// in shared memory, and the block leaves one partial row of each sum for a second launch.
// The list is ascending, so a gate row's rows are consecutive; dgate leaves a row at a time - straight to its place where no other
// worker has rows of it (all but a worker's first and last gate row).
// Every instruction besides the arithmetic counts here: with the five sums in shared memory, read and written for every row, the
// shared memory was the bound (25088 x 768: 62 us; in registers, one row at a time, 67).
template <typename T, int kNV, int kLanes, bool kMany, bool kFull, bool kLayer, bool kPost>
__global__ void __launch_bounds__(norm_backward_threads(kNV * Vec<T>::N, kMany), 1) norm_backward_kernel(const NormBwdParams p) {
    constexpr bool kMulti = kLanes == 0;
    constexpr int VN = Vec<T>::N, P = VN / 2, E2 = kNV * P, kQ = VN / 4;      // kQ: float4 of a vector's sums
    constexpr int kU = norm_backward_rows(kNV * VN, kMany);
    extern __shared__ float4 sums_s[];                // [worker of the block][wanted sum][vector of the thread][kQ][thread]
    __shared__ float4 scratch[kMulti ? (kMany ? 1 : kNormMostWorkers) * 64 : 1];
    pdl_launch_dependents();
    pdl_wait();
    if (block_sees_error(p.status_word)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int width = kMulti ? p.warps * 32 : kLanes, mine = threadIdx.x / width;          // threads of a worker; which one of the block
    RowThreads<kLanes> row = {(int)threadIdx.x % width, width, p.warps, mine + 1, 0, scratch + mine * 64};
    const int t = row.t, threads = row.threads();
    const int64_t worker = (int64_t)blockIdx.x * p.per_block + mine;
    const int64_t M_keep = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    if (blockIdx.x < (unsigned)p.blocks) {
        const int64_t chunk = norm_chunk(M_keep, p.workers);
        const int64_t lo = worker * chunk < M_keep ? worker * chunk : M_keep, hi = lo + chunk < M_keep ? lo + chunk : M_keep;
        const int64_t C = (int64_t)p.vecs * VN;
        const int per_sum = kNV * kQ * threads, wanted = __popc(p.want);
        float4* own = sums_s + (int64_t)mine * wanted * per_sum + t;
        auto place = [&](int k) { return own + __popc(p.want & ((1 << k) - 1)) * per_sum; };   // of a wanted sum
        for (int i = 0; i < wanted * kNV * kQ; ++i) own[i * threads] = make_float4(0.f, 0.f, 0.f, 0.f);
        bool in[kNV];
#pragma unroll
        for (int j = 0; j < kNV; ++j) in[j] = kFull || t + j * threads < p.vecs;
        const f32x2 none = pair(0.f, 0.f);
        f32x2 pre1[E2], pre0[E2], S1[E2], S0[E2];
#pragma unroll
        for (int e = 0; e < E2; ++e) pre1[e] = pre0[e] = S1[e] = S0[e] = none;
        // the gate rows of the first and the last entry, and that of the rows in S1 and S0 (kNoGate before there is one: entries outside
        // the tensor have none)
        constexpr uint32_t kNoGate = 0xffffffffu;
        uint32_t first = kNoGate, last = kNoGate, cur = p.gate != nullptr ? kNoGate : 0u;
        if (p.gate != nullptr && lo < hi) {
            const int32_t a = mapped_row(p.keep_rows, lo), b = mapped_row(p.keep_rows, hi - 1);
            if (a >= 0 && a < p.M) first = p.gate_group((uint32_t)a);
            if (b >= 0 && b < p.M) last = p.gate_group((uint32_t)b);
        }
        auto accumulate = [&](float4* a, const f32x2* f, bool old) {     // into shared memory (old: or a row of memory)
            const float2 u = both(f[0]), v = both(f[1]);
            float4 s = make_float4(u.x, u.y, v.x, v.y);
            if (old) s = make_float4(s.x + a->x, s.y + a->y, s.z + a->z, s.w + a->w);
            *a = s;
        };
        auto put_gate = [&]() {                           // the end of a gate row (or, without a gate, of the list): S1 and S0 go where they belong
            if (cur == kNoGate) return;
            const bool partial = cur == first || cur == last;
            float* to = partial ? p.gate_sums + (worker * 2 + (cur == first ? 0 : 1)) * C : p.dgate + (int64_t)cur * C;
#pragma unroll
            for (int j = 0; j < kNV; ++j) {
                if (!in[j]) continue;
                const int v = t + j * threads;
                f32x2 f[P], w[P];
                if (p.want & 16) {
#pragma unroll
                    for (int e = 0; e < P; ++e) f[e] = S1[j * P + e];
                    if constexpr (kPost) {
                        load_f32<VN>(p.post_w + v * VN, w);
#pragma unroll
                        for (int e = 0; e < P; ++e) f[e] = mul(f[e], w[e]);
                        if (p.post_b != nullptr) {
                            load_f32<VN>(p.post_b + v * VN, w);
#pragma unroll
                            for (int e = 0; e < P; ++e) f[e] = fma(S0[j * P + e], w[e], f[e]);
                        }
                    }
#pragma unroll
                    for (int h = 0; h < kQ; ++h) {
                        if (p.one_gate) accumulate(place(4) + (j * kQ + h) * threads, f + 2 * h, true);
                        else accumulate(reinterpret_cast<float4*>(to + (int64_t)v * VN) + h, f + 2 * h, !partial && p.accumulate);
                    }
                }
                if constexpr (kPost) {
#pragma unroll
                    for (int e = 0; e < P; ++e) w[e] = pair(1.f, 1.f);
                    if (p.gate != nullptr) Vec<T>::unpack(__ldg(p.gate + (int64_t)cur * p.vecs + v), w);
                    auto add_to = [&](int k, const f32x2* s) {
#pragma unroll
                        for (int e = 0; e < P; ++e) f[e] = mul(s[e], w[e]);
#pragma unroll
                        for (int h = 0; h < kQ; ++h) accumulate(place(k) + (j * kQ + h) * threads, f + 2 * h, true);
                    };
                    if (p.want & 1) add_to(0, &S1[j * P]);
                    if (p.want & 2) add_to(1, &S0[j * P]);
                }
            }
#pragma unroll
            for (int e = 0; e < E2; ++e) S1[e] = S0[e] = none;
        };
        auto total = [](f32x2 a) { return both(a).x + both(a).y; };
        // (several rows a warp: every group of lanes goes round as often as the others, with nothing to do behind its last row)
        constexpr bool kSplit = !kMulti && kLanes < 32;
        const int rounds = kSplit ? (int)chunk : (int)(hi - lo);
        int64_t at = lo * p.vecs + t;
        auto ids = [&](int i, int32_t (&k)[kU]) {         // (-1: no row, or an entry outside the tensor, which is skipped)
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                k[u] = lo + i + u < hi ? mapped_row(p.keep_rows, lo + i + u) : -1;
                if (k[u] >= p.M) k[u] = -1;
            }
        };
        int32_t next[kU];
        ids(0, next);
        for (int i = 0; i < rounds; i += kU, at += kU * (int64_t)p.vecs) {
            int32_t k[kU];
            bool have[kU], live[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                k[u] = next[u];
                have[u] = lo + i + u < hi;
                live[u] = k[u] >= 0;
            }
            f32x2 x[kU][E2], y[kU][E2], g[kU][E2], q[kU][E2];            // R, then what its norm makes of it; Y likewise; dZ; dZ pre_w
            uint4 dq[kU][kNV];
            ids(i + kU, next);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                uint4 rq[kNV], yq[kNV], zq[kNV];
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int64_t from = at + (int64_t)u * p.vecs + j * threads;
                    const bool ok = in[j] && have[u];
                    rq[j] = ok && p.dZ != nullptr ? __ldcg(p.R_keep + from) : zero;
                    zq[j] = ok && p.dZ != nullptr ? __ldcg(p.dZ + from) : zero;
                    yq[j] = ok && p.Y_keep != nullptr ? __ldcg(p.Y_keep + from) : zero;
                    dq[u][j] = in[j] && live[u] && p.dR != nullptr ? __ldcg(p.dR + (int64_t)k[u] * p.vecs + t + j * threads) : zero;
                }
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    Vec<T>::unpack(rq[j], &x[u][j * P]);
                    Vec<T>::unpack(yq[j], &y[u][j * P]);
                    Vec<T>::unpack(zq[j], &g[u][j * P]);
                }
            }
#pragma unroll
            for (int j = 0; j < kNV; ++j) {
                f32x2 w[P];
#pragma unroll
                for (int e = 0; e < P; ++e) w[e] = none;
                if (in[j] && p.dZ != nullptr) load_f32<VN>(p.pre_w + (t + j * threads) * VN, w);
#pragma unroll
                for (int u = 0; u < kU; ++u)
#pragma unroll
                    for (int e = 0; e < P; ++e) q[u][j * P + e] = mul(g[u][j * P + e], w[e]);
            }
            float s1[3 * kU], s2[3 * kU];
            if constexpr (kLayer) {
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    f32x2 sx = x[u][0], sy = y[u][0], sq = q[u][0];
#pragma unroll
                    for (int e = 1; e < E2; ++e) {
                        sx = add(sx, x[u][e]);
                        if constexpr (kPost) sy = add(sy, y[u][e]);
                        sq = add(sq, q[u][e]);
                    }
                    s1[3 * u] = total(sx);
                    s1[3 * u + 1] = kPost ? total(sy) : 0.f;
                    s1[3 * u + 2] = total(sq);
                }
                row.sums(s1);
#pragma unroll
                for (int u = 0; u < kU; ++u)
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        const float mx = in[j] ? -s1[3 * u] * p.inv_c : 0.f, my = in[j] ? -s1[3 * u + 1] * p.inv_c : 0.f;   // (threads past the row keep zeros)
#pragma unroll
                        for (int e = j * P; e < (j + 1) * P; ++e) {
                            x[u][e] = add(x[u][e], pair(mx, mx));
                            if constexpr (kPost) y[u][e] = add(y[u][e], pair(my, my));
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                f32x2 sx = mul(x[u][0], x[u][0]), sy = mul(y[u][0], y[u][0]), sq = mul(q[u][0], x[u][0]);
#pragma unroll
                for (int e = 1; e < E2; ++e) {
                    sx = fma(x[u][e], x[u][e], sx);
                    if constexpr (kPost) sy = fma(y[u][e], y[u][e], sy);
                    sq = fma(q[u][e], x[u][e], sq);
                }
                s2[3 * u] = total(sx);
                s2[3 * u + 1] = kPost ? total(sy) : 0.f;
                s2[3 * u + 2] = total(sq);
            }
            row.sums(s2);
            float s3[2 * kU], rstd_y[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                s3[2 * u] = s3[2 * u + 1] = 0.f;
                const float rstd = rsqrtf(fmaf(s2[3 * u], p.inv_c, p.eps));
                rstd_y[u] = kPost ? rsqrtf(fmaf(s2[3 * u + 1], p.inv_c, p.eps)) : 1.f;
                if (!live[u]) continue;
                // d + rstd (q - mean(q) - n mean(q n)), n = rstd x
                const float k0 = kLayer ? -s1[3 * u + 2] * p.inv_c * rstd : 0.f, k1 = -(s2[3 * u + 2] * p.inv_c * rstd) * rstd;
                if (p.gate != nullptr) {
                    const uint32_t group = p.gate_group((uint32_t)k[u]);
                    if (group != cur) {
                        put_gate();
                        cur = group;
                    }
                }
                f32x2 sq = none, sqn = none;
                const f32x2 rr = pair(rstd, rstd);
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    if (!in[j]) continue;
                    f32x2 out[P], d[P], w[P];
                    Vec<T>::unpack(dq[u][j], d);
                    if (p.dZ != nullptr) {
#pragma unroll
                        for (int e = 0; e < P; ++e) {
                            const int c = j * P + e;
                            const f32x2 n = mul(x[u][c], rr);
                            d[e] = add(d[e], fma(q[u][c], rr, fma(n, pair(k1, k1), pair(k0, k0))));     // the whole gradient of R
                            pre1[c] = fma(g[u][c], n, pre1[c]);
                            pre0[c] = add(pre0[c], g[u][c]);
                        }
                    }
                    if (p.dH != nullptr) {
#pragma unroll
                        for (int e = 0; e < P; ++e) out[e] = mul(d[e], pair(p.scale, p.scale));
                        p.dH[(int64_t)k[u] * p.vecs + t + j * threads] = Vec<T>::pack(out);
                    }
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const int c = j * P + e;
                        if constexpr (kPost) y[u][c] = mul(y[u][c], pair(rstd_y[u], rstd_y[u]));
                        S1[c] = fma(d[e], y[u][c], S1[c]);
                        S0[c] = add(S0[c], d[e]);
                    }
                    if (p.gate != nullptr) {
                        Vec<T>::unpack(__ldg(p.gate + (int64_t)cur * p.vecs + t + j * threads), w);
#pragma unroll
                        for (int e = 0; e < P; ++e) d[e] = mul(d[e], w[e]);
                    }
                    if constexpr (kPost) {
                        load_f32<VN>(p.post_w + (t + j * threads) * VN, w);
#pragma unroll
                        for (int e = 0; e < P; ++e) {
                            d[e] = mul(d[e], w[e]);
                            sq = add(sq, d[e]);
                            sqn = fma(d[e], y[u][j * P + e], sqn);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < P; ++e) g[u][j * P + e] = d[e];
                }
                s3[2 * u] = total(sq);
                s3[2 * u + 1] = total(sqn);
            }
            if constexpr (kPost) {
                __syncwarp();
                row.sums(s3);
            }
            if (p.dY != nullptr) {
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    if (!have[u]) continue;
                    const float c0 = kLayer ? -s3[2 * u] * p.inv_c * rstd_y[u] : 0.f, c1 = -s3[2 * u + 1] * p.inv_c * rstd_y[u];
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        if (!in[j]) continue;
                        if constexpr (kPost) {
#pragma unroll
                            for (int e = j * P; e < (j + 1) * P; ++e)
                                g[u][e] = fma(g[u][e], pair(rstd_y[u], rstd_y[u]), fma(y[u][e], pair(c1, c1), pair(c0, c0)));
                        }
                        p.dY[at + (int64_t)u * p.vecs + j * threads] = live[u] ? Vec<T>::pack(&g[u][j * P]) : zero;
                    }
                }
            }
            __syncwarp();
        }
        if (lo < hi) put_gate();
#pragma unroll
        for (int j = 0; j < kNV; ++j)
#pragma unroll
            for (int h = 0; h < kQ; ++h) {
                if (p.want & 4) accumulate(place(2) + (j * kQ + h) * threads, &pre1[j * P + 2 * h], false);
                if (p.want & 8) accumulate(place(3) + (j * kQ + h) * threads, &pre0[j * P + 2 * h], false);
            }
        // the block's workers together, in their order
        __syncthreads();
        for (int i = threadIdx.x; i < wanted * per_sum; i += blockDim.x) {
            const int which = i / per_sum, rest = i - which * per_sum;   // (sum, (vector, quarter), thread)
            int k = p.want;                                              // the which-th bit that is set
            for (int b = 0; b < which; ++b) k &= k - 1;
            k = __ffs(k) - 1;
            if (k == 4 && !p.one_gate) continue;
            const int jh = rest / threads, v = rest % threads + jh / kQ * threads;
            if (v >= p.vecs) continue;
            float4 s = sums_s[i];
            for (int w = 1; w < p.per_block; ++w) {
                const float4 q = sums_s[(int64_t)w * wanted * per_sum + i];
                s = make_float4(s.x + q.x, s.y + q.y, s.z + q.z, s.w + q.w);
            }
            reinterpret_cast<float4*>(p.sums + ((int64_t)k * p.blocks + blockIdx.x) * C + (int64_t)v * VN)[jh % kQ] = s;
        }
        if (p.dY != nullptr) {                            // rows past M_keep are cleared
            const int64_t warps = (int64_t)p.blocks * (blockDim.x >> 5), me = (int64_t)blockIdx.x * (blockDim.x >> 5) + warp;
            for (int64_t m = M_keep + me; m < p.M_keep_cap; m += warps)
                for (int v = lane; v < p.vecs; v += 32) p.dY[m * p.vecs + v] = zero;
        }
    }
    // the rows outside the list take the residual's gradient alone; every warp - of the blocks that do nothing else, if there are
    // any - has its share of all rows
    const int copy_from = (int)gridDim.x > p.blocks ? p.blocks : 0;
    const int64_t warps = ((int64_t)gridDim.x - copy_from) * (blockDim.x >> 5), me = ((int64_t)blockIdx.x - copy_from) * (blockDim.x >> 5) + warp;
    if (p.copy_rest && me >= 0) {
        const int64_t from = p.M * me / warps, to = p.M * (me + 1) / warps;
        warp_visit_dropped_rows(p.keep_rows, M_keep, from, to, lane, [&](int64_t base, uint32_t todo) {
            // eight rows at a time, 32 vectors of each: their loads before their stores
            constexpr int kB = 8;
            while (todo) {
                int64_t at[kB];
#pragma unroll
                for (int b = 0; b < kB; ++b) {
                    at[b] = todo ? (base + __ffs(todo) - 1) * p.vecs : -1;
                    todo &= todo - 1;
                }
                for (int v0 = lane; v0 < p.vecs; v0 += 32) {
                    uint4 v[kB];
#pragma unroll
                    for (int b = 0; b < kB; ++b) v[b] = at[b] >= 0 && p.dR != nullptr ? __ldcg(p.dR + at[b] + v0) : zero;
#pragma unroll
                    for (int b = 0; b < kB; ++b) {
                        if (at[b] < 0) continue;
                        f32x2 f[P];
                        Vec<T>::unpack(v[b], f);
#pragma unroll
                        for (int e = 0; e < P; ++e) f[e] = mul(f[e], pair(p.scale, p.scale));
                        p.dH[at[b] + v0] = Vec<T>::pack(f);
                    }
                }
            }
        });
    }
}

// Adds the blocks' partial rows in a fixed order - 32 columns a block, slice i of 16 takes rows i, i + 16, ..., and the slices are added
// as a tree - and, for a gate of several rows, the workers' partial rows of each: the same, or, where a gate row has few workers,
// 256 columns of two gate rows a block.  (Blocks of 1024 threads, one an SM: 12544 of 25088 x 768 with 128 gate rows 59.7 us, 58.2 so.)
constexpr int kReduceThreads = 512, kReduceSlices = kReduceThreads / 32, kReduceGates = kReduceThreads / 256;
struct NormReduceParams {
    const float *sums, *gate_sums;
    float* out[kNormSums];
    float* dgate;                                     // of several rows, else nullptr
    const int32_t *keep_rows, *M_keep_dev, *status_word;
    int64_t M, M_keep_cap, workers, gate_group, gate_rows;
    int C, accumulate, blocks, few_workers, tiles, gate_tiles;       // column tiles of a sum / of a gate row
    int outputs, output[kNormSums];                                  // which of the sums are wanted
};
__device__ __forceinline__ float add_rows(const float* from, int64_t stride, int64_t n) {
    float s = 0.f;
    for (int64_t i = 0; i < n; i += 8) {              // eight loads together, the last ones too
        float f[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) f[u] = i + u < n ? __ldg(from + (i + u) * stride) : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += f[u];
    }
    return s;
}
// First positions of the ascending list whose entries are at least value[0], value[1]: two searches as warp_lower_bound's, side by side.
__device__ __forceinline__ void warp_lower_bounds(const int32_t* rows, int64_t n, const int64_t (&value)[2], int lane, int64_t (&lo)[2]) {
    int64_t hi[2] = {n, n};
    lo[0] = lo[1] = 0;
    while (hi[0] > lo[0] || hi[1] > lo[1]) {
        bool below[2];
        int64_t step[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            step[u] = (hi[u] - lo[u] + 31) / 32;
            const int64_t at = lo[u] + lane * step[u];
            below[u] = at < hi[u] && (int64_t)__ldg(rows + at) < value[u];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int c = __popc(__ballot_sync(0xffffffffu, below[u]));
            if (hi[u] <= lo[u]) continue;
            const int64_t last = lo[u] + (c - 1) * step[u];          // below
            const int64_t end = c == 0 || step[u] == 1 ? 0 : last + step[u];
            if (c != 0) lo[u] = last + 1;
            hi[u] = end == 0 ? lo[u] : end < hi[u] ? end : hi[u];
        }
    }
}
__global__ void __launch_bounds__(kReduceThreads) norm_reduce_kernel(const NormReduceParams p) {
    __shared__ float part[kReduceThreads];
    pdl_launch_dependents();
    pdl_wait();
    if (block_sees_error(p.status_word)) return;
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    float *out = nullptr, s = 0.f;
    int64_t c;
    bool tree = true;
    if (blockIdx.x < (unsigned)(p.outputs * p.tiles)) {
        const int k = p.output[blockIdx.x / p.tiles];
        out = p.out[k];
        c = (int64_t)(blockIdx.x % p.tiles) * 32 + lane;
        if (c < p.C && slice < p.blocks)
            s = add_rows(p.sums + ((int64_t)k * p.blocks + slice) * p.C + c, (int64_t)kReduceSlices * p.C, (p.blocks - slice + kReduceSlices - 1) / kReduceSlices);
    } else {
        const int64_t M_keep = load_m_keep(p.M_keep_dev, p.M_keep_cap), chunk = norm_chunk(M_keep, p.workers);
        const int64_t id = (int64_t)blockIdx.x - p.outputs * p.tiles;
        int64_t group = id / p.gate_tiles, step = kReduceSlices, start = slice;
        c = id % p.gate_tiles * 32 + lane;
        if (p.few_workers) {
            tree = false;
            group = group * kReduceGates + (threadIdx.x >> 8);
            c = id % p.gate_tiles * 256 + (threadIdx.x & 255);
            step = 1;
            start = 0;
        }
        if (group < p.gate_rows) {
            // the kept rows [a, b) of this gate row (without entries past the tensor), and the workers that had them
            const int64_t r0 = group * p.gate_group, r1 = r0 + p.gate_group < p.M ? r0 + p.gate_group : p.M;
            int64_t at[2];
            if (p.keep_rows == nullptr) {
                at[0] = r0 < M_keep ? r0 : M_keep;
                at[1] = r1 < M_keep ? r1 : M_keep;
            } else {
                const int64_t rows[2] = {r0, r1};
                warp_lower_bounds(p.keep_rows, M_keep, rows, lane, at);
            }
            const int64_t a = at[0], b = at[1];
            const int64_t w0 = a < b ? (uint32_t)a / (uint32_t)chunk : 0, w1 = a < b ? (uint32_t)(b - 1) / (uint32_t)chunk + 1 : 0;
            // inside one worker's rows it is already written
            if (!(w1 - w0 == 1 && a > w0 * chunk && b < (w0 + 1) * chunk && b < M_keep)) out = p.dgate + group * p.C;
            // a worker that begins before this gate row has it as its last one, the others as their first
            const float* from = p.gate_sums + c;
            const int64_t inner = w0 + (a < b && w0 * chunk < a ? 1 : 0);
            if (out != nullptr && c < p.C) {
                if (inner > w0 && start == 0) s = __ldg(from + (w0 * 2 + 1) * p.C);
                if (inner + start < w1) s += add_rows(from + (inner + start) * 2 * p.C, step * 2 * p.C, (w1 - inner - start + step - 1) / step);
            }
        }
    }
    if (tree) {
        part[threadIdx.x] = s;
        for (int h = kReduceSlices / 2; h > 0; h /= 2) {
            __syncthreads();
            if (slice < h) part[threadIdx.x] += part[threadIdx.x + h * 32];
        }
        if (slice != 0) return;
        s = part[threadIdx.x];
    }
    if (out != nullptr && c < p.C) out[c] = s + (p.accumulate ? out[c] : 0.f);
}

// ---- host ----
// (a gate row of M rows or more is the only one)
inline FastDiv group_div(const void* gate, int64_t gate_group, int64_t M) { return FastDiv(gate == nullptr ? 1u : (uint32_t)(gate_group < M ? gate_group : M)); }

struct NormShape {
    int vecs, nv, lanes, warps, per;                  // vectors of a row, of a thread; lanes of a row (0: warps of it); numbers of a vector
};
// Eight numbers a thread up to 1024 channels (backward: 4096): several rows a warp up to 128 channels, several warps a row from 256
// on.  (Rows of up to 1024 channels in one warp, up to 32 numbers a thread, take fewer instructions but leave registers for 14
// warps an SM, which spend ten cycles an instruction: 25088 x 768 forward 52 us.)  Beyond, 16 or 32 numbers.
inline NormShape norm_shape(sbp_dtype dt, int64_t C, bool backward) {
    NormShape s;
    s.per = dt == SBP_BF16 ? 8 : 4;
    s.vecs = (int)(C / s.per);
    s.lanes = C <= 64 ? 8 : C <= 128 ? 16 : C <= 256 ? 32 : 0;
    s.nv = C <= (backward ? 4096 : 1024) ? 8 / s.per : backward && dt == SBP_BF16 ? 2 : 4;
    s.warps = s.lanes > 0 ? 1 : (s.vecs + 32 * s.nv - 1) / (32 * s.nv);
    return s;
}
inline bool norm_many_warps(const NormShape& s) { return s.warps > 4; }
// Backward blocks: as many workers as the sums of one leave room for in shared memory, up to 16 warps
constexpr size_t kNormSmem = 200 * 1024;
static_assert(kNormSmem >= (size_t)kNormSums * kNormMaxC * 4, "the sums of one worker");
inline int norm_per_block(const NormShape& s, int sums) {
    const int threads = s.lanes > 0 ? s.lanes : 32 * s.warps;
    const size_t bytes = (size_t)threads * (sums > 0 ? sums : 1) * s.nv * s.per * 4;
    int64_t n = (int64_t)(kNormSmem / bytes);
    const int most = norm_backward_threads(s.nv * s.per, norm_many_warps(s)) / threads;
    if (n > most) n = most;
    if (s.lanes > 0) n = n / (32 / s.lanes) * (32 / s.lanes);        // whole warps
    else if (n > (norm_many_warps(s) ? 1 : kNormMostWorkers)) n = norm_many_warps(s) ? 1 : kNormMostWorkers;
    return n < 1 ? 1 : (int)n;
}

struct NormGrid {
    int blocks, per_block;
    int64_t workers;
};
// a block an SM; few rows: as many workers as rows (or as a quarter of the rows outside the list, which they copy), over the blocks evenly
inline NormGrid norm_grid(const NormShape& s, int sums, int64_t M, int64_t M_keep_cap) {
    NormGrid g;
    if ((M - M_keep_cap + 3) / 4 > M_keep_cap) M_keep_cap = (M - M_keep_cap + 3) / 4;
    g.per_block = norm_per_block(s, sums);
    const int64_t step = s.lanes > 0 ? 32 / s.lanes : 1;             // workers of a warp
    const int64_t each = (M_keep_cap + kNumSMs - 1) / kNumSMs, even = (each + step - 1) / step * step;
    if (even < g.per_block) g.per_block = even < step ? (int)step : (int)even;
    const int64_t blocks = (M_keep_cap + g.per_block - 1) / g.per_block;
    g.blocks = (int)(blocks < 1 ? 1 : blocks < kNumSMs ? blocks : kNumSMs);
    g.workers = (int64_t)g.blocks * g.per_block;
    return g;
}

template <typename T, int kNV, int kLanes, bool kMany, bool kFull, typename Params>
cudaError_t launch_norm(const Params& p, bool layer, bool post, dim3 grid, dim3 block, size_t smem, cudaStream_t stream) {
    auto with = [&](auto layer_c, auto post_c) {
        if constexpr (std::is_same_v<Params, NormFwdParams>) {
            return launch_pdl(norm_forward_kernel<T, kNV, kLanes, kFull, decltype(layer_c)::value, decltype(post_c)::value>, grid, block, smem, stream, p);
        } else {
            constexpr auto kernel = norm_backward_kernel<T, kNV, kLanes, kMany, kFull, decltype(layer_c)::value, decltype(post_c)::value>;
            const cudaError_t e = opt_in_dynamic_smem<kernel>((int)kNormSmem);
            return e == cudaSuccess ? launch_pdl(kernel, grid, block, smem, stream, p) : e;
        }
    };
    if (layer) return post ? with(std::true_type(), std::true_type()) : with(std::true_type(), std::false_type());
    return post ? with(std::false_type(), std::true_type()) : with(std::false_type(), std::false_type());
}
// the shapes that norm_shape makes
template <typename T, typename Params>
cudaError_t pick_norm(const NormShape& s, const Params& p, bool layer, bool post, dim3 grid, dim3 block, size_t smem, cudaStream_t stream) {
    constexpr bool kBackward = std::is_same_v<Params, NormBwdParams>, kWide = std::is_same_v<T, float>;
    const bool full = s.vecs == s.nv * (s.lanes > 0 ? s.lanes : 32 * s.warps);
    auto with = [&](auto nv, auto lanes, auto many) {
        return full ? launch_norm<T, decltype(nv)::value, decltype(lanes)::value, decltype(many)::value, true>(p, layer, post, grid, block, smem, stream)
                    : launch_norm<T, decltype(nv)::value, decltype(lanes)::value, decltype(many)::value, false>(p, layer, post, grid, block, smem, stream);
    };
    constexpr std::integral_constant<int, kWide ? 2 : 1> eight;      // vectors of eight numbers
    const std::false_type few;
    if (s.lanes == 8) return with(eight, std::integral_constant<int, 8>(), few);
    if (s.lanes == 16) return with(eight, std::integral_constant<int, 16>(), few);
    if (s.lanes == 32) return with(eight, std::integral_constant<int, 32>(), few);
    const std::integral_constant<int, 0> warps;
    if constexpr (kBackward) {
        const std::true_type many;
        if (s.nv == eight) return norm_many_warps(s) ? with(eight, warps, many) : with(eight, warps, few);
        return with(std::integral_constant<int, kWide ? 4 : 2>(), warps, many);
    } else {
        return s.nv == eight ? with(eight, warps, few) : with(std::integral_constant<int, 4>(), warps, few);
    }
}

}  // namespace

int64_t block_norm_max_channels() { return kNormMaxC; }

cudaError_t launch_block_norm_forward(sbp_dtype dt, bool layer, const void* H, const void* Y, const float* post_w, const float* post_b,
                                      const void* gate, int64_t gate_group, float scale, const float* pre_w, const float* pre_b, float eps,
                                      int64_t M, int64_t C, void* R, void* Z, const int32_t* keep_rows, const int32_t* M_keep_dev,
                                      int64_t M_keep_cap, void* Y_keep, void* R_keep, void* Z_keep, const int32_t* status_word,
                                      cudaStream_t stream) {
    const NormShape s = norm_shape(dt, C, false);
    NormFwdParams p = {};
    p.H = (const uint4*)H;
    p.Y = (const uint4*)Y;
    p.post_w = post_w;
    p.post_b = post_b;
    p.pre_w = pre_w;
    p.pre_b = pre_b;
    p.gate = (const uint4*)gate;
    p.gate_group = group_div(gate, gate_group, M);
    p.R = (uint4*)R;
    p.Z = (uint4*)Z;
    p.Y_keep = (uint4*)Y_keep;
    p.R_keep = (uint4*)R_keep;
    p.Z_keep = (uint4*)Z_keep;
    p.keep_rows = keep_rows;
    p.M_keep_dev = M_keep_dev;
    p.M_keep_cap = M_keep_cap;
    p.caches = Y_keep != nullptr || R_keep != nullptr || Z_keep != nullptr;
    p.status_word = status_word;
    p.M = M;
    p.vecs = s.vecs;
    p.scale = scale;
    p.eps = eps;
    p.inv_c = 1.f / (float)C;
    // rows a warp (a block, for long rows): enough of them for several waves, and never more rows than the mask of kept rows has bits
    const bool multi = s.lanes == 0;
    const int64_t groups = multi ? 1 : 32 / s.lanes, waves = M / (groups * kNumSMs * (multi ? 4 : 48));
    const int64_t chunk = groups * (waves >= 4 ? 4 : waves >= 2 ? 2 : 1), workers = (M + chunk - 1) / chunk;
    p.chunk = (int)chunk;
    const int per_block = multi ? 1 : 8;
    const dim3 grid((unsigned)((workers + per_block - 1) / per_block)), block(32 * (multi ? s.warps : per_block));
    return dt == SBP_BF16 ? pick_norm<__nv_bfloat16>(s, p, layer, post_w != nullptr, grid, block, 0, stream)
                          : pick_norm<float>(s, p, layer, post_w != nullptr, grid, block, 0, stream);
}

size_t block_norm_backward_workspace_bytes(sbp_dtype dt, int64_t M, int64_t M_keep_cap, int64_t C) {
    // (fewer sums leave room for more workers a block)
    const NormShape s = norm_shape(dt, C, true);
    size_t most = 0;
    for (int sums = 1; sums <= kNormSums; ++sums) {
        const NormGrid g = norm_grid(s, sums, M, M_keep_cap);
        const size_t rows = (size_t)kNormSums * g.blocks + 2 * (size_t)g.workers;
        most = rows > most ? rows : most;
    }
    return most * (size_t)C * sizeof(float);
}

cudaError_t launch_block_norm_backward(sbp_dtype dt, bool layer, const void* dR, const void* dZ, const void* R_keep, const void* Y_keep,
                                       const float* post_w, const float* post_b, const void* gate, int64_t gate_group, float scale,
                                       const float* pre_w, float eps, const int32_t* keep_rows, const int32_t* M_keep_dev, int64_t M,
                                       int64_t M_keep_cap, int64_t C, void* dH, void* dY, float* dpost_w, float* dpost_b, float* dgate,
                                       float* dpre_w, float* dpre_b, bool accumulate, float* workspace, const int32_t* status_word,
                                       cudaStream_t stream) {
    const NormShape s = norm_shape(dt, C, true);
    NormBwdParams p = {};
    p.dR = (const uint4*)dR;
    p.dZ = (const uint4*)dZ;
    p.R_keep = (const uint4*)R_keep;
    p.Y_keep = (const uint4*)Y_keep;
    p.post_w = post_w;
    p.post_b = post_b;
    p.pre_w = pre_w;
    p.gate = (const uint4*)gate;
    p.gate_group = group_div(gate, gate_group, M);
    p.dH = (uint4*)dH;
    p.dY = (uint4*)dY;
    p.keep_rows = keep_rows;
    p.M_keep_dev = M_keep_dev;
    p.status_word = status_word;
    p.M = M;
    p.M_keep_cap = M_keep_cap;
    p.dgate = dgate;
    p.want = (dpost_w ? 1 : 0) | (dpost_b ? 2 : 0) | (dpre_w ? 4 : 0) | (dpre_b ? 8 : 0) | (dgate ? 16 : 0);
    if (gate_group > M) gate_group = M;
    const int64_t gate_rows = dgate != nullptr ? (M + gate_group - 1) / gate_group : 0;
    p.one_gate = gate_rows == 1;
    int sums = 0;
    for (int k = 0; k < kNormSums; ++k) sums += p.want >> k & 1;
    const NormGrid g = norm_grid(s, sums, M, M_keep_cap);
    p.per_block = g.per_block;
    p.workers = g.workers;
    p.blocks = g.blocks;
    p.sums = workspace;
    p.gate_sums = workspace + (size_t)kNormSums * g.blocks * C;
    p.vecs = s.vecs;
    p.warps = s.warps;
    p.accumulate = accumulate;
    p.copy_rest = dH != nullptr && !(dH == dR && scale == 1.f);
    p.scale = scale;
    p.eps = eps;
    p.inv_c = 1.f / (float)C;
    const int threads = s.lanes > 0 ? s.lanes : 32 * s.warps;
    const size_t smem = (size_t)g.per_block * threads * sums * s.nv * s.per * 4;
    // few rows leave SMs free: blocks there copy the rows outside the list meanwhile
    const int64_t idle = p.copy_rest && M > M_keep_cap && g.blocks < kNumSMs ? kNumSMs - g.blocks : 0, wanted_copies = (M + 3) / 4;
    const dim3 grid((unsigned)(g.blocks + (idle < wanted_copies ? idle : wanted_copies))), block((unsigned)(g.per_block * threads));
    const bool post = post_w != nullptr;
    const cudaError_t e = dt == SBP_BF16 ? pick_norm<__nv_bfloat16>(s, p, layer, post, grid, block, smem, stream)
                                         : pick_norm<float>(s, p, layer, post, grid, block, smem, stream);
    if (e != cudaSuccess || p.want == 0) return e;
    NormReduceParams r = {};
    r.sums = p.sums;
    r.gate_sums = p.gate_sums;
    r.out[0] = dpost_w;
    r.out[1] = dpost_b;
    r.out[2] = dpre_w;
    r.out[3] = dpre_b;
    r.out[4] = p.one_gate ? dgate : nullptr;
    r.dgate = p.one_gate ? nullptr : dgate;
    r.keep_rows = keep_rows;
    r.M_keep_dev = M_keep_dev;
    r.status_word = status_word;
    r.M = M;
    r.M_keep_cap = M_keep_cap;
    r.workers = p.workers;
    r.gate_group = gate_group;
    r.gate_rows = p.one_gate ? 0 : gate_rows;
    r.C = (int)C;
    r.accumulate = accumulate;
    r.blocks = g.blocks;
    for (int k = 0; k < kNormSums; ++k)
        if (r.out[k] != nullptr) r.output[r.outputs++] = k;
    r.few_workers = r.gate_rows > 0 && p.workers / r.gate_rows <= 16;
    r.tiles = (int)((C + 31) / 32);
    r.gate_tiles = r.few_workers ? (int)((C + 255) / 256) : r.tiles;
    const int64_t blocks = (int64_t)r.outputs * r.tiles + (r.few_workers ? (r.gate_rows + kReduceGates - 1) / kReduceGates : r.gate_rows) * r.gate_tiles;
    return launch_pdl(norm_reduce_kernel, dim3((unsigned)blocks), dim3(kReduceThreads), 0, stream, r);
}

}  // namespace sbp
