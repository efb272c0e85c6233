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
#include "row_math.cuh"
#include "zero_rows.cuh"

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
    int64_t gate_group;
    int vecs, warps, chunk;                           // 16-byte vectors of a row; warps that share a row; rows of a worker
    float scale, eps, inv_c;
    int caches;
};

// A worker (a warp, or a block where a row is long) takes `chunk` <= 32 consecutive rows, kU at a time; a thread holds kNV vectors
// of each.  Which of the rows are kept, and the place of each in the caches, comes from one search of the list a chunk.
template <typename T, int kNV, int kU, bool kMulti, bool kLayer, bool kPost>
__global__ void __launch_bounds__(kMulti ? 512 : 256, kMulti ? 1 : 2)
norm_forward_kernel(const NormFwdParams p) {
    constexpr int VN = Vec<T>::N;
    constexpr int E = kNV * VN;
    __shared__ float scratch[kMulti ? 2 * 32 * kU : 1];
    pdl_launch_dependents();
    pdl_wait();
    if (p.status_word != nullptr && *reinterpret_cast<const volatile int32_t*>(p.status_word) != 0) return;
    const int lane = threadIdx.x & 31;
    const int64_t worker = kMulti ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int64_t workers = kMulti ? (int64_t)gridDim.x : (int64_t)gridDim.x * (blockDim.x >> 5);
    const int t = kMulti ? (int)threadIdx.x : lane, threads = kMulti ? (int)blockDim.x : 32;
    const int64_t M_keep = p.caches ? load_m_keep(p.M_keep_dev, p.M_keep_cap) : 0;
    const int64_t lo = worker * p.chunk, hi = lo + p.chunk < p.M ? lo + p.chunk : p.M;
    int turn = 0;

    if (lo < hi) {
        uint32_t kept = 0u;                           // bit d: row lo + d is in the list
        int64_t place = 0;                            // of the first of them
        if (p.caches) {
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
        for (int64_t row0 = lo; row0 < hi; row0 += kU) {
            float x[kU][E];
            uint4 yq[kU][kNV], hq[kU][kNV];
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int v = t + j * threads;
                    const bool in = v < p.vecs && row0 + u < hi;
                    yq[u][j] = in && p.Y != nullptr ? ld_row(p.Y + (row0 + u) * p.vecs + v) : make_uint4(0u, 0u, 0u, 0u);
                    hq[u][j] = in && p.H != nullptr ? ld_row(p.H + (row0 + u) * p.vecs + v) : make_uint4(0u, 0u, 0u, 0u);
                }
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < kNV; ++j) Vec<T>::unpack(yq[u][j], &x[u][j * VN]);
            auto normalise = [&](const float* w, const float* b) {
                float s[kU];
                if constexpr (kLayer) {
#pragma unroll
                    for (int u = 0; u < kU; ++u) {
                        s[u] = 0.f;
#pragma unroll
                        for (int e = 0; e < E; ++e) s[u] += x[u][e];
                    }
                    row_sums<kU, kMulti>(s, scratch, p.warps, turn);
#pragma unroll
                    for (int u = 0; u < kU; ++u)
#pragma unroll
                        for (int j = 0; j < kNV; ++j) {
                            const float mean = t + j * threads < p.vecs ? s[u] * p.inv_c : 0.f;     // threads past the row hold zeros
#pragma unroll
                            for (int e = 0; e < VN; ++e) x[u][j * VN + e] -= mean;
                        }
                }
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    s[u] = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) s[u] = fmaf(x[u][e], x[u][e], s[u]);
                }
                row_sums<kU, kMulti>(s, scratch, p.warps, turn);
#pragma unroll
                for (int u = 0; u < kU; ++u) s[u] = rsqrtf(fmaf(s[u], p.inv_c, p.eps));
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int v = t + j * threads;
                    if (v >= p.vecs) continue;
                    float wf[VN], bf[VN];
                    load_f32<VN>(w + v * VN, wf);
                    if (b != nullptr) load_f32<VN>(b + v * VN, bf);
#pragma unroll
                    for (int u = 0; u < kU; ++u)
#pragma unroll
                        for (int e = 0; e < VN; ++e) {
                            const float n = x[u][j * VN + e] * s[u];
                            x[u][j * VN + e] = b != nullptr ? fmaf(n, wf[e], bf[e]) : n * wf[e];
                        }
                }
            };
            if constexpr (kPost) normalise(p.post_w, p.post_b);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int64_t row = row0 + u;
                const bool live = row < hi;
                const bool keep = live && (kept >> (int)(row - lo) & 1u);
                const int64_t slot = place + __popc(kept & ((1u << (int)((row - lo) & 31)) - 1u));
                const uint4* gate = p.gate != nullptr && live ? p.gate + row / p.gate_group * p.vecs : nullptr;
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int v = t + j * threads;
                    if (v >= p.vecs || !live) continue;
                    float h[VN];
                    Vec<T>::unpack(hq[u][j], h);
                    if (gate != nullptr) {
                        float g[VN];
                        Vec<T>::unpack(__ldg(gate + v), g);
#pragma unroll
                        for (int e = 0; e < VN; ++e) x[u][j * VN + e] *= g[e];
                    }
                    if (p.H != nullptr) {
#pragma unroll
                        for (int e = 0; e < VN; ++e) x[u][j * VN + e] = fmaf(p.scale, h[e], x[u][j * VN + e]);
                    }
                    const uint4 r = Vec<T>::pack(&x[u][j * VN]);
                    if (p.R != nullptr) p.R[row * p.vecs + v] = r;
                    if (keep) {
                        if (p.R_keep != nullptr) p.R_keep[slot * p.vecs + v] = r;
                        if (p.Y_keep != nullptr) p.Y_keep[slot * p.vecs + v] = yq[u][j];
                    }
                }
            }
            if (p.pre_w != nullptr) {
                normalise(p.pre_w, p.pre_b);
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    const int64_t row = row0 + u;
                    const bool keep = row < hi && (kept >> (int)(row - lo) & 1u);
                    const int64_t slot = place + __popc(kept & ((1u << (int)((row - lo) & 31)) - 1u));
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        const int v = t + j * threads;
                        if (v >= p.vecs || row >= hi) continue;
                        const uint4 z = Vec<T>::pack(&x[u][j * VN]);
                        if (p.Z != nullptr) p.Z[row * p.vecs + v] = z;
                        if (keep && p.Z_keep != nullptr) p.Z_keep[slot * p.vecs + v] = z;
                    }
                }
            }
        }
    }
    // rows past M_keep of the caches are cleared
    if (p.caches) {
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        for (int64_t m = M_keep + worker; m < p.M_keep_cap; m += workers)
            for (int v = t; v < p.vecs; v += threads) {
                if (p.Y_keep != nullptr) p.Y_keep[m * p.vecs + v] = zero;
                if (p.R_keep != nullptr) p.R_keep[m * p.vecs + v] = zero;
                if (p.Z_keep != nullptr) p.Z_keep[m * p.vecs + v] = zero;
            }
    }
}

// ---- backward ----
struct NormBwdParams {
    const uint4 *dR, *dZ, *R_keep, *Y_keep;
    const float *post_w, *post_b, *pre_w;
    const uint4* gate;
    uint4 *dH, *dY;
    const int32_t *keep_rows, *M_keep_dev, *status_word;
    int64_t M, M_keep_cap, gate_group;
    float* dgate;
    float* sums;                                      // [kNormSums][workers][C]: dw_post, db_post, dw_pre, db_pre
    float* gate_sums;                                 // [workers][2][C]: first and last gate row of each worker
    int64_t workers;
    int want;                                         // bits 0..3: those sums; 4: dgate
    int vecs, warps, accumulate, copy_rest;
    float scale, eps, inv_c;
};
constexpr int kNormSums = 4;

__device__ __forceinline__ int64_t norm_chunk(int64_t M_keep, int64_t workers) { return (M_keep + workers - 1) / workers; }

// A worker takes consecutive kept rows, kU at a time; a thread holds the same kNV vectors of every row, so that its share of
// the weights' gradients stays in registers and leaves once, as a partial row that a second launch adds up.  The gate's
// gradient is a sum over the rows of one gate row; the list is ascending, so a gate row's rows are consecutive: the sum is put
// away when the gate row changes - straight into dgate where no other worker has rows of it (all but a worker's first and
// last gate row).
template <typename T, int kNV, int kU, bool kMulti, bool kLayer, bool kPost>
__global__ void __launch_bounds__(kMulti ? 512 : 128, kMulti ? 1 : 4)
norm_backward_kernel(const NormBwdParams p) {
    constexpr int VN = Vec<T>::N;
    constexpr int E = kNV * VN;
    __shared__ float scratch[kMulti ? 2 * 32 * 3 * kU : 1];
    pdl_launch_dependents();
    pdl_wait();
    if (p.status_word != nullptr && *reinterpret_cast<const volatile int32_t*>(p.status_word) != 0) return;
    const int lane = threadIdx.x & 31;
    const int64_t worker = kMulti ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int t = kMulti ? (int)threadIdx.x : lane, threads = kMulti ? (int)blockDim.x : 32;
    const int64_t M_keep = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const int64_t chunk = norm_chunk(M_keep, p.workers);
    const int64_t lo = worker * chunk < M_keep ? worker * chunk : M_keep, hi = lo + chunk < M_keep ? lo + chunk : M_keep;
    int turn = 0;

    if (worker < p.workers && lo < hi) {
        float acc[kNormSums][E], gacc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
            for (int k = 0; k < kNormSums; ++k) acc[k][e] = 0.f;
            gacc[e] = 0.f;
        }
        const bool want_gate = p.want & 16;
        int64_t first = 0, last = 0, cur = 0;
        if (p.gate != nullptr) {
            first = cur = mapped_row(p.keep_rows, lo) / p.gate_group;
            last = mapped_row(p.keep_rows, hi - 1) / p.gate_group;
        }
        const int64_t C = (int64_t)p.vecs * VN;
        auto put_gate = [&]() {
            const bool partial = cur == first || cur == last;
            float* to = partial ? p.gate_sums + (worker * 2 + (cur == first ? 0 : 1)) * C : p.dgate + cur * C;
            const bool add = !partial && p.accumulate;
#pragma unroll
            for (int j = 0; j < kNV; ++j) {
                const int v = t + j * threads;
                if (v >= p.vecs) continue;
#pragma unroll
                for (int e = 0; e < VN; e += 4) {
                    float4* q = reinterpret_cast<float4*>(to + (int64_t)v * VN + e);
                    float4 s = make_float4(gacc[j * VN + e], gacc[j * VN + e + 1], gacc[j * VN + e + 2], gacc[j * VN + e + 3]);
                    if (add) {
                        const float4 old = *q;
                        s.x += old.x;
                        s.y += old.y;
                        s.z += old.z;
                        s.w += old.w;
                    }
                    *q = s;
                }
            }
#pragma unroll
            for (int e = 0; e < E; ++e) gacc[e] = 0.f;
        };
        for (int64_t m0 = lo; m0 < hi; m0 += kU) {
            int64_t row[kU];
            uint4 rq[kU][kNV], yq[kU][kNV], zq[kU][kNV], dq[kU][kNV];
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                row[u] = m0 + u < hi ? (int64_t)mapped_row(p.keep_rows, m0 + u) : -1;
                if (row[u] >= p.M) row[u] = -1;
            }
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int v = t + j * threads;
                    const bool in = v < p.vecs && row[u] >= 0;
                    rq[u][j] = in && p.dZ != nullptr ? ld_row(p.R_keep + (m0 + u) * p.vecs + v) : zero;
                    zq[u][j] = in && p.dZ != nullptr ? ld_row(p.dZ + (m0 + u) * p.vecs + v) : zero;
                    yq[u][j] = in && p.Y_keep != nullptr ? ld_row(p.Y_keep + (m0 + u) * p.vecs + v) : zero;
                    dq[u][j] = in && p.dR != nullptr ? ld_row(p.dR + row[u] * p.vecs + v) : zero;
                }
            float x[kU][E], y[kU][E], g[kU][E];        // R, then what its norm makes of it; Y likewise; gradients
            float wpre[E];
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    Vec<T>::unpack(rq[u][j], &x[u][j * VN]);
                    Vec<T>::unpack(yq[u][j], &y[u][j * VN]);
                    Vec<T>::unpack(zq[u][j], &g[u][j * VN]);
                }
#pragma unroll
            for (int j = 0; j < kNV; ++j) {
                const int v = t + j * threads;
#pragma unroll
                for (int e = 0; e < VN; ++e) wpre[j * VN + e] = 0.f;
                if (v < p.vecs && p.dZ != nullptr) load_f32<VN>(p.pre_w + v * VN, &wpre[j * VN]);
            }
            float s1[3 * kU], s2[3 * kU];
            if constexpr (kLayer) {
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    s1[3 * u] = s1[3 * u + 1] = s1[3 * u + 2] = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        s1[3 * u] += x[u][e];
                        if constexpr (kPost) s1[3 * u + 1] += y[u][e];
                        s1[3 * u + 2] = fmaf(g[u][e], wpre[e], s1[3 * u + 2]);
                    }
                }
                row_sums<3 * kU, kMulti>(s1, scratch, p.warps, turn);
#pragma unroll
                for (int u = 0; u < kU; ++u)
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        const bool in = t + j * threads < p.vecs;            // threads past the row hold zeros, and keep them
                        const float mx = in ? s1[3 * u] * p.inv_c : 0.f, my = in ? s1[3 * u + 1] * p.inv_c : 0.f;
#pragma unroll
                        for (int e = 0; e < VN; ++e) {
                            x[u][j * VN + e] -= mx;
                            if constexpr (kPost) y[u][j * VN + e] -= my;
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                s2[3 * u] = s2[3 * u + 1] = s2[3 * u + 2] = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s2[3 * u] = fmaf(x[u][e], x[u][e], s2[3 * u]);
                    if constexpr (kPost) s2[3 * u + 1] = fmaf(y[u][e], y[u][e], s2[3 * u + 1]);
                    s2[3 * u + 2] = fmaf(g[u][e] * wpre[e], x[u][e], s2[3 * u + 2]);
                }
            }
            row_sums<3 * kU, kMulti>(s2, scratch, p.warps, turn);
            float s3[2 * kU], rstd_y[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const float rstd = rsqrtf(fmaf(s2[3 * u], p.inv_c, p.eps));
                rstd_y[u] = kPost ? rsqrtf(fmaf(s2[3 * u + 1], p.inv_c, p.eps)) : 1.f;
                const float mg = kLayer ? s1[3 * u + 2] * p.inv_c : 0.f;
                const float mgx = s2[3 * u + 2] * rstd * p.inv_c;             // mean of g n
                s3[2 * u] = s3[2 * u + 1] = 0.f;
                if (row[u] < 0) continue;
                if (p.gate != nullptr && row[u] / p.gate_group != cur) {
                    if (want_gate) put_gate();
                    cur = row[u] / p.gate_group;
                }
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int v = t + j * threads;
                    if (v >= p.vecs) continue;
                    float d[VN];
                    Vec<T>::unpack(dq[u][j], d);
#pragma unroll
                    for (int e = 0; e < VN; ++e) {
                        const int i = j * VN + e;
                        const float n = x[u][i] * rstd, dz = g[u][i];
                        acc[2][i] = fmaf(dz, n, acc[2][i]);
                        acc[3][i] += dz;
                        float q = dz * wpre[i];
                        if (p.dZ != nullptr) d[e] = fmaf(rstd, q - mg - n * mgx, d[e]);
                        g[u][i] = d[e];                                        // the whole gradient with respect to R
                        d[e] *= p.scale;
                    }
                    if (p.dH != nullptr) p.dH[row[u] * p.vecs + v] = Vec<T>::pack(d);
                    float wp[VN], bp[VN], gt[VN];
                    if constexpr (kPost) {
                        load_f32<VN>(p.post_w + v * VN, wp);
                        if (p.post_b != nullptr) load_f32<VN>(p.post_b + v * VN, bp);
                    }
                    if (p.gate != nullptr) Vec<T>::unpack(__ldg(p.gate + cur * p.vecs + v), gt);
#pragma unroll
                    for (int e = 0; e < VN; ++e) {
                        const int i = j * VN + e;
                        const float n = y[u][i] * rstd_y[u];
                        if (p.gate != nullptr) {
                            float un = n;
                            if constexpr (kPost) un = p.post_b != nullptr ? fmaf(n, wp[e], bp[e]) : n * wp[e];
                            gacc[i] = fmaf(g[u][i], un, gacc[i]);
                            g[u][i] *= gt[e];
                        }
                        if constexpr (kPost) {
                            acc[0][i] = fmaf(g[u][i], n, acc[0][i]);
                            acc[1][i] += g[u][i];
                            y[u][i] = n;
                            g[u][i] *= wp[e];
                            s3[2 * u] += g[u][i];
                            s3[2 * u + 1] = fmaf(g[u][i], n, s3[2 * u + 1]);
                        }
                    }
                }
            }
            if constexpr (kPost) row_sums<2 * kU, kMulti>(s3, scratch, p.warps, turn);
            if (p.dY != nullptr) {
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    if (m0 + u >= hi) continue;
                    const float mq = kLayer ? s3[2 * u] * p.inv_c : 0.f, mqn = s3[2 * u + 1] * p.inv_c;
#pragma unroll
                    for (int j = 0; j < kNV; ++j) {
                        const int v = t + j * threads;
                        if (v >= p.vecs) continue;
                        if constexpr (kPost) {
#pragma unroll
                            for (int e = 0; e < VN; ++e) {
                                const int i = j * VN + e;
                                g[u][i] = rstd_y[u] * (g[u][i] - mq - y[u][i] * mqn);
                            }
                        }
                        p.dY[(m0 + u) * p.vecs + v] = Vec<T>::pack(&g[u][j * VN]);
                    }
                }
            }
        }
        if (want_gate) put_gate();
#pragma unroll
        for (int k = 0; k < kNormSums; ++k) {
            if (!(p.want >> k & 1)) continue;
            float* to = p.sums + ((int64_t)k * p.workers + worker) * C;
#pragma unroll
            for (int j = 0; j < kNV; ++j) {
                const int v = t + j * threads;
                if (v >= p.vecs) continue;
#pragma unroll
                for (int e = 0; e < VN; e += 4)
                    *reinterpret_cast<float4*>(to + (int64_t)v * VN + e) =
                        make_float4(acc[k][j * VN + e], acc[k][j * VN + e + 1], acc[k][j * VN + e + 2], acc[k][j * VN + e + 3]);
            }
        }
    }
    if (worker >= p.workers) return;
    if (p.dY != nullptr) {                            // rows past M_keep are cleared
        for (int64_t m = M_keep + worker; m < p.M_keep_cap; m += p.workers)
            for (int v = t; v < p.vecs; v += threads) p.dY[m * p.vecs + v] = make_uint4(0u, 0u, 0u, 0u);
    }
    // the rows outside the list take the residual's gradient alone; every warp has its share of all rows
    if (p.copy_rest) {
        const int64_t warps = p.workers * p.warps, warp = kMulti ? worker * p.warps + (threadIdx.x >> 5) : worker;
        const int64_t from = p.M * warp / warps, to = p.M * (warp + 1) / warps;
        warp_visit_dropped_rows(p.keep_rows, M_keep, from, to, lane, [&](int64_t base, uint32_t todo) {
            while (todo) {
                const int64_t r = base + __ffs(todo) - 1;
                todo &= todo - 1;
                constexpr int kB = 4;
                for (int v0 = lane; v0 < p.vecs; v0 += 32 * kB) {
                    uint4 q[kB];
#pragma unroll
                    for (int b = 0; b < kB; ++b)
                        q[b] = v0 + 32 * b < p.vecs && p.dR != nullptr ? ld_row(p.dR + r * p.vecs + v0 + 32 * b) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int b = 0; b < kB; ++b) {
                        if (v0 + 32 * b >= p.vecs) continue;
                        float f[VN];
                        Vec<T>::unpack(q[b], f);
#pragma unroll
                        for (int e = 0; e < VN; ++e) f[e] *= p.scale;
                        p.dH[r * p.vecs + v0 + 32 * b] = Vec<T>::pack(f);
                    }
                }
            }
        });
    }
}

// Adds the workers' partial rows in a fixed order.  A block makes 256 / slices columns of one output: slice i takes partial rows
// i, i + slices, ..., and the slices are added as a tree.
struct NormReduceParams {
    const float *sums, *gate_sums;
    float* out[kNormSums];
    float* dgate;
    const int32_t *keep_rows, *M_keep_dev, *status_word;
    int64_t M_keep_cap, workers, groups, gate_group;
    int C, accumulate, slices, gate_slices, sum_tiles, gate_tiles;       // column tiles of a sum / of a gate row
};
__global__ void __launch_bounds__(256) norm_reduce_kernel(const NormReduceParams p) {
    __shared__ float part[256];
    pdl_launch_dependents();
    pdl_wait();
    if (p.status_word != nullptr && *reinterpret_cast<const volatile int32_t*>(p.status_word) != 0) return;
    const int64_t M_keep = load_m_keep(p.M_keep_dev, p.M_keep_cap);
    const int64_t chunk = norm_chunk(M_keep, p.workers);
    const int64_t used = chunk > 0 ? (M_keep + chunk - 1) / chunk : 0;
    const bool is_sum = blockIdx.x < (unsigned)(kNormSums * p.sum_tiles);
    const int slices = is_sum ? p.slices : p.gate_slices;
    const int cols = 256 / slices, col = threadIdx.x % cols, slice = threadIdx.x / cols;
    float* out;
    int64_t w0, w1, a = 0, c0;
    int64_t group = -1;
    if (is_sum) {
        const int k = blockIdx.x / p.sum_tiles;
        out = p.out[k];
        if (out == nullptr) return;
        c0 = (int64_t)(blockIdx.x % p.sum_tiles) * cols;
        w0 = 0;
        w1 = used;
        a = k;
    } else {
        const int64_t id = (int64_t)blockIdx.x - kNormSums * p.sum_tiles;
        group = id / p.gate_tiles;
        c0 = id % p.gate_tiles * cols;
        out = p.dgate + group * p.C;
        // the kept rows [a, b) of this gate row, and the workers that had them
        const int64_t r0 = group * p.gate_group, r1 = r0 + p.gate_group;
        int64_t b;
        if (p.keep_rows == nullptr) {
            a = r0 < M_keep ? r0 : M_keep;
            b = r1 < M_keep ? r1 : M_keep;
        } else {
            a = warp_lower_bound(p.keep_rows, M_keep, r0, threadIdx.x & 31);
            b = warp_lower_bound(p.keep_rows, M_keep, r1, threadIdx.x & 31);
        }
        w0 = a < b ? a / chunk : 0;
        w1 = a < b ? (b - 1) / chunk + 1 : 0;
        if (w1 - w0 == 1 && a > w0 * chunk && b < (w0 + 1) * chunk && b < M_keep) return;       // inside one worker's rows: already written
    }
    const int64_t c = c0 + col;
    float s = 0.f;
    if (c < p.C) {
#pragma unroll 8
        for (int64_t w = w0 + slice; w < w1; w += slices) {
            // a worker that begins before this gate row has it as its last one
            const float* from = is_sum ? p.sums + (a * p.workers + w) * p.C : p.gate_sums + (w * 2 + (w * chunk < a ? 1 : 0)) * p.C;
            s += __ldg(from + c);
        }
    }
    part[threadIdx.x] = s;
    for (int h = slices / 2; h > 0; h /= 2) {
        __syncthreads();
        if (slice < h) part[threadIdx.x] += part[threadIdx.x + h * cols];
    }
    if (slice == 0 && c < p.C) out[c] = part[threadIdx.x] + (p.accumulate ? out[c] : 0.f);
}

// ---- host ----
constexpr int kNormMaxC = 8192;

struct NormShape {
    int vecs, nv, warps;                              // vectors of a row, vectors a thread holds, warps a row
};
// most vectors a thread holds: forward 32 bf16 or 16 fp32 numbers (a warp a row up to 1024 bf16 or 512 fp32 channels), backward
// 8 numbers, which leave room for the five sums, and 16 only where a row would need more than sixteen warps
inline NormShape norm_shape(sbp_dtype dt, int64_t C, bool backward) {
    NormShape s;
    const int per = dt == SBP_BF16 ? 8 : 4;
    s.vecs = (int)(C / per);
    if (!backward) {
        s.nv = 4;
        s.warps = s.vecs <= 128 ? 1 : (s.vecs + 127) / 128;
        if (s.warps == 1) s.nv = (s.vecs + 31) / 32;
    } else {
        s.nv = dt == SBP_BF16 ? 1 : 2;
        if (s.vecs <= 32) s.nv = 1;
        if ((s.vecs + 32 * s.nv - 1) / (32 * s.nv) > 16) s.nv *= 2;
        s.warps = (s.vecs + 32 * s.nv - 1) / (32 * s.nv);
    }
    return s;
}
inline int64_t norm_backward_workers(const NormShape& s, int64_t M_keep_cap) {
    const int64_t most = (int64_t)kNumSMs * (s.warps == 1 ? 16 : s.warps < 16 ? 16 / s.warps : 1);
    const int64_t want = (M_keep_cap + 1) / 2;
    return want < 1 ? 1 : want < most ? want : most;
}

template <typename T, int kNV, int kU, bool kMulti>
cudaError_t launch_norm_forward(const NormFwdParams& p, bool layer, bool post, dim3 grid, dim3 block, cudaStream_t stream) {
    if (layer)
        return post ? launch_pdl(norm_forward_kernel<T, kNV, kU, kMulti, true, true>, grid, block, 0, stream, p)
                    : launch_pdl(norm_forward_kernel<T, kNV, kU, kMulti, true, false>, grid, block, 0, stream, p);
    return post ? launch_pdl(norm_forward_kernel<T, kNV, kU, kMulti, false, true>, grid, block, 0, stream, p)
                : launch_pdl(norm_forward_kernel<T, kNV, kU, kMulti, false, false>, grid, block, 0, stream, p);
}
template <typename T>
cudaError_t pick_norm_forward(const NormShape& s, const NormFwdParams& p, bool layer, bool post, dim3 grid, dim3 block, cudaStream_t stream) {
    if (s.warps > 1) return launch_norm_forward<T, 4, 1, true>(p, layer, post, grid, block, stream);
    switch (s.nv) {
        case 1: return launch_norm_forward<T, 1, 4, false>(p, layer, post, grid, block, stream);
        case 2: return launch_norm_forward<T, 2, 2, false>(p, layer, post, grid, block, stream);
        case 3: return launch_norm_forward<T, 3, 1, false>(p, layer, post, grid, block, stream);
        default: return launch_norm_forward<T, 4, 1, false>(p, layer, post, grid, block, stream);
    }
}
template <typename T, int kNV, bool kMulti>
cudaError_t launch_norm_backward_kernel(const NormBwdParams& p, bool layer, bool post, dim3 grid, dim3 block, cudaStream_t stream) {
    constexpr int kU = kNV * Vec<T>::N <= 4 ? 2 : 1;
    if (layer)
        return post ? launch_pdl(norm_backward_kernel<T, kNV, kU, kMulti, true, true>, grid, block, 0, stream, p)
                    : launch_pdl(norm_backward_kernel<T, kNV, kU, kMulti, true, false>, grid, block, 0, stream, p);
    return post ? launch_pdl(norm_backward_kernel<T, kNV, kU, kMulti, false, true>, grid, block, 0, stream, p)
                : launch_pdl(norm_backward_kernel<T, kNV, kU, kMulti, false, false>, grid, block, 0, stream, p);
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
    p.gate_group = gate_group;
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
    p.warps = s.warps;
    p.scale = scale;
    p.eps = eps;
    p.inv_c = 1.f / (float)C;
    const int per_block = s.warps > 1 ? 1 : 8;
    // rows a worker: enough workers for several waves, and never more rows than the mask of kept rows has bits
    const int64_t chunk = s.warps > 1 ? 1 : M >= 4 * 148 * 24 ? 4 : M >= 2 * 148 * 24 ? 2 : 1;
    p.chunk = (int)chunk;
    const int64_t workers = (M + chunk - 1) / chunk;
    const dim3 grid((unsigned)((workers + per_block - 1) / per_block)), block(32 * (s.warps > 1 ? s.warps : per_block));
    return dt == SBP_BF16 ? pick_norm_forward<__nv_bfloat16>(s, p, layer, post_w != nullptr, grid, block, stream)
                          : pick_norm_forward<float>(s, p, layer, post_w != nullptr, grid, block, stream);
}

size_t block_norm_backward_workspace_bytes(sbp_dtype dt, int64_t M_keep_cap, int64_t C) {
    return (size_t)norm_backward_workers(norm_shape(dt, C, true), M_keep_cap) * (kNormSums + 2) * (size_t)C * sizeof(float);
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
    p.gate_group = gate_group;
    p.dH = (uint4*)dH;
    p.dY = (uint4*)dY;
    p.keep_rows = keep_rows;
    p.M_keep_dev = M_keep_dev;
    p.status_word = status_word;
    p.M = M;
    p.M_keep_cap = M_keep_cap;
    p.dgate = dgate;
    p.workers = norm_backward_workers(s, M_keep_cap);
    p.sums = workspace;
    p.gate_sums = workspace + (size_t)kNormSums * p.workers * C;
    p.want = (dpost_w ? 1 : 0) | (dpost_b ? 2 : 0) | (dpre_w ? 4 : 0) | (dpre_b ? 8 : 0) | (dgate ? 16 : 0);
    p.vecs = s.vecs;
    p.warps = s.warps;
    p.accumulate = accumulate;
    p.copy_rest = dH != nullptr && !(dH == dR && scale == 1.f);
    p.scale = scale;
    p.eps = eps;
    p.inv_c = 1.f / (float)C;
    const int per_block = s.warps > 1 ? 1 : 4;
    const dim3 grid((unsigned)((p.workers + per_block - 1) / per_block)), block(32 * (s.warps > 1 ? s.warps : per_block));
    const bool post = post_w != nullptr;
    cudaError_t e;
    if (dt == SBP_BF16) {
        e = s.warps == 1 ? launch_norm_backward_kernel<__nv_bfloat16, 1, false>(p, layer, post, grid, block, stream)
            : s.nv == 1  ? launch_norm_backward_kernel<__nv_bfloat16, 1, true>(p, layer, post, grid, block, stream)
                         : launch_norm_backward_kernel<__nv_bfloat16, 2, true>(p, layer, post, grid, block, stream);
    } else {
        e = s.warps == 1 ? (s.nv == 1 ? launch_norm_backward_kernel<float, 1, false>(p, layer, post, grid, block, stream)
                                      : launch_norm_backward_kernel<float, 2, false>(p, layer, post, grid, block, stream))
            : s.nv == 2  ? launch_norm_backward_kernel<float, 2, true>(p, layer, post, grid, block, stream)
                         : launch_norm_backward_kernel<float, 4, true>(p, layer, post, grid, block, stream);
    }
    if (e != cudaSuccess || p.want == 0) return e;
    NormReduceParams r = {};
    r.sums = p.sums;
    r.gate_sums = p.gate_sums;
    r.out[0] = dpost_w;
    r.out[1] = dpost_b;
    r.out[2] = dpre_w;
    r.out[3] = dpre_b;
    r.dgate = dgate;
    r.keep_rows = keep_rows;
    r.M_keep_dev = M_keep_dev;
    r.status_word = status_word;
    r.M_keep_cap = M_keep_cap;
    r.workers = p.workers;
    r.groups = dgate != nullptr ? (M + gate_group - 1) / gate_group : 0;
    r.gate_group = gate_group;
    r.C = (int)C;
    r.accumulate = accumulate;
    auto slices_for = [](int64_t rows) { return rows > 64 ? 32 : rows > 8 ? 8 : 1; };
    r.slices = slices_for(p.workers);
    r.gate_slices = r.groups > 0 ? slices_for(p.workers / r.groups) : 1;
    r.sum_tiles = (int)((C + 256 / r.slices - 1) / (256 / r.slices));
    r.gate_tiles = (int)((C + 256 / r.gate_slices - 1) / (256 / r.gate_slices));
    const int64_t blocks = (int64_t)kNormSums * r.sum_tiles + r.groups * r.gate_tiles;
    return launch_pdl(norm_reduce_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, r);
}

}  // namespace sbp
