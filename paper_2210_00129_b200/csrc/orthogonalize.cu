// Orthogonalising updates by Newton-Schulz products (the step that the Muon optimiser makes of a weight's gradient):
//
//   X = U / (|U| + eps),   then `steps` times   A = X X^T,  B = b A + c A^2,  X <- a X + B X        (a, b, c below)
//
// on the smaller side of U [rows, cols] (A = X^T X and X <- a X + X B where rows > cols).  A singular value s goes to
// a s + b s^3 + c s^5 each time, which after five steps has brought all but the smallest ones to between 0.7 and 1.2.
//
// Precision.  What the steps do to errors decides the number formats.  A small singular value grows by a factor a = 3.44 a step,
// and so does whatever rounding puts where U has none: rounding X to bf16 leaves 0.3 of the result's norm in wrong directions
// for a gradient of rank 20, to fp16 0.04.  But only the a X term does that - B X turns directions that X has.  So X is
// held as the sum of two fp16 numbers (22 bits), the a X term takes both, in fp32, and the products take the first.
// The diagonals of A and B carry most of what the products weigh and stay in fp32 beside them.  That leaves 1e-3 of the norm,
// half of what rounding the result to bf16 adds (512 x 512 normal: 0.75e-3; all products in bf16: 1e-2).  Results in fp32,
// and matrices with a side up to kExactSide (whose few roundings do not average out), take both numbers of every operand:
// three products instead of one, 1e-6.  There the tensor core's running sum, which it cuts short instead of rounding (7e-8 of
// it for each 64 deep block), is read out every kPartBlocks blocks and added up in fp32 registers, the small products first.
// X, A and B are held times 2^12, which keeps the small numbers of large matrices out of fp16's subnormals.
//
// Each product is one launch of a persistent kernel over 128 x 128 tiles of all matrices: TMA loads (either orientation of X
// is read in place), tcgen05.mma into two accumulators in turns, and an epilogue that forms the next operand from the sums.
// A and B are symmetric: only tiles on and above the diagonal are made, and stored both ways.
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

namespace sbp {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kUp = 4096.f, kDown = 1.f / 4096.f;                 // X, A and B are held times 2^12
constexpr int kExactSide = 128;
constexpr int kPartBlocks = 4;

constexpr int kTile = 128, kDeep = 64, kUmmaDeep = 16;
constexpr uint32_t kRow = 128;                                      // bytes of a 64 deep row
constexpr uint32_t kOperand = kTile * kRow, kHalfOperand = 64 * kRow;
constexpr int kStages = 4;
constexpr uint32_t kStage = 2 * kOperand;
constexpr uint32_t kStagingBytes = 32 * 64 * 4;                     // of an epilogue warp: 32 rows x 64 sums
constexpr uint32_t kMirrorBytes = 64 * 32 * 2;                      // the same tile the other way, fp16, twice
constexpr uint32_t kWarpBytes = kStagingBytes + 2 * kMirrorBytes;
constexpr uint32_t kOrthoSmem = kStages * kStage + 256 + 4 * kWarpBytes + 1024;
constexpr int kOrthoThreads = 192;                                  // 0-3 epilogue, 4 copies, 5 products
constexpr int kEpilogueBarrier = 1;

enum { kGram = 0, kPoly = 1, kStep = 2 };

struct OrthoControl {
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
    uint32_t tmem_slot;
    int abort_flag;
};
static_assert(sizeof(OrthoControl) <= 256, "control block");

struct OrthoParams {
    __half *X, *S;                   // planes [2 buffers][first, second][count][rows][ldx] and [A, B][first(, second)][count][m][ldm]
    float *diag_a, *diag_b;          // [count][ldm]
    void* out;                       // the last step's result [count][rows][cols], else nullptr
    int64_t x_plane, s_plane;        // elements of one matrix's plane
    int count, rows, cols, m, ldx, ldm;
    int buffer;                      // of X, read; the other one is written
    int s_planes;                    // 1, or 2 where A and B have their second numbers
    int tiles_i, tiles_j;            // of the result (symmetric ones: tiles_i each way)
    int blocks;                      // 64 deep blocks of the reduction
    int tall, out_bf16;
    float scale;
    int32_t* status_word;
};

struct OrthoTile {
    int matrix, i, j;
};
template <int kMode>
__device__ __forceinline__ OrthoTile ortho_tile(const OrthoParams& p, uint32_t q, uint32_t per) {
    OrthoTile t;
    t.matrix = (int)(q / per);
    uint32_t r = q - (uint32_t)t.matrix * per;
    if constexpr (kMode == kStep) {
        t.i = (int)(r / (uint32_t)p.tiles_j);
        t.j = (int)(r % (uint32_t)p.tiles_j);
    } else {                                                         // columns of the upper triangle: j + 1 tiles in column j
        int j = (int)((sqrtf(8.f * (float)r + 1.f) - 1.f) * 0.5f);
        while ((uint32_t)(j + 1) * (uint32_t)(j + 2) / 2 <= r) ++j;
        while ((uint32_t)j * (uint32_t)(j + 1) / 2 > r) --j;
        t.j = j;
        t.i = (int)(r - (uint32_t)j * (uint32_t)(j + 1) / 2);
    }
    return t;
}

__device__ __forceinline__ void unpack_half(const uint4& q, float* f) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
}
// the fp16 numbers nearest to f, and the rest of f
__device__ __forceinline__ uint4 pack_half(float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        const float2 r = __half22float2(v);
        f[2 * i] -= r.x;
        f[2 * i + 1] -= r.y;
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int kMode, bool kExact>
__global__ void __launch_bounds__(kOrthoThreads, 1)
ortho_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const OrthoParams p) {
    extern __shared__ uint8_t smem_raw[];
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t raw = ptx::smem_addr(smem_raw), ring = (raw + 1023u) & ~1023u;
    OrthoControl* ctl = reinterpret_cast<OrthoControl*>(smem_raw + (ring - raw) + kStages * kStage);

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(ptx::smem_addr(&ctl->full[s]), 1);
            ptx::mbar_init(ptx::smem_addr(&ctl->empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(ptx::smem_addr(&ctl->acc_full[a]), 1);
            ptx::mbar_init(ptx::smem_addr(&ctl->acc_empty[a]), 4);
        }
        ctl->abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&map_a);
        ptx::prefetch_tensormap(&map_b);
    }
    if (warp == 5) ptx::tmem_alloc(ptx::smem_addr(&ctl->tmem_slot), 2 * kTile);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&ctl->tmem_slot);
    volatile int* abort_flag = &ctl->abort_flag;
    int32_t* status_word = p.status_word;
    pdl_wait();
    const bool skip = status_word != nullptr && *reinterpret_cast<volatile int32_t*>(status_word) != 0;

    constexpr bool kSymmetric = kMode != kStep;
    const uint32_t per = kSymmetric ? (uint32_t)p.tiles_i * (uint32_t)(p.tiles_i + 1) / 2 : (uint32_t)p.tiles_i * (uint32_t)p.tiles_j;
    const uint32_t total = per * (uint32_t)p.count;
    // which operands are read across (their reduction runs along rows of X): both of a tall matrix's A, X of a wide one's step
    const bool across_a = kMode == kGram && p.tall, across_b = across_a || (kMode == kStep && !p.tall);
    // the parts of a tile's sum: (block, operands' planes) in the order of issue; exact: second x first, first x second, first x first
    const int terms = kExact ? 3 : 1;
    const int all_blocks = terms * p.blocks;
    const int small = kExact ? 2 * p.blocks : 0;                     // blocks of the small products, one part
    auto part_end = [&](int k) {                                     // whether block k is a part's last one
        if (k == all_blocks - 1) return true;
        return kExact && (k == small - 1 || (k >= small && (k - small) % kPartBlocks == kPartBlocks - 1));
    };

    if (skip) {
        // an earlier call failed: the outputs are left alone
    } else if (warp == 4) {
        const bool leader = ptx::elect_one();
        uint32_t it = 0;
        bool ok = true;
        for (uint32_t q = blockIdx.x; q < total && ok; q += gridDim.x) {
            const OrthoTile t = ortho_tile<kMode>(p, q, per);
            for (int k = 0; k < all_blocks; ++k, ++it) {
                const int term = kExact ? k / p.blocks : 2, y = (kExact ? k % p.blocks : k) * kDeep;
                const int second_a = term == 0 ? 1 : 0, second_b = term == 1 ? 1 : 0;
                int za, zb;
                if constexpr (kMode == kGram) {
                    za = (p.buffer * 2 + second_a) * p.count + t.matrix;
                    zb = (p.buffer * 2 + second_b) * p.count + t.matrix;
                } else if constexpr (kMode == kPoly) {
                    za = second_a * p.count + t.matrix;
                    zb = second_b * p.count + t.matrix;
                } else {
                    const int zx = (p.buffer * 2 + (p.tall ? second_a : second_b)) * p.count + t.matrix;
                    const int zs = (p.s_planes + (p.tall ? second_b : second_a)) * p.count + t.matrix;
                    za = p.tall ? zx : zs;
                    zb = p.tall ? zs : zx;
                }
                const int s = it % kStages;
                ok = ptx::mbar_wait(ptx::smem_addr(&ctl->empty[s]), ((it / kStages) & 1u) ^ 1u, abort_flag, status_word);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t full = ptx::smem_addr(&ctl->full[s]), a = ring + s * kStage, b = a + kOperand;
                if (leader) ptx::mbar_arrive_expect_tx(full, kStage);
                if (across_a) {
                    ptx::tma_load_3d_warp(a, &map_a, t.i * kTile, y, za, full, leader);
                    ptx::tma_load_3d_warp(a + kHalfOperand, &map_a, t.i * kTile + 64, y, za, full, leader);
                } else {
                    ptx::tma_load_3d_warp(a, &map_a, y, t.i * kTile, za, full, leader);
                }
                if (across_b) {
                    ptx::tma_load_3d_warp(b, &map_b, t.j * kTile, y, zb, full, leader);
                    ptx::tma_load_3d_warp(b + kHalfOperand, &map_b, t.j * kTile + 64, y, zb, full, leader);
                } else {
                    ptx::tma_load_3d_warp(b, &map_b, y, t.j * kTile, zb, full, leader);
                }
            }
        }
        if (!ok) {                                                   // let the copies already issued land before shared memory goes away
            for (uint32_t j = (it > (uint32_t)kStages ? it - kStages : 0u); j < it; ++j) {
                const uint32_t bar = ptx::smem_addr(&ctl->full[j % kStages]);
                for (int spin = 0; spin < (1 << 14); ++spin)
                    if (ptx::mbar_try_wait(bar, (j / kStages) & 1u)) break;
            }
        }
        __syncwarp();
    } else if (warp == 5) {
        const bool leader = ptx::elect_one();
        uint32_t it = 0, used = 0;
        bool ok = true;
        const uint32_t idesc = ptx::umma_idesc_f16(kTile, kTile, across_a, across_b);
        const uint32_t a_step = (across_a ? kUmmaDeep * kRow : kUmmaDeep * 2u) >> 4, b_step = (across_b ? kUmmaDeep * kRow : kUmmaDeep * 2u) >> 4;
        const uint32_t a_lo = ptx::umma_desc_lo(ring, across_a ? kHalfOperand : 16u);
        const uint32_t b_lo = ptx::umma_desc_lo(ring + kOperand, across_b ? kHalfOperand : 16u);
        for (uint32_t q = blockIdx.x; q < total && ok; q += gridDim.x) {
            bool fresh = true;
            for (int k = 0; k < all_blocks; ++k, ++it) {
                const uint32_t acc = used & 1u;
                if (fresh) {
                    ok = ptx::mbar_wait(ptx::smem_addr(&ctl->acc_empty[acc]), ((used >> 1) & 1u) ^ 1u, abort_flag, status_word);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                }
                const uint32_t s = it % kStages;
                ok = ptx::mbar_wait(ptx::smem_addr(&ctl->full[s]), (it / kStages) & 1u, abort_flag, status_word);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const uint32_t a = a_lo + s * (kStage >> 4), b = b_lo + s * (kStage >> 4);
#pragma unroll
                for (uint32_t u = 0; u < kDeep / kUmmaDeep; ++u)
                    ptx::umma_bf16_warp<false>(tmem + acc * kTile, ptx::umma_desc_of(a + u * a_step), ptx::umma_desc_of(b + u * b_step), idesc,
                                               !(fresh && u == 0u), leader);
                fresh = false;
                if (leader) ptx::umma_commit(ptx::smem_addr(&ctl->empty[s]));
                if (part_end(k)) {
                    if (leader) ptx::umma_commit(ptx::smem_addr(&ctl->acc_full[acc]));
                    ++used;
                    fresh = true;
                }
                __syncwarp();
            }
        }
        __syncwarp();
    } else {
        uint32_t used = 0;
        bool ok = true;
        uint8_t* staging = smem_raw + (ring - raw) + kStages * kStage + 256 + warp * kWarpBytes;
        uint8_t* mirror = staging + kStagingBytes;
        const int sub = lane >> 3, ch = lane & 7;
        auto take = [&](uint32_t& taddr) {                           // the next part's sums, once they are there
            const uint32_t acc = used & 1u;
            if (lane == 0) ok = ptx::mbar_wait(ptx::smem_addr(&ctl->acc_full[acc]), (used >> 1) & 1u, abort_flag, status_word);
            ok = !ptx::bar_or<kEpilogueBarrier, 128>(!ok);           // the four warps go on, or give up, together
            ptx::tc_fence_after_sync();
            taddr = tmem + acc * kTile + ((uint32_t)(warp * 32) << 16);
        };
        auto give_back = [&]() {
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&ctl->acc_empty[used & 1u]));
            ++used;
        };
        for (uint32_t q = blockIdx.x; q < total; q += gridDim.x) {
            const OrthoTile t = ortho_tile<kMode>(p, q, per);
            float sum[kExact ? kTile : 1];
            uint32_t taddr = 0;
            if constexpr (kExact) {
#pragma unroll
                for (int i = 0; i < kTile; ++i) sum[i] = 0.f;
                const int parts = 1 + (p.blocks + kPartBlocks - 1) / kPartBlocks;
                for (int part = 0; part < parts; ++part) {
                    take(taddr);
                    if (!ok) break;
#pragma unroll
                    for (int c = 0; c < kTile; c += 32) {
                        float v[32];
                        ptx::tmem_ld_32x32(taddr + c, v);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[c + i] += v[i];
                    }
                    give_back();
                }
            } else {
                take(taddr);
            }
            if (!ok) break;
            const int row0 = t.i * kTile + warp * 32, col0 = t.j * kTile;
            const int rows = kSymmetric ? p.m : p.rows, ld = kSymmetric ? p.ldm : p.ldx;
            __half* S = p.S + (int64_t)t.matrix * p.s_plane;         // (first numbers of A)
            const int64_t s_all = (int64_t)p.count * p.s_plane, x_all = (int64_t)p.count * p.x_plane;
#pragma unroll
            for (int c0 = 0; c0 < kTile; c0 += 64) {
                // a lane has one row of the accumulator: through shared memory into rows of eight lanes
                if constexpr (kExact) {
#pragma unroll
                    for (int g = 0; g < 16; ++g)
                        *reinterpret_cast<float4*>(staging + lane * 256 + ((g ^ (lane & 7)) << 4)) =
                            make_float4(sum[c0 + 4 * g], sum[c0 + 4 * g + 1], sum[c0 + 4 * g + 2], sum[c0 + 4 * g + 3]);
                } else {
                    float va[32], vb[32];
                    ptx::tmem_ld_32x32(taddr + c0, va);
                    ptx::tmem_ld_32x32(taddr + c0 + 32, vb);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        *reinterpret_cast<float4*>(staging + lane * 256 + ((g ^ (lane & 7)) << 4)) =
                            make_float4(va[4 * g], va[4 * g + 1], va[4 * g + 2], va[4 * g + 3]);
                        *reinterpret_cast<float4*>(staging + lane * 256 + (((g + 8) ^ (lane & 7)) << 4)) =
                            make_float4(vb[4 * g], vb[4 * g + 1], vb[4 * g + 2], vb[4 * g + 3]);
                    }
                    if (c0 + 64 == kTile) give_back();
                }
                __syncwarp();
                const int col = col0 + c0 + ch * 8;
#pragma unroll 2
                for (int i = 0; i < 8; ++i) {
                    const int r = i * 4 + sub, row = row0 + r;
                    float v[8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 f = *reinterpret_cast<const float4*>(staging + r * 256 + (((2 * ch + h) ^ (r & 7)) << 4));
                        v[4 * h] = f.x;
                        v[4 * h + 1] = f.y;
                        v[4 * h + 2] = f.z;
                        v[4 * h + 3] = f.w;
                    }
                    const bool in = row < rows && col < ld;          // (columns between the matrix's and its pitch are written and never read)
                    const int64_t at = (int64_t)row * ld + col;
                    if constexpr (kMode == kGram) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            v[e] *= kDown;                           // 2^24 A as it comes, 2^12 A as it is held
                            if (in && row == col + e) p.diag_a[(int64_t)t.matrix * p.ldm + row] = v[e] * kDown;
                        }
                    } else if constexpr (kMode == kPoly) {
                        float first[8] = {}, second[8] = {};
                        if (in) unpack_half(*reinterpret_cast<const uint4*>(S + at), first);
                        if (kExact && in) unpack_half(*reinterpret_cast<const uint4*>(S + s_all + at), second);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float a2 = v[e] * (kDown * kDown);
                            if (in && row == col + e) {
                                // the diagonal in fp32: A_ii as its product left it, and (A^2)_ii with that in A_ii's place
                                const float d = p.diag_a[(int64_t)t.matrix * p.ldm + row];
                                const float h = first[e] * kDown, l = kExact ? second[e] * kDown : 0.f;
                                p.diag_b[(int64_t)t.matrix * p.ldm + row] = kNsB * d + kNsC * (a2 + (d - h) * (d + h) - 2.f * h * l);
                                v[e] = 0.f;
                            } else {
                                v[e] = fmaf(kNsB, first[e] + second[e], kNsC * a2 * kUp);
                            }
                        }
                    } else {
                        float first[8] = {}, second[8] = {};
                        const __half* X = p.X + (int64_t)p.buffer * 2 * x_all + (int64_t)t.matrix * p.x_plane;
                        if (in) {
                            unpack_half(*reinterpret_cast<const uint4*>(X + at), first);
                            unpack_half(*reinterpret_cast<const uint4*>(X + x_all + at), second);
                        }
                        const float* diag = p.diag_b + (int64_t)t.matrix * p.ldm;
                        float f[8];
                        if (p.tall) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) f[e] = in ? kNsA + diag[col + e] : 0.f;      // (ld and ldm are the same here)
                        } else {
                            const float d = in ? kNsA + diag[row] : 0.f;
#pragma unroll
                            for (int e = 0; e < 8; ++e) f[e] = d;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = fmaf(f[e], second[e], fmaf(f[e], first[e], v[e] * kDown));
                    }
                    if constexpr (kMode == kStep) {
                        if (p.out != nullptr) {
                            if (row >= p.rows) continue;
                            const int64_t o = ((int64_t)t.matrix * p.rows + row) * p.cols + col;
                            const float k = p.scale * kDown;
                            if (p.out_bf16) {
                                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + o;
                                if (p.cols % 8 == 0) {
                                    if (col < p.cols) {
                                        uint32_t w[4];
#pragma unroll
                                        for (int e = 0; e < 4; ++e) {
                                            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e] * k, v[2 * e + 1] * k);
                                            w[e] = *reinterpret_cast<const uint32_t*>(&b);
                                        }
                                        *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
                                    }
                                } else {
#pragma unroll
                                    for (int e = 0; e < 8; ++e)
                                        if (col + e < p.cols) out[e] = __float2bfloat16_rn(v[e] * k);
                                }
                            } else {
                                float* out = static_cast<float*>(p.out) + o;
                                if (p.cols % 4 == 0) {
#pragma unroll
                                    for (int e = 0; e < 8; e += 4)
                                        if (col + e < p.cols)
                                            *reinterpret_cast<float4*>(out + e) = make_float4(v[e] * k, v[e + 1] * k, v[e + 2] * k, v[e + 3] * k);
                                } else {
#pragma unroll
                                    for (int e = 0; e < 8; ++e)
                                        if (col + e < p.cols) out[e] = v[e] * k;
                                }
                            }
                        } else if (in) {
                            __half* X = p.X + (int64_t)(p.buffer ^ 1) * 2 * x_all + (int64_t)t.matrix * p.x_plane;
                            *reinterpret_cast<uint4*>(X + at) = pack_half(v);
                            *reinterpret_cast<uint4*>(X + x_all + at) = pack_half(v);
                        }
                    } else {
                        __half* to = S + (kMode == kPoly ? p.s_planes * s_all : 0);
                        const uint4 first = pack_half(v);
                        uint4 second = make_uint4(0u, 0u, 0u, 0u);
                        if constexpr (kExact) second = pack_half(v);
                        if (in) {
                            *reinterpret_cast<uint4*>(to + at) = first;
                            if constexpr (kExact) *reinterpret_cast<uint4*>(to + s_all + at) = second;
                        }
                        if (t.i != t.j) {                            // the other way: 64 rows of 32, 16-byte pieces swizzled
                            const uint32_t a[4] = {first.x, first.y, first.z, first.w}, b[4] = {second.x, second.y, second.z, second.w};
                            uint8_t* m = mirror + (((r >> 3) ^ (ch & 3)) << 4) + (r & 7) * 2;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                *reinterpret_cast<uint16_t*>(m + (ch * 8 + e) * 64) = (uint16_t)(a[e >> 1] >> (16 * (e & 1)));
                                if constexpr (kExact)
                                    *reinterpret_cast<uint16_t*>(m + kMirrorBytes + (ch * 8 + e) * 64) = (uint16_t)(b[e >> 1] >> (16 * (e & 1)));
                            }
                        }
                    }
                }
                __syncwarp();
                if constexpr (kSymmetric) {
                    if (t.i != t.j) {
                        __half* to = S + (kMode == kPoly ? p.s_planes * s_all : 0);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int c = i * 8 + (lane >> 2), g = lane & 3;
                            const int row = col0 + c0 + c, at_col = row0 + g * 8;
                            const uint8_t* m = mirror + c * 64 + ((g ^ ((c >> 3) & 3)) << 4);
                            if (row < p.m && at_col < p.ldm) {
                                const int64_t at = (int64_t)row * p.ldm + at_col;
                                *reinterpret_cast<uint4*>(to + at) = *reinterpret_cast<const uint4*>(m);
                                if constexpr (kExact) *reinterpret_cast<uint4*>(to + s_all + at) = *reinterpret_cast<const uint4*>(m + kMirrorBytes);
                            }
                        }
                        __syncwarp();
                    }
                }
            }
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 5) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 2 * kTile);
    }
}

// ---- the start: momentum, the norm, the two fp16 numbers of U / (|U| + eps) ----
constexpr int kStartThreads = 256;
constexpr int kStartBlocksMost = 64;                                 // blocks a matrix

struct StartParams {
    const float* G;
    float* momentum;                 // nullable
    double* partial;                 // [count][blocks]: sums of squares
    __half* X;
    int64_t x_plane, elements;       // of a matrix: with pitch, without
    int count, rows, cols, ldx, blocks, nesterov;
    float beta;
    double eps;
    const int32_t* status_word;
};

__device__ __forceinline__ float updated(const StartParams& p, float g, float mom) {        // U from G and the averaged gradient
    return p.nesterov ? fmaf(p.beta, mom, g) : mom;
}

// Averages the gradients and adds up the squares of U, in 64 bits: no square overflows or is lost.
template <bool kVec>
__global__ void __launch_bounds__(kStartThreads) ortho_norm_kernel(const StartParams p) {
    __shared__ double part[kStartThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    if (p.status_word != nullptr && *reinterpret_cast<const volatile int32_t*>(p.status_word) != 0) return;
    const int matrix = blockIdx.y;
    const int64_t base = (int64_t)matrix * p.elements;
    double s = 0.0;
    auto one = [&](float g, float& mom) {
        float u = g;
        if (p.momentum != nullptr) {
            mom = fmaf(p.beta, mom, g);
            u = updated(p, g, mom);
        }
        s = fma((double)u, (double)u, s);
    };
    const int64_t stride = (int64_t)gridDim.x * kStartThreads;
    if constexpr (kVec) {
        const float4* G = reinterpret_cast<const float4*>(p.G + base);
        float4* mom = p.momentum != nullptr ? reinterpret_cast<float4*>(p.momentum + base) : nullptr;
#pragma unroll 4
        for (int64_t i = (int64_t)blockIdx.x * kStartThreads + threadIdx.x; i < p.elements / 4; i += stride) {
            const float4 g = __ldg(G + i);
            float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
            if (mom != nullptr) m = mom[i];
            one(g.x, m.x);
            one(g.y, m.y);
            one(g.z, m.z);
            one(g.w, m.w);
            if (mom != nullptr) mom[i] = m;
        }
    } else {
        for (int64_t i = (int64_t)blockIdx.x * kStartThreads + threadIdx.x; i < p.elements; i += stride) {
            float m = p.momentum != nullptr ? p.momentum[base + i] : 0.f;
            one(__ldg(p.G + base + i), m);
            if (p.momentum != nullptr) p.momentum[base + i] = m;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kStartThreads / 32; ++w) s += part[w];
        p.partial[(int64_t)matrix * p.blocks + blockIdx.x] = s;
    }
}

// Writes U / (|U| + eps) as two fp16 numbers.
__global__ void __launch_bounds__(kStartThreads) ortho_scale_kernel(const StartParams p) {
    pdl_launch_dependents();
    pdl_wait();
    if (p.status_word != nullptr && *reinterpret_cast<const volatile int32_t*>(p.status_word) != 0) return;
    const int matrix = blockIdx.y;
    double s = 0.0;
    for (int b = 0; b < p.blocks; ++b) s += p.partial[(int64_t)matrix * p.blocks + b];
    const double norm = sqrt(s) + p.eps;
    // 2^12 / norm as a power of two and a number near 2^12, each of which fp32 holds
    int e = norm > 0.0 && isfinite(norm) ? ilogb(norm) : 0;
    e = e > 126 ? 126 : e < -126 ? -126 : e;
    const float power = scalbnf(1.f, -e), factor = (float)(4096.0 / ldexp(norm, -e));
    const int64_t groups = (int64_t)p.rows * (p.ldx / 8);
    const float* G = p.G + (int64_t)matrix * p.elements;
    const float* mom = p.momentum != nullptr ? p.momentum + (int64_t)matrix * p.elements : nullptr;
    __half* X = p.X + (int64_t)matrix * p.x_plane;
    const int64_t second = (int64_t)p.count * p.x_plane;
    for (int64_t i = (int64_t)blockIdx.x * kStartThreads + threadIdx.x; i < groups; i += (int64_t)gridDim.x * kStartThreads) {
        const int row = (int)(i / (p.ldx / 8)), col = (int)(i % (p.ldx / 8)) * 8;
        const int64_t at = (int64_t)row * p.cols + col;
        float v[8];
        if (p.cols % 8 == 0) {
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const float4 g = __ldg(reinterpret_cast<const float4*>(G + at + h));
                float4 u = g;
                if (mom != nullptr) {
                    const float4 m = __ldg(reinterpret_cast<const float4*>(mom + at + h));
                    u = make_float4(updated(p, g.x, m.x), updated(p, g.y, m.y), updated(p, g.z, m.z), updated(p, g.w, m.w));
                }
                v[h] = u.x;
                v[h + 1] = u.y;
                v[h + 2] = u.z;
                v[h + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 8; ++h) {
                v[h] = 0.f;
                if (col + h >= p.cols) continue;
                const float g = __ldg(G + at + h);
                v[h] = mom != nullptr ? updated(p, g, __ldg(mom + at + h)) : g;
            }
        }
#pragma unroll
        for (int h = 0; h < 8; ++h) v[h] = v[h] * power * factor;
        *reinterpret_cast<uint4*>(X + (int64_t)row * p.ldx + col) = pack_half(v);
        *reinterpret_cast<uint4*>(X + second + (int64_t)row * p.ldx + col) = pack_half(v);
    }
}

// ---- host ----
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}
// fp16 [planes][rows][cols] with a pitch of ld elements, boxes of box_rows x 64, 128-byte swizzle, zeros outside the matrix
bool plane_map(CUtensorMap* map, const __half* base, int64_t planes, int64_t rows, int64_t cols, int64_t ld, uint32_t box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(rows * ld) * 2};
    const cuuint32_t box[3] = {64, box_rows, 1}, steps[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct OrthoLayout {
    int64_t m, ldx, ldm, x_plane, s_plane;
    int s_planes, start_blocks;
    bool exact;
    size_t S, diag_a, diag_b, partial, bytes;        // offsets behind the planes of X
};
OrthoLayout ortho_layout(sbp_dtype dt, int64_t count, int64_t rows, int64_t cols) {
    OrthoLayout l;
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    l.m = rows < cols ? rows : cols;
    l.ldx = (cols + 7) / 8 * 8;
    l.ldm = (l.m + 7) / 8 * 8;
    l.exact = dt == SBP_F32 || l.m <= kExactSide;
    l.s_planes = l.exact ? 2 : 1;
    l.x_plane = rows * l.ldx;
    l.s_plane = l.m * l.ldm;
    const int64_t want = (rows * cols / 4 + 4 * kStartThreads - 1) / (4 * kStartThreads);
    l.start_blocks = (int)(want < 1 ? 1 : want < kStartBlocksMost ? want : kStartBlocksMost);
    l.S = up((size_t)(4 * count * l.x_plane) * 2);
    l.diag_a = l.S + up((size_t)(2 * l.s_planes * count * l.s_plane) * 2);
    l.diag_b = l.diag_a + up((size_t)(count * l.ldm) * 4);
    l.partial = l.diag_b + up((size_t)(count * l.ldm) * 4);
    l.bytes = l.partial + up((size_t)count * l.start_blocks * 8);
    return l;
}

template <int kMode, bool kExact>
cudaError_t launch_product(const CUtensorMap& a, const CUtensorMap& b, const OrthoParams& p, cudaStream_t stream) {
    const cudaError_t e = opt_in_dynamic_smem<ortho_product_kernel<kMode, kExact>>((int)kOrthoSmem);
    if (e != cudaSuccess) return e;
    const int64_t per = kMode == kStep ? (int64_t)p.tiles_i * p.tiles_j : (int64_t)p.tiles_i * (p.tiles_i + 1) / 2, total = per * p.count;
    return launch_pdl(ortho_product_kernel<kMode, kExact>, dim3((unsigned)(total < kNumSMs ? total : kNumSMs)), dim3(kOrthoThreads), kOrthoSmem,
                      stream, a, b, p);
}

}  // namespace

size_t orthogonalize_workspace_bytes(sbp_dtype dt, int64_t count, int64_t rows, int64_t cols) { return ortho_layout(dt, count, rows, cols).bytes; }

// the tiles of a launch, and the planes a tensor map counts, are 32-bit numbers
bool orthogonalize_supported(int64_t count, int64_t rows, int64_t cols) {
    const int64_t tiles = (rows + kTile - 1) / kTile * ((cols + kTile - 1) / kTile);
    return rows <= (1 << 16) && cols <= (1 << 16) && count <= (1 << 16) - 1 && tiles * count < (1ll << 30);
}

cudaError_t launch_orthogonalize(sbp_dtype dt, const float* G, float* momentum, float beta, bool nesterov, int64_t count, int64_t rows, int64_t cols,
                                 int steps, double eps, float scale, void* O, void* workspace, int32_t* status_word, cudaStream_t stream) {
    const OrthoLayout l = ortho_layout(dt, count, rows, cols);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    StartParams s = {};
    s.G = G;
    s.momentum = momentum;
    s.partial = reinterpret_cast<double*>(ws + l.partial);
    s.X = reinterpret_cast<__half*>(ws);
    s.x_plane = l.x_plane;
    s.elements = rows * cols;
    s.count = (int)count;
    s.rows = (int)rows;
    s.cols = (int)cols;
    s.ldx = (int)l.ldx;
    s.blocks = l.start_blocks;
    s.nesterov = nesterov;
    s.beta = beta;
    s.eps = eps;
    s.status_word = status_word;
    const dim3 start_grid((unsigned)l.start_blocks, (unsigned)count);
    cudaError_t e = rows * cols % 4 == 0 ? launch_pdl(ortho_norm_kernel<true>, start_grid, dim3(kStartThreads), 0, stream, s)
                                         : launch_pdl(ortho_norm_kernel<false>, start_grid, dim3(kStartThreads), 0, stream, s);
    if (e != cudaSuccess) return e;
    if ((e = launch_pdl(ortho_scale_kernel, start_grid, dim3(kStartThreads), 0, stream, s)) != cudaSuccess) return e;

    OrthoParams p = {};
    p.X = s.X;
    p.S = reinterpret_cast<__half*>(ws + l.S);
    p.diag_a = reinterpret_cast<float*>(ws + l.diag_a);
    p.diag_b = reinterpret_cast<float*>(ws + l.diag_b);
    p.x_plane = l.x_plane;
    p.s_plane = l.s_plane;
    p.count = (int)count;
    p.rows = (int)rows;
    p.cols = (int)cols;
    p.m = (int)l.m;
    p.ldx = (int)l.ldx;
    p.ldm = (int)l.ldm;
    p.s_planes = l.s_planes;
    p.tall = rows > cols;
    p.out_bf16 = dt == SBP_BF16;
    p.scale = scale;
    p.status_word = status_word;
    CUtensorMap x_rows, x_across, s_rows;
    if (!plane_map(&x_rows, p.X, 4 * count, rows, cols, l.ldx, kTile) || !plane_map(&x_across, p.X, 4 * count, rows, cols, l.ldx, 64) ||
        !plane_map(&s_rows, p.S, 2 * l.s_planes * count, l.m, l.m, l.ldm, kTile))
        return cudaErrorUnknown;
    const CUtensorMap& gram = p.tall ? x_across : x_rows;
    const int tiles_m = (int)((l.m + kTile - 1) / kTile);
    for (int step = 0; step < steps; ++step) {
        p.buffer = step & 1;
        p.tiles_i = p.tiles_j = tiles_m;
        p.blocks = (int)(((p.tall ? rows : cols) + kDeep - 1) / kDeep);
        e = l.exact ? launch_product<kGram, true>(gram, gram, p, stream) : launch_product<kGram, false>(gram, gram, p, stream);
        if (e != cudaSuccess) return e;
        p.blocks = (int)((l.m + kDeep - 1) / kDeep);
        e = l.exact ? launch_product<kPoly, true>(s_rows, s_rows, p, stream) : launch_product<kPoly, false>(s_rows, s_rows, p, stream);
        if (e != cudaSuccess) return e;
        p.tiles_i = (int)((rows + kTile - 1) / kTile);
        p.tiles_j = (int)((cols + kTile - 1) / kTile);
        p.out = step == steps - 1 ? O : nullptr;
        const CUtensorMap &a = p.tall ? x_rows : s_rows, &b = p.tall ? s_rows : x_across;
        e = l.exact ? launch_product<kStep, true>(a, b, p, stream) : launch_product<kStep, false>(a, b, p, stream);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace sbp
