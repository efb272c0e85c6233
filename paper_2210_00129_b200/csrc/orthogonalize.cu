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
// three products instead of one: no further from 64 bits than the iteration in fp32 (533 x 1926 normal: 1.5e-6 and 3.3e-6 of the
// norm after five steps; rank 20: 1.5e-5 and 3.0e-5).  There the tensor core's running sum, which it cuts short instead of rounding
// (7e-8 of it for each 64 deep block), is read out every four blocks and added up in fp32 registers, the small products first.  On
// the diagonals of A and A^2 all terms have one sign, the cuts add up, and the steps grow what they leave (8.3e-6): the tiles there
// are read out twice a block (2 x 4096 x 1024 574 us -> 590; once a block 573 and 2.4e-6).
// X, A and B are held times 2^12, which keeps the small numbers of large matrices out of fp16's subnormals.
//
// All products of a call run in one launch of a persistent kernel.  Its items are the tiles of all products of all matrices, in the
// order step, product, matrix, tile; blocks draw the next one from a counter, and an item waits until the tiles of its matrix
// that it depends on are done (a count for each matrix).  Items only wait for items drawn before them, so some block can always
// go on, however many are resident.  With several matrices the tiles of others, and the products under an epilogue, hide part of
// the 7 us from a tile's stores to the first product that reads them, but not all of it: the chain of dependent products is the
// bound (12 of 768 x 768: 3 us of products a tile).  (One launch a product, seventeen a call, cost 8 us each before their first
// tile.)  Operands come by TMA, X in either
// orientation as it lies; tcgen05.mma into accumulators in turns; the epilogue forms the next operand from the sums.  A and B
// are symmetric: only tiles on and above the diagonal are made, and stored both ways.
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

#include <type_traits>

namespace sbp {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kUp = 4096.f, kDown = 1.f / 4096.f;                 // X, A and B are held times 2^12
constexpr int kExactSide = 128;

constexpr int kTile = 128, kDeep = 64, kUmmaDeep = 16;               // rows of a tile, depth of a stage and of an instruction
constexpr uint32_t kRow = 128;                                      // bytes of a 64 deep row
constexpr uint32_t kOperand = kTile * kRow, kHalfOperand = 64 * kRow;
constexpr int kCopyWarp = 0, kProductWarp = 1, kTellWarp = 2, kDrawWarp = 3, kFirstEpilogueWarp = 4;
constexpr uint32_t kStagingBytes = 32 * 1024;                       // of all epilogue warps
constexpr uint32_t kHalfBytes = 32 * 32 * 2;                        // 32 x 32 numbers in fp16
constexpr uint32_t kRing = 192 * 1024, kControl = 512;
constexpr uint32_t kOrthoSmem = kRing + kControl + kStagingBytes + 1024;
constexpr int kMostStages = 6, kItems = 4;

enum { kGram = 0, kPoly = 1, kStep = 2 };
// 16 deep products whose sum is read out together where both numbers of every operand are taken: two on the diagonal of A and its square
__device__ __forceinline__ int part_products(int mode, int i, int j) { return mode != kStep && i == j ? 2 : 16; }

struct alignas(16) OrthoControl {
    uint64_t full[kMostStages], empty[kMostStages];                  // a stage's operands: in place, read
    uint64_t acc_full[2], acc_empty[2], small_full[2], small_empty[2];
    uint64_t item_full[kItems], item_empty[kItems], stored[kItems];  // an item: drawn and ready, read by all, its tile written
    int4 item[kItems][2];            // its eight numbers
    uint32_t tmem_slot;
    int abort_flag;
};
static_assert(sizeof(OrthoControl) <= kControl, "control block");

struct OrthoParams {
    __half *X, *S;                   // planes [2 buffers][first, second][count][rows][ldx] and [A(, its second), B, its second][count][m][ldm]
    float *diag_a, *diag_b;          // [count][ldm]
    void* out;                       // the last step's result [count][rows][cols]
    uint32_t* drawn;                 // items drawn so far
    int32_t* done;                   // [count]: finished items of the matrix
    int32_t* shares;                 // [count][sym_tiles]: finished shares of A's tile that another item adds up
    float4* share;                   // [cuts - 1][count][sym_tiles][128 x 128 sums]
    int64_t x_plane, s_plane;        // elements of one matrix's plane
    int count, rows, cols, m, ldx, ldm, steps;
    int b_plane;                     // of B's first numbers: 1, or 2 where A has second ones
    uint32_t sym_tiles, step_tiles, step_cols;       // of a matrix: tiles of A or B, of X; columns of tiles of X
    int gram_blocks, m_blocks;       // 64 deep blocks of A's reduction, and of the others
    int cuts;                        // shares of A's reduction, where its tiles alone leave blocks idle
    int tall, out_bf16;
    float scale;
    int32_t* status_word;
};

// a product's tile: rows 128 i and columns kWidth j of matrix `matrix`'s A, B or next X
struct OrthoItem {
    int step, mode, matrix, i, j;
    int tile, cut;                   // A: which of the matrix's tiles, which share of its reduction
    int32_t need;                    // of done[matrix]; -1: there are no more items
};
template <int kWidth>
__device__ __forceinline__ OrthoItem ortho_item(const OrthoParams& p, uint32_t q) {
    OrthoItem t;
    const uint32_t gram_items = p.sym_tiles * (uint32_t)p.cuts, matrix_items = gram_items + p.sym_tiles + p.step_tiles;
    t.step = (int)(q / (matrix_items * (uint32_t)p.count));
    uint32_t r = q - (uint32_t)t.step * matrix_items * (uint32_t)p.count;
    t.need = (int)((uint32_t)t.step * matrix_items);
    t.cut = 0;
    const uint32_t grams = gram_items * (uint32_t)p.count, polys = p.sym_tiles * (uint32_t)p.count;
    if (r < grams + polys) {
        t.mode = r < grams ? kGram : kPoly;
        if (t.mode == kGram) {                                       // the shares of a tile one after the other: the last adds up
            t.matrix = (int)(r / gram_items);
            r -= (uint32_t)t.matrix * gram_items;
            t.cut = (int)(r % (uint32_t)p.cuts);
            r /= (uint32_t)p.cuts;
        } else {
            r -= grams;
            t.matrix = (int)(r / p.sym_tiles);
            r -= (uint32_t)t.matrix * p.sym_tiles;
            t.need += (int)gram_items;
        }
        t.tile = (int)r;
        // column j has the tiles that reach the diagonal or lie above it: 128 j .. wide tiles j + 1 of them, 256 wide ones 2 j + 2
        constexpr uint32_t kF = kWidth / kTile;
        uint32_t j = (uint32_t)((sqrtf(8.f / kF * (float)r + 1.f) - 1.f) * 0.5f);
        while (kF * (j + 1) * (j + 2) / 2 <= r) ++j;
        while (kF * j * (j + 1) / 2 > r) --j;
        t.j = (int)j;
        t.i = (int)(r - kF * j * (j + 1) / 2);
    } else {
        t.mode = kStep;
        r -= grams + polys;
        t.matrix = (int)(r / p.step_tiles);
        r -= (uint32_t)t.matrix * p.step_tiles;
        t.tile = (int)r;
        t.i = (int)(r / p.step_cols);
        t.j = (int)(r % p.step_cols);
        t.need += (int)(gram_items + p.sym_tiles);
    }
    return t;
}
// the 64 deep blocks [from, from + n) of an item's reduction
__device__ __forceinline__ int ortho_blocks(const OrthoParams& p, const OrthoItem& t, int& from) {
    from = t.mode == kGram ? p.gram_blocks * t.cut / p.cuts : 0;
    return t.mode == kGram ? p.gram_blocks * (t.cut + 1) / p.cuts - from : p.m_blocks;
}

// Waits (bounded, as every wait here) until `need` tiles of a matrix are finished; what they wrote is then visible to this
// thread, and to what it hands the item to, copies by TMA included.
__device__ __forceinline__ bool wait_done(const int32_t* done, int32_t need, volatile int* abort_flag, int32_t* status_word) {
    int32_t v;
    uint64_t t0 = 0;
    for (uint32_t spins = 0;; ++spins) {
        // (an acquiring load here, over and over, would empty the SM's L1 each time and hold up the other warps' loads)
        asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(done) : "memory");
        if (v >= need) break;
        __nanosleep(32);
        if (*abort_flag) return false;
        if (spins == 0) t0 = ptx::global_timer_ns();
        else if ((spins & 63u) == 0u && ptx::global_timer_ns() - t0 > ptx::kWaitLimitNs) {
            *abort_flag = 1;
            report_device_error(status_word, SBP_ERR_TIMEOUT);
            return false;
        }
    }
    asm volatile("fence.acq_rel.gpu;\n\tfence.proxy.async;" ::: "memory");
    return true;
}
// Block `k` of a tile's sum: which 64 deep block of the reduction, from which planes.  A step in fp16 makes B X, B = a + b A + c A^2,
// of the first numbers, and of the 128 rows and columns of B around its diagonal, whose second numbers are kept as well, also
// first x second and second x first: that is a X to 22 bits.  These, and the blocks of the diagonal itself, come last: the tensor
// core cuts its running sum, which is small until then.
struct OrthoBlock {
    int at;                          // 64 deep block
    int second_x, second_s;          // second numbers of X, of B
    int narrow;                      // 0: the tile's columns, 1 + h: columns 128 h .. + 127 of it
};
template <int kWidth>
__device__ __forceinline__ int step_extras(const OrthoParams& p) { return p.tall ? 4 * (kWidth / kTile) : 4; }
template <int kWidth>
__device__ __forceinline__ OrthoBlock step_block(const OrthoParams& p, const OrthoItem& t, int k) {
    constexpr int kF = kWidth / kTile;
    const int len = p.tall ? 2 * kF : 2, lo = p.tall ? 2 * kF * t.j : 2 * t.i, hi = lo + len < p.m_blocks ? lo + len : p.m_blocks;
    // (the first block has all columns of the tile: where there are no other blocks, the diagonal's come first)
    const int others = p.m_blocks - (hi - lo), extras = step_extras<kWidth>(p), first = others > 0 ? others : hi - lo;
    OrthoBlock b = {k < lo || others == 0 ? k : k + (hi - lo), 0, 0, 0};
    if (k >= first + extras) {
        b.at = lo + (k - first - extras);
    } else if (k >= first) {
        const int e = k - first;
        b.at = lo + (e >> 1);                                        // (past the matrix: zeros)
        b.second_x = e & 1;
        b.second_s = b.second_x ^ 1;
        if (p.tall && kF > 1) b.narrow = 1 + (e >> 2);
    }
    return b;
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

// eight numbers of a result's row, from column `col` on
__device__ __forceinline__ void put_result(const OrthoParams& p, int64_t row, int col, const float (&v)[8]) {
    const int64_t o = row * p.cols + col;
    const float k = p.scale * kDown;
    if (p.out_bf16) {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + o;
        if (p.cols % 8 == 0) {
            if (col >= p.cols) return;
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e] * k, v[2 * e + 1] * k);
                w[e] = *reinterpret_cast<const uint32_t*>(&b);
            }
            *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
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
                if (col + e < p.cols) *reinterpret_cast<float4*>(out + e) = make_float4(v[e] * k, v[e + 1] * k, v[e + 2] * k, v[e + 3] * k);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < p.cols) out[e] = v[e] * k;
        }
    }
}

// An accumulator's turns: which of two is next, and which of its phases.
struct Turns {
    uint32_t used = 0;
    __device__ __forceinline__ uint32_t slot() const { return used & 1u; }
    __device__ __forceinline__ uint32_t phase() const { return (used >> 1) & 1u; }
};

struct OrthoWarp {                   // what an epilogue warp works with
    OrthoControl* ctl;
    uint8_t* staging;
    volatile int* abort_flag;
    uint32_t tmem;                   // of its quarter of the accumulators' rows
    int lane, quad, half;
    Turns acc, small;
};

// Waits for the sums of the next part; hands back an accumulator that has been read.
__device__ __forceinline__ bool take_sums(OrthoWarp& w, uint64_t* full, const Turns& t, int32_t* status_word) {
    bool ok = true;
    if (w.lane == 0) ok = ptx::mbar_wait(ptx::smem_addr(&full[t.slot()]), t.phase(), w.abort_flag, status_word);
    ok = __all_sync(0xffffffffu, ok);
    ptx::tc_fence_after_sync();
    return ok;
}
__device__ __forceinline__ void give_back(OrthoWarp& w, uint64_t* empty, Turns& t) {
    ptx::tc_fence_before_sync();
    __syncwarp();
    if (w.lane == 0) ptx::mbar_arrive(ptx::smem_addr(&empty[t.slot()]));
    ++t.used;
}

// Shares of a tile of A: a warp's sums, 32 columns of a row a lane, to where the warp of the same place in the last share's item finds
// them; and those of all other shares added to that one's, in their order.
__device__ __forceinline__ float4* share_place(const OrthoParams& p, const OrthoItem& t, const OrthoWarp& w, int cut, int col) {
    const int64_t tile = ((int64_t)cut * p.count + t.matrix) * p.sym_tiles + t.tile;
    return p.share + tile * (kTile * kTile / 4) + (w.quad * 4 + col / 32) * (32 * 8) + w.lane;       // (col: of the tile, a multiple of 32)
}
template <int kFrom, int kSize>
__device__ __forceinline__ void put_share(const OrthoParams& p, const OrthoItem& t, const OrthoWarp& w, int col, const float (&v)[kSize]) {
    float4* to = share_place(p, t, w, t.cut, col);
#pragma unroll
    for (int g = 0; g < 8; ++g) to[g * 32] = make_float4(v[kFrom + 4 * g], v[kFrom + 4 * g + 1], v[kFrom + 4 * g + 2], v[kFrom + 4 * g + 3]);
}
template <int kFrom, int kSize>
__device__ __forceinline__ void add_shares(const OrthoParams& p, const OrthoItem& t, const OrthoWarp& w, int col, float (&v)[kSize]) {
    for (int cut = 0; cut < p.cuts - 1; ++cut) {
        const float4* from = share_place(p, t, w, cut, col);
        float4 q[8];
#pragma unroll
        for (int g = 0; g < 8; ++g) q[g] = __ldcg(from + g * 32);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            v[kFrom + 4 * g] += q[g].x;
            v[kFrom + 4 * g + 1] += q[g].y;
            v[kFrom + 4 * g + 2] += q[g].z;
            v[kFrom + 4 * g + 3] += q[g].w;
        }
    }
}
__device__ __forceinline__ bool wait_shares(const OrthoParams& p, const OrthoItem& t, const OrthoWarp& w) {
    bool ok = true;
    if (w.lane == 0)
        ok = wait_done(p.shares + (int64_t)t.matrix * p.sym_tiles + t.tile, (t.step + 1) * (p.cuts - 1), w.abort_flag, p.status_word);
    return __all_sync(0xffffffffu, ok);
}

// The epilogue of one tile by one warp where the products take both numbers of every operand: 32 rows, 64 columns, 32 at a time.
// The sums of the parts are added up in registers, then combined with numbers from memory.
template <int kMode>
__device__ __forceinline__ bool ortho_epilogue_exact(const OrthoParams& p, const OrthoItem& t, OrthoWarp& w) {
    constexpr bool kSymmetric = kMode != kStep;
    constexpr int kWidth = kTile, kCols = 64, kChunks = 2;
    const int lane = w.lane, sub = lane >> 2, ch = lane & 3;
    const int rows = kSymmetric ? p.m : p.rows, ld = kSymmetric ? p.ldm : p.ldx;
    const int row0 = t.i * kTile + w.quad * 32, col0 = t.j * kWidth + w.half * kCols;
    const int64_t s_all = (int64_t)p.count * p.s_plane, x_all = (int64_t)p.count * p.x_plane;
    __half* S = p.S + (int64_t)t.matrix * p.s_plane;                 // (first numbers of A)
    __half* X = p.X + (int64_t)t.matrix * p.x_plane;
    float* diag_a = p.diag_a + (int64_t)t.matrix * p.ldm;
    float* diag_b = p.diag_b + (int64_t)t.matrix * p.ldm;
    const __half* from = kMode == kPoly ? S : X + (int64_t)(t.step & 1) * 2 * x_all;
    __half* to = kMode == kGram ? S : kMode == kPoly ? S + p.b_plane * s_all : X + (int64_t)((t.step & 1) ^ 1) * 2 * x_all;
    const int64_t from_second = kMode == kPoly ? s_all : x_all, to_second = kMode == kStep ? x_all : s_all;
    constexpr bool kCombine = kMode != kGram;
    const bool last = kMode == kStep && t.step == p.steps - 1;
    const bool mirrored = kSymmetric && t.j > t.i;

    // what the sums are combined with is asked for a chunk ahead (columns between the matrix's and its pitch are written and never
    // read); past the L1, which may hold an earlier step's numbers
    uint4 first_q[2][4], second_q[2][4];
    float f[2][8];                                              // step: a + the diagonal of B; second product: the diagonal of A
    auto ask = [&](int c, int b) {
        const int col = col0 + c * 32 + ch * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + i * 8 + sub;
            const bool in = row < rows && col < ld;
            const int64_t at = (int64_t)row * ld + col;
            if constexpr (kCombine) first_q[b][i] = in ? __ldcg(reinterpret_cast<const uint4*>(from + at)) : make_uint4(0u, 0u, 0u, 0u);
            if constexpr (kCombine) second_q[b][i] = in ? __ldcg(reinterpret_cast<const uint4*>(from + from_second + at)) : make_uint4(0u, 0u, 0u, 0u);
            if (kMode == kStep && !p.tall) f[b][i] = in ? kNsA + __ldcg(diag_b + row) : 0.f;
            if (kMode == kPoly) f[b][i] = in && t.j == t.i ? __ldcg(diag_a + row) : 0.f;
        }
        if (kMode == kStep && p.tall) {                              // one for each column (ld and ldm are the same here)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[b][e] = col < ld ? kNsA + __ldcg(diag_b + col + e) : 0.f;
        }
    };
    if constexpr (kMode != kGram) {
        ask(0, 0);
    }
    float sum[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) sum[i] = 0.f;
    {
        int from_block;
        const int products = ortho_blocks(p, t, from_block) * (kDeep / kUmmaDeep), each = part_products(kMode, t.i, t.j);
        auto add = [&](uint32_t taddr) {
#pragma unroll
            for (int c = 0; c < kCols; c += 32) {
                float v[32];
                ptx::tmem_ld_32x32(taddr + c, v);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) sum[c + i] += v[i];
            }
        };
        for (int part = 0; part < products; part += each) {
            if (!take_sums(w, w.ctl->acc_full, w.acc, p.status_word)) return false;
            add(w.tmem + w.acc.slot() * kWidth + w.half * kCols);
            give_back(w, w.ctl->acc_empty, w.acc);
        }
        if (!take_sums(w, w.ctl->small_full, w.small, p.status_word)) return false;
        add(w.tmem + (2 + w.small.slot()) * kWidth + w.half * kCols);
        give_back(w, w.ctl->small_empty, w.small);
    }
    if constexpr (kMode == kGram) {
        if (t.cut < p.cuts - 1) {
            put_share<0>(p, t, w, w.half * kCols, sum);
            put_share<32>(p, t, w, w.half * kCols + 32, sum);
            return true;
        }
        if (p.cuts > 1) {
            if (!wait_shares(p, t, w)) return false;
            add_shares<0>(p, t, w, w.half * kCols, sum);
            add_shares<32>(p, t, w, w.half * kCols + 32, sum);
        }
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (kCombine && c + 1 < kChunks) ask(c + 1, c + 1);
        // a lane has one row of the accumulator: through shared memory into rows of four lanes
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            const float* v = &sum[c * 32 + 4 * g];
            *reinterpret_cast<float4*>(w.staging + lane * 128 + ((g ^ (lane & 7)) << 4)) = make_float4(v[0], v[1], v[2], v[3]);
        }
        __syncwarp();
        const int col = col0 + c * 32 + ch * 8;
        uint4 first_out[4], second_out[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 8 + sub, row = row0 + r;
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 x = *reinterpret_cast<const float4*>(w.staging + r * 128 + (((2 * ch + h) ^ (r & 7)) << 4));
                v[4 * h] = x.x;
                v[4 * h + 1] = x.y;
                v[4 * h + 2] = x.z;
                v[4 * h + 3] = x.w;
            }
            const bool in = row < rows && col < ld;
            const int64_t at = (int64_t)row * ld + col;
            float first[8] = {}, second[8] = {};
            if constexpr (kCombine) {
                unpack_half(first_q[c][i], first);
                unpack_half(second_q[c][i], second);
            }
            if constexpr (kMode == kGram) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] *= kDown;                                   // 2^24 A as it comes, 2^12 A as it is held
                    if (in && row == col + e) diag_a[row] = v[e] * kDown;
                }
            } else if constexpr (kMode == kPoly) {
                // the diagonal in fp32: A_ii as its product left it, and (A^2)_ii with that in A_ii's place
                const float d = f[c][i];
                float on_diagonal = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float a2 = v[e] * (kDown * kDown), h = first[e] * kDown, l = second[e] * kDown;
                    v[e] = fmaf(kNsB, first[e] + second[e], kNsC * a2 * kUp);
                    if (row == col + e) {
                        on_diagonal = kNsB * d + kNsC * (a2 + (d - h) * (d + h) - 2.f * h * l);
                        v[e] = 0.f;
                    }
                }
                if (in && row >= col && row < col + 8) diag_b[row] = on_diagonal;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float k = p.tall ? f[c][e] : f[c][i];
                    v[e] = fmaf(k, second[e], fmaf(k, first[e], v[e] * kDown));
                }
            }
            if (last) {
                if (row < p.rows) put_result(p, (int64_t)t.matrix * p.rows + row, col, v);
            } else {
                first_out[i] = pack_half(v);
                second_out[i] = pack_half(v);
                if (in) {
                    *reinterpret_cast<uint4*>(to + at) = first_out[i];
                    *reinterpret_cast<uint4*>(to + to_second + at) = second_out[i];
                }
            }
        }
        __syncwarp();
        if (mirrored) {                                              // the other way: 32 rows of 32, 16-byte pieces swizzled
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a[4] = {first_out[i].x, first_out[i].y, first_out[i].z, first_out[i].w};
                const uint32_t b[4] = {second_out[i].x, second_out[i].y, second_out[i].z, second_out[i].w};
                uint8_t* m = w.staging + ch * 512 + ((i ^ ch) << 4) + sub * 2;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    *reinterpret_cast<uint16_t*>(m + e * 64) = (uint16_t)(a[e >> 1] >> (16 * (e & 1)));
                    *reinterpret_cast<uint16_t*>(m + kHalfBytes + e * 64) = (uint16_t)(b[e >> 1] >> (16 * (e & 1)));
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = col0 + c * 32 + i * 8 + sub, at_col = row0 + ch * 8;
                const uint8_t* m = w.staging + (i * 8 + sub) * 64 + ((ch ^ i) << 4);
                if (row < p.m && at_col < p.ldm) {
                    const int64_t at = (int64_t)row * p.ldm + at_col;
                    *reinterpret_cast<uint4*>(to + at) = *reinterpret_cast<const uint4*>(m);
                    *reinterpret_cast<uint4*>(to + s_all + at) = *reinterpret_cast<const uint4*>(m + kHalfBytes);
                }
            }
            __syncwarp();
        }
    }
    return true;
}

// 32 x 32 numbers of a bf16 result, a row a lane, into the output (fp32 ones take both numbers of every operand).
__device__ __forceinline__ void put_results(const OrthoParams& p, int matrix, int row0, int c0, const float (&v)[32], OrthoWarp& w) {
    const int lane = w.lane;
    if (p.cols % 8 != 0) {                                           // rows that begin anywhere
        if (row0 + lane < p.rows) {
            const int64_t o = ((int64_t)matrix * p.rows + row0 + lane) * p.cols + c0;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                if (c0 + e >= p.cols) continue;
                static_cast<__nv_bfloat16*>(p.out)[o + e] = __float2bfloat16_rn(v[e]);
            }
        }
        return;
    }
    uint32_t b[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        b[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint4*>(w.staging + lane * 64 + ((g ^ ((lane >> 1) & 3)) << 4)) = make_uint4(b[4 * g], b[4 * g + 1], b[4 * g + 2], b[4 * g + 3]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (lane >> 2), row = row0 + r, col = c0 + (lane & 3) * 8;
        if (row < p.rows && col < p.cols)
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + ((int64_t)matrix * p.rows + row) * p.cols + col) =
                *reinterpret_cast<const uint4*>(w.staging + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4));
    }
    __syncwarp();
}

// The epilogue where the products take the first numbers: kCols columns of 32 rows, a row a lane.  The next X has its a X in the sums
// already; the second product's sums are combined with A.
template <int kMode, int kWidth, int kCols>
__device__ __forceinline__ bool ortho_epilogue(const OrthoParams& p, const OrthoItem& t, OrthoWarp& w) {
    constexpr bool kSymmetric = kMode != kStep;
    constexpr int kChunks = kCols / 32;
    const int lane = w.lane, sub = lane >> 2, ch = lane & 3;
    const int rows = kSymmetric ? p.m : p.rows, ld = kSymmetric ? p.ldm : p.ldx;
    const int row0 = t.i * kTile + w.quad * 32, col0 = t.j * kWidth + w.half * kCols;
    const int64_t s_all = (int64_t)p.count * p.s_plane, x_all = (int64_t)p.count * p.x_plane;
    __half* S = p.S + (int64_t)t.matrix * p.s_plane;
    __half* to = kMode == kGram ? S : kMode == kPoly ? S + p.b_plane * s_all
                                                     : p.X + (int64_t)((t.step & 1) ^ 1) * 2 * x_all + (int64_t)t.matrix * p.x_plane;
    float* diag_a = p.diag_a + (int64_t)t.matrix * p.ldm;
    const bool last = kMode == kStep && t.step == p.steps - 1;
    // below the diagonal a wide tile's half repeats what another tile stores
    const int block_j = col0 / kTile;
    const bool below = kSymmetric && block_j < t.i, mirrored = kSymmetric && block_j > t.i, on_diagonal = kSymmetric && block_j == t.i;
    const bool put_second = kMode == kStep || (kMode == kPoly && on_diagonal);
    // 64 bytes a row, 16-byte pieces swizzled: a row a lane, and rows of four lanes
    auto own = [&](int g) { return reinterpret_cast<uint4*>(w.staging + lane * 64 + ((g ^ ((lane >> 1) & 3)) << 4)); };
    auto shared = [&](int i) {
        const int r = i * 8 + sub;
        return reinterpret_cast<uint4*>(w.staging + r * 64 + ((ch ^ ((r >> 1) & 3)) << 4));
    };
    // A is asked for before the sums are there; past the L1, which may hold an earlier step's numbers
    uint4 a_q[kMode == kPoly ? kChunks : 1][4];
    float d = 0.f;
    if constexpr (kMode == kPoly) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = row0 + i * 8 + sub, col = col0 + c * 32 + ch * 8;
                a_q[c][i] = row < rows && col < ld && !below ? __ldcg(reinterpret_cast<const uint4*>(S + (int64_t)row * ld + col))
                                                             : make_uint4(0u, 0u, 0u, 0u);
            }
        if (on_diagonal && row0 + lane < p.m) d = __ldcg(diag_a + row0 + lane);
    }
    if (!take_sums(w, w.ctl->acc_full, w.acc, p.status_word)) return false;
    const uint32_t taddr = w.tmem + w.acc.slot() * kWidth + w.half * kCols;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        float v[32];
        ptx::tmem_ld_32x32(taddr + c * 32, v);
        ptx::tmem_ld_wait();
        if (c == kChunks - 1) give_back(w, w.ctl->acc_empty, w.acc);
        const int c0 = col0 + c * 32;
        if constexpr (kMode == kGram && kWidth == kTile) {           // (wider tiles are not cut)
            if (t.cut < p.cuts - 1) {
                put_share<0>(p, t, w, w.half * kCols + c * 32, v);
                continue;
            }
            if (p.cuts > 1) {
                if (c == 0 && !wait_shares(p, t, w)) return false;
                add_shares<0>(p, t, w, w.half * kCols + c * 32, v);
            }
        }
        if (below || c0 >= ld || row0 >= rows) continue;
        // 2^24 times the sum as it comes; 2^12 as it is held
        if (last) {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] *= p.scale * (kDown * kDown);
            put_results(p, t.matrix, row0, c0, v, w);
            continue;
        }
        if constexpr (kMode == kPoly) {
#pragma unroll
            for (int i = 0; i < 4; ++i) *shared(i) = a_q[c][i];
            __syncwarp();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float a[8];
                unpack_half(*own(g), a);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float s = v[8 * g + e];
                    v[8 * g + e] = fmaf(kNsB, a[e], kNsC * kDown * s);
                    if (c0 == row0 && 8 * g + e == lane) {
                        // the diagonal of B, a included, from A_ii in fp32: as its product left it, and in its place in (A^2)_ii
                        const float h = a[e] * kDown;
                        v[8 * g + e] = (kNsA + kNsB * d + kNsC * (s * (kDown * kDown) + (d - h) * (d + h))) * kUp;
                    }
                }
            }
            __syncwarp();
        } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] *= kDown;
            if (kMode == kGram && c0 == row0) {
#pragma unroll
                for (int e = 0; e < 32; ++e) d = e == lane ? v[e] : d;
                if (row0 + lane < p.m) diag_a[row0 + lane] = d * kDown;
            }
        }
        uint32_t first[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const __half2 h = __floats2half2_rn(v[2 * e], v[2 * e + 1]);
            first[e] = *reinterpret_cast<const uint32_t*>(&h);
            if constexpr (kMode != kGram) {
                const float2 r = __half22float2(h);
                v[2 * e] -= r.x;
                v[2 * e + 1] -= r.y;
            }
        }
        auto put = [&](const uint32_t (&x)[16], __half* plane) {
#pragma unroll
            for (int g = 0; g < 4; ++g) *own(g) = make_uint4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = row0 + i * 8 + sub, col = c0 + ch * 8;
                if (row < rows && col < ld) *reinterpret_cast<uint4*>(plane + (int64_t)row * ld + col) = *shared(i);
            }
            __syncwarp();
        };
        put(first, to);
        if (kMode != kGram && put_second) {
            uint32_t second[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const __half2 h = __floats2half2_rn(v[2 * e], v[2 * e + 1]);
                second[e] = *reinterpret_cast<const uint32_t*>(&h);
            }
            put(second, to + (kMode == kStep ? x_all : s_all));
        }
        if (mirrored) {
            // the other way: two lanes have rows r, r + 1 of columns c, c + 1; after an exchange one has column c of both, the
            // other column c + 1, and 16 lanes store 64 bytes
            const int col = row0 + (lane & ~1);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t other = __shfl_xor_sync(0xffffffffu, first[e], 1);
                const uint32_t pair = lane & 1 ? __byte_perm(other, first[e], 0x7632) : __byte_perm(first[e], other, 0x5410);
                const int row = c0 + 2 * e + (lane & 1);
                if (row < p.m && col < p.ldm) *reinterpret_cast<uint32_t*>(to + (int64_t)row * p.ldm + col) = pair;
            }
        }
    }
    return true;
}

// Epilogue warps: their loads, stores and fences take longer than their arithmetic, so sixteen, as many as the registers allow; eight
// where the sums are added up in registers.
__host__ __device__ constexpr int ortho_epilogue_warps(bool exact) { return exact ? 8 : 16; }
__host__ __device__ constexpr int ortho_threads(bool exact) { return 32 * (kFirstEpilogueWarp + ortho_epilogue_warps(exact)); }

// kExact: both numbers of every operand, three products; kWidth: columns of a tile.
template <bool kExact, int kWidth>
__global__ void __launch_bounds__(ortho_threads(kExact), 1)
ortho_kernel(const __grid_constant__ CUtensorMap x_rows, const __grid_constant__ CUtensorMap x_across, const __grid_constant__ CUtensorMap s_rows,
             const OrthoParams p) {
    static_assert(!kExact || kWidth == kTile, "the sums in registers have room for 128 columns");
    constexpr uint32_t kPlane = kOperand + kWidth * kRow, kStage = (kExact ? 2 : 1) * kPlane;
    constexpr int kStages = kRing / kStage;
    static_assert(kStages <= kMostStages, "stages");
    constexpr uint32_t kTmemCols = (kExact ? 4 : 2) * kWidth;
    constexpr int kEpilogueWarps = ortho_epilogue_warps(kExact), kCols = kWidth / (kEpilogueWarps / 4);
    extern __shared__ uint8_t smem_raw[];
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t raw = ptx::smem_addr(smem_raw), ring = (raw + 1023u) & ~1023u;
    OrthoControl* ctl = reinterpret_cast<OrthoControl*>(smem_raw + (ring - raw) + kRing);

    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(ptx::smem_addr(&ctl->full[s]), 1);
            ptx::mbar_init(ptx::smem_addr(&ctl->empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(ptx::smem_addr(&ctl->acc_full[a]), 1);
            ptx::mbar_init(ptx::smem_addr(&ctl->acc_empty[a]), kEpilogueWarps);
            ptx::mbar_init(ptx::smem_addr(&ctl->small_full[a]), 1);
            ptx::mbar_init(ptx::smem_addr(&ctl->small_empty[a]), kEpilogueWarps);
        }
        for (int i = 0; i < kItems; ++i) {
            ptx::mbar_init(ptx::smem_addr(&ctl->item_full[i]), 1);
            ptx::mbar_init(ptx::smem_addr(&ctl->item_empty[i]), kEpilogueWarps + 3);
            ptx::mbar_init(ptx::smem_addr(&ctl->stored[i]), kEpilogueWarps);
        }
        ctl->abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&x_rows);
        ptx::prefetch_tensormap(&x_across);
        ptx::prefetch_tensormap(&s_rows);
    }
    if (warp == kProductWarp) ptx::tmem_alloc(ptx::smem_addr(&ctl->tmem_slot), kTmemCols);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&ctl->tmem_slot);
    volatile int* abort_flag = &ctl->abort_flag;
    int32_t* status_word = p.status_word;
    pdl_wait();
    const bool skip = block_sees_error(status_word);
    const uint32_t total = (uint32_t)p.steps * ((uint32_t)(p.cuts + 1) * p.sym_tiles + p.step_tiles) * (uint32_t)p.count;

    // the item in the ring's next place, for the warps that do not draw; false behind the last one, and where a wait ran out
    auto next_item = [&](uint32_t n, OrthoItem& t, bool free_place = true) {
        const uint32_t s = n % kItems;
        bool ok = ptx::mbar_wait(ptx::smem_addr(&ctl->item_full[s]), (n / kItems) & 1u, abort_flag, status_word);
        ok = __all_sync(0xffffffffu, ok);
        const int4 a = ctl->item[s][0], b = ctl->item[s][1];
        t = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        __syncwarp();
        if (free_place && lane == 0) ptx::mbar_arrive(ptx::smem_addr(&ctl->item_empty[s]));
        return ok && t.need >= 0;
    };

    if (skip) {
        // an earlier call failed: the outputs are left alone
    } else if (warp == kCopyWarp) {
        const bool leader = ptx::elect_one();
        uint32_t it = 0;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            OrthoItem t;
            if (!next_item(n, t)) break;
            // which operands are read across: both of a tall matrix's A (its reduction runs down X), X of a wide one's step
            const bool across_a = t.mode == kGram && p.tall, across_b = across_a || (t.mode == kStep && !p.tall);
            const bool a_is_x = t.mode == kGram || (t.mode == kStep && p.tall), b_is_x = t.mode == kGram || (t.mode == kStep && !p.tall);
            const CUtensorMap* map_a = a_is_x ? (across_a ? &x_across : &x_rows) : &s_rows;
            const CUtensorMap* map_b = b_is_x ? (across_b ? &x_across : &x_rows) : &s_rows;
            const int x_first = (t.step & 1) * 2, s_first = t.mode == kStep ? p.b_plane : 0;
            const int za = (a_is_x ? x_first : s_first) * p.count + t.matrix, zb = (b_is_x ? x_first : s_first) * p.count + t.matrix;
            const bool with_extras = !kExact && t.mode == kStep;
            int from;
            const int blocks = ortho_blocks(p, t, from) + (with_extras ? step_extras<kWidth>(p) : 0);
            for (int k = 0; k < blocks && ok; ++k, ++it) {
                const OrthoBlock blk = with_extras ? step_block<kWidth>(p, t, k) : OrthoBlock{from + k, 0, 0, 0};
                const int y = blk.at * kDeep;
                const uint32_t s = it % kStages;
                ok = ptx::mbar_wait(ptx::smem_addr(&ctl->empty[s]), ((it / kStages) & 1u) ^ 1u, abort_flag, status_word);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t full = ptx::smem_addr(&ctl->full[s]);
                if (leader) ptx::mbar_arrive_expect_tx(full, blk.narrow ? 2 * kOperand : kStage);
#pragma unroll
                for (int second = 0; second < (kExact ? 2 : 1); ++second) {
                    const uint32_t a = ring + s * kStage + second * kPlane, b = a + kOperand;
                    const int z_a = za + (second + (a_is_x ? blk.second_x : blk.second_s)) * p.count;
                    const int z_b = zb + (second + (b_is_x ? blk.second_x : blk.second_s)) * p.count;
                    if (across_a) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) ptx::tma_load_3d_warp(a + h * kHalfOperand, map_a, t.i * kTile + 64 * h, y, z_a, full, leader);
                    } else {
                        ptx::tma_load_3d_warp(a, map_a, y, t.i * kTile, z_a, full, leader);
                    }
                    if (across_b) {
#pragma unroll
                        for (int h = 0; h < kWidth / 64; ++h)
                            ptx::tma_load_3d_warp(b + h * kHalfOperand, map_b, t.j * kWidth + 64 * h, y, z_b, full, leader);
                    } else if (blk.narrow) {
                        ptx::tma_load_3d_warp(b, map_b, y, t.j * kWidth + kTile * (blk.narrow - 1), z_b, full, leader);
                    } else {
#pragma unroll
                        for (int h = 0; h < kWidth / kTile; ++h)
                            ptx::tma_load_3d_warp(b + h * kOperand, map_b, y, t.j * kWidth + kTile * h, z_b, full, leader);
                    }
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
    } else if (warp == kProductWarp) {
        const bool leader = ptx::elect_one();
        uint32_t it = 0;
        Turns acc, small;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            OrthoItem t;
            if (!next_item(n, t)) break;
            const bool across_a = t.mode == kGram && p.tall, across_b = across_a || (t.mode == kStep && !p.tall);
            const bool with_extras = !kExact && t.mode == kStep;
            int from;
            const int blocks = ortho_blocks(p, t, from) + (with_extras ? step_extras<kWidth>(p) : 0);
            const int each = part_products(t.mode, t.i, t.j), last_product = blocks * (kDeep / kUmmaDeep) - 1;
            const uint32_t idesc = ptx::umma_idesc_f16(kTile, kWidth, across_a, across_b);
            const uint32_t a_step = (across_a ? kUmmaDeep * kRow : kUmmaDeep * 2u) >> 4, b_step = (across_b ? kUmmaDeep * kRow : kUmmaDeep * 2u) >> 4;
            const uint32_t a_lo = ptx::umma_desc_lo(ring, across_a ? kHalfOperand : 16u);
            const uint32_t b_lo = ptx::umma_desc_lo(ring + kOperand, across_b ? kHalfOperand : 16u);
            auto wait_empty = [&](uint64_t* empty, const Turns& turn) {
                const bool got = ptx::mbar_wait(ptx::smem_addr(&empty[turn.slot()]), turn.phase() ^ 1u, abort_flag, status_word);
                return (bool)__all_sync(0xffffffffu, got);
            };
            if (kExact) ok = wait_empty(ctl->small_empty, small);
            for (int k = 0; k < blocks && ok; ++k, ++it) {
                if (!kExact && k == 0 && !(ok = wait_empty(ctl->acc_empty, acc))) break;
                const uint32_t s = it % kStages;
                ok = ptx::mbar_wait(ptx::smem_addr(&ctl->full[s]), (it / kStages) & 1u, abort_flag, status_word);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const uint32_t a = a_lo + s * (kStage >> 4), b = b_lo + s * (kStage >> 4);
                if constexpr (kExact) {
                    const uint32_t d2 = tmem + (2 + small.slot()) * kWidth, two = kPlane >> 4;
#pragma unroll
                    for (uint32_t u = 0; u < kDeep / kUmmaDeep; ++u) {
                        const int at = k * (int)(kDeep / kUmmaDeep) + (int)u;
                        const bool fresh = (at & (each - 1)) == 0;
                        if (fresh) {
                            if (!(ok = wait_empty(ctl->acc_empty, acc))) break;
                            ptx::tc_fence_after_sync();
                        }
                        const uint32_t au = a + u * a_step, bu = b + u * b_step, d = tmem + acc.slot() * kWidth;
                        ptx::umma_bf16_warp<false>(d2, ptx::umma_desc_of(au + two), ptx::umma_desc_of(bu), idesc, (k | u) != 0u, leader);
                        ptx::umma_bf16_warp<false>(d, ptx::umma_desc_of(au), ptx::umma_desc_of(bu), idesc, !fresh, leader);
                        ptx::umma_bf16_warp<false>(d2, ptx::umma_desc_of(au), ptx::umma_desc_of(bu + two), idesc, true, leader);
                        if ((at & (each - 1)) == each - 1 || at == last_product) {
                            if (leader) ptx::umma_commit(ptx::smem_addr(&ctl->acc_full[acc.slot()]));
                            ++acc.used;
                        }
                    }
                    if (!ok) break;
                } else {
                    const uint32_t d = tmem + acc.slot() * kWidth;
                    const int narrow = with_extras ? step_block<kWidth>(p, t, k).narrow : 0;
                    const uint32_t di = narrow ? d + kTile * (narrow - 1) : d, id = narrow ? ptx::umma_idesc_f16(kTile, kTile, false, false) : idesc;
#pragma unroll
                    for (uint32_t u = 0; u < kDeep / kUmmaDeep; ++u)
                        ptx::umma_bf16_warp<false>(di, ptx::umma_desc_of(a + u * a_step), ptx::umma_desc_of(b + u * b_step), id, (k | u) != 0u, leader);
                }
                if (leader) ptx::umma_commit(ptx::smem_addr(&ctl->empty[s]));
                if (!kExact && k == blocks - 1) {
                    if (leader) ptx::umma_commit(ptx::smem_addr(&ctl->acc_full[acc.slot()]));
                    ++acc.used;
                }
                if (kExact && k == blocks - 1) {
                    if (leader) ptx::umma_commit(ptx::smem_addr(&ctl->small_full[small.slot()]));
                    ++small.used;
                }
                __syncwarp();
            }
        }
        __syncwarp();
    } else if (warp == kDrawWarp) {
        // Draws items and waits until they are ready: the counter's and the counts' answers take 3000 clocks, half as long as a tile's
        // products.  The ring's places allow one item beyond those being copied, multiplied and stored.
        for (uint32_t n = 0;; ++n) {
            const uint32_t slot = n % kItems;
            bool ok = ptx::mbar_wait(ptx::smem_addr(&ctl->item_empty[slot]), ((n / kItems) & 1u) ^ 1u, abort_flag, status_word);
            if (!__all_sync(0xffffffffu, ok)) break;
            uint32_t q = 0;
            if (lane == 0) q = atomicAdd(p.drawn, 1u);
            q = __shfl_sync(0xffffffffu, q, 0);
            OrthoItem t = {};
            t.need = -1;
            if (q < total) {
                t = ortho_item<kWidth>(p, q);
                if (lane == 0) ok = wait_done(p.done + t.matrix, t.need, abort_flag, status_word);
                if (!__all_sync(0xffffffffu, ok)) break;
            }
            if (lane == 0) {
                ctl->item[slot][0] = make_int4(t.step, t.mode, t.matrix, t.i);
                ctl->item[slot][1] = make_int4(t.j, t.tile, t.cut, t.need);
                ptx::mbar_arrive(ptx::smem_addr(&ctl->item_full[slot]));
            }
            if (q >= total) break;
        }
        __syncwarp();
    } else if (warp == kTellWarp) {
        // Tells the other blocks of a finished tile: a fence waits until its stores have arrived, 1.5 us, which the epilogue warps
        // would otherwise spend.  An item's place in the ring is only freed then, so that no barrier here is passed twice.
        for (uint32_t n = 0;; ++n) {
            OrthoItem t;
            if (!next_item(n, t, false)) break;
            bool ok = ptx::mbar_wait(ptx::smem_addr(&ctl->stored[n % kItems]), (n / kItems) & 1u, abort_flag, status_word);
            if (!__all_sync(0xffffffffu, ok)) break;
            if (lane == 0) {
                asm volatile("fence.proxy.async;\n\tfence.acq_rel.gpu;" ::: "memory");
                asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(p.done + t.matrix) : "memory");
                if (t.mode == kGram && t.cut < p.cuts - 1)
                    asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(p.shares + (int64_t)t.matrix * p.sym_tiles + t.tile) : "memory");
                ptx::mbar_arrive(ptx::smem_addr(&ctl->item_empty[n % kItems]));
            }
            __syncwarp();
        }
    } else if (warp >= kFirstEpilogueWarp) {
        // the accumulator's rows 32 (warp % 4) .. + 31, kCols of its columns
        OrthoWarp w;
        w.ctl = ctl;
        w.staging = smem_raw + (ring - raw) + kRing + kControl + (warp - kFirstEpilogueWarp) * (kStagingBytes / kEpilogueWarps);
        w.abort_flag = abort_flag;
        w.lane = lane;
        w.quad = warp & 3;
        w.half = (warp - kFirstEpilogueWarp) >> 2;
        w.tmem = tmem + ((uint32_t)(w.quad * 32) << 16);
        for (uint32_t n = 0;; ++n) {
            OrthoItem t;
            if (!next_item(n, t)) break;
            bool ok;
            if constexpr (kExact) {
                ok = t.mode == kGram   ? ortho_epilogue_exact<kGram>(p, t, w)
                     : t.mode == kPoly ? ortho_epilogue_exact<kPoly>(p, t, w)
                                       : ortho_epilogue_exact<kStep>(p, t, w);
            } else {
                ok = t.mode == kGram   ? ortho_epilogue<kGram, kWidth, kCols>(p, t, w)
                     : t.mode == kPoly ? ortho_epilogue<kPoly, kWidth, kCols>(p, t, w)
                                       : ortho_epilogue<kStep, kWidth, kCols>(p, t, w);
            }
            if (!ok) break;
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&ctl->stored[n % kItems]));
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == kProductWarp) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, kTmemCols);
    }
}

// 2^12 / norm as a power of two and a number near 2^12, each of which fp32 holds
__device__ __forceinline__ void inverse_norm(double norm, float& power, float& factor) {
    int e = norm > 0.0 && isfinite(norm) ? ilogb(norm) : 0;
    e = e > 126 ? 126 : e < -126 ? -126 : e;
    power = scalbnf(1.f, -e);
    const double f = 4096.0 / ldexp(norm, -e);
    factor = norm > 0.0 && f > 3e38 ? 3e38f : (float)f;              // (an eps below 2^-149, alone: of zeros, which stay zeros)
}

// ---- the start: momentum, the norm, the two fp16 numbers of U / (|U| + eps) ----
constexpr int kStartThreads = 256;
constexpr int kStartBlocks = 8 * kNumSMs;                            // of all matrices, about

struct StartParams {
    const float* G;
    float* momentum;                 // nullable
    double* partial;                 // [count][blocks]: sums of squares
    uint32_t* counters;              // the products', cleared here: one, `count`, and a few a matrix
    int counters_each;
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
    if (block_sees_error(p.status_word)) return;
    const int matrix = blockIdx.y;
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0) p.counters[1 + matrix] = 0u;
        if (threadIdx.x == 1 && matrix == 0) p.counters[0] = 0u;
        for (int i = threadIdx.x; i < p.counters_each; i += kStartThreads) p.counters[1 + p.count + matrix * p.counters_each + i] = 0u;
    }
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
        constexpr int kBatch = 4;                     // loads of a thread before its stores, which might be to the same places for all it knows
        for (int64_t i = (int64_t)blockIdx.x * kStartThreads + threadIdx.x; i < p.elements / 4; i += kBatch * stride) {
            float4 g[kBatch], m[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const bool in = i + u * stride < p.elements / 4;
                g[u] = in ? __ldg(G + i + u * stride) : make_float4(0.f, 0.f, 0.f, 0.f);
                m[u] = in && mom != nullptr ? mom[i + u * stride] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                one(g[u].x, m[u].x);
                one(g[u].y, m[u].y);
                one(g[u].z, m[u].z);
                one(g[u].w, m[u].w);
                if (mom != nullptr && i + u * stride < p.elements / 4) mom[i + u * stride] = m[u];
            }
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
    if (block_sees_error(p.status_word)) return;
    const int matrix = blockIdx.y;
    __shared__ double part[kStartThreads / 32];
    double s = 0.0;
    for (int b = threadIdx.x; b < p.blocks; b += kStartThreads) s += p.partial[(int64_t)matrix * p.blocks + b];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < kStartThreads / 32; ++w) s += part[w];
    const double norm = sqrt(s) + p.eps;
    float power, factor;
    inverse_norm(norm, power, factor);
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

// ---- matrices with a side of at most 128: one launch, X in shared memory ----
// A matrix with m = min(rows, cols) <= 128 is a cluster of up to eight blocks, each with a slice of at most 256 of the longer side's
// positions in its shared memory for the whole call: as [128, slice] in 64 wide blocks of 128-byte rows, which are the
// reduction-major operand of A and, unchanged, the other operand of B X (a tall matrix is turned when it is read).  A's partial
// sums over the slices go to the blocks that own their rows, and A comes back to all of them, through distributed shared memory;
// everything else stays in the block.  Momentum and norm included, it is one launch without a wait on another cluster.
// Both fp16 numbers of every operand, as the other exact products.  A's sums and those of its square go to three accumulators in turns,
// which are added up in fp32: 100 x 257 81.5 us, error 0.8e-6; one accumulator 78.9 us, 1.7e-6 (the iteration in fp32: 1.5e-6).
constexpr int kSmallSide = 128, kSmallSlice = 256, kSmallCluster = 8, kSmallThreads = 512;
constexpr uint32_t kSmallBlock = 128 * kRow;                        // 128 x 64 numbers
constexpr uint32_t kSmallX = 4 * kSmallBlock, kSmallS = 2 * kSmallBlock;         // a plane of X, of A and B
constexpr uint32_t kSmallSmem = 2 * kSmallX + 2 * kSmallS + 1024;
static_assert(kSmallS * 2 == 128 * 128 * 4, "the partial sums of the rows a block owns take the place of A");

struct SmallParams {
    const float* G;
    float* momentum;
    void* out;
    int rows, cols, m, n, slice, tall, steps, nesterov, out_bf16;
    float beta, scale;
    double eps;
    int32_t* status_word;
};

__device__ __forceinline__ void st_cluster(uint32_t addr, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint2 v) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(addr), "r"(v.x), "r"(v.y) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
}
// byte offset of numbers (row, col .. ) of a [128, 64 k] plane: 64 wide blocks, 128-byte rows, 16-byte pieces swizzled
__device__ __forceinline__ uint32_t small_at(int row, int col) {
    return (uint32_t)(col >> 6) * kSmallBlock + (uint32_t)row * kRow + ((((uint32_t)col >> 3 & 7u) ^ ((uint32_t)row & 7u)) << 4) + ((uint32_t)col & 7u) * 2;
}
__global__ void __launch_bounds__(kSmallThreads, 1) ortho_small_kernel(const SmallParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t product_done;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_slot;
    __shared__ double warp_squares[kSmallThreads / 32], block_squares[kSmallCluster];
    __shared__ float diag_a[kSmallSide], diag_b[kSmallSide];
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, tid = threadIdx.x;
    uint32_t blocks, rank = ptx::cluster_ctarank();
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(blocks));
    const int matrix = blockIdx.x / blocks;
    const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* X = smem_raw + (base - raw);                           // first numbers, second numbers
    uint8_t* S = X + 2 * kSmallX;
    const uint32_t x_addr = base, s_addr = base + 2 * kSmallX;

    pdl_launch_dependents();
    if (tid == 0) {
        ptx::mbar_init(ptx::smem_addr(&product_done), 1);
        abort_slot = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 0) ptx::tmem_alloc(ptx::smem_addr(&tmem_slot), 512);
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    for (uint32_t i = tid; i < 2 * kSmallX / 16; i += kSmallThreads) reinterpret_cast<uint4*>(X)[i] = zero;
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);
    volatile int* abort_flag = &abort_slot;
    pdl_wait();
    // (a block that goes on alone would wait for the others of its cluster, so they agree below)
    const bool skip = block_sees_error(p.status_word);
    bool ok = !skip;

    // ---- momentum, norm, X ----
    const int64_t elements = (int64_t)p.rows * p.cols;
    const float* G = p.G + matrix * elements;
    float* mom = p.momentum != nullptr ? p.momentum + matrix * elements : nullptr;
    const int j0 = (int)rank * p.slice, width = p.n - j0 < p.slice ? p.n - j0 : p.slice;        // this block's positions (none: <= 0)
    // numbers of G in groups along its rows (outer, inner ..): of four where they are aligned
    const int outers = p.tall ? width : p.m, inners = p.tall ? p.m : width;
    auto place = [&](int outer, int inner) { return p.tall ? (int64_t)(j0 + outer) * p.cols + inner : (int64_t)outer * p.cols + j0 + inner; };
    auto visit_by = [&](auto size, auto f) {                         // f(u[], mo[]: gradient, momentum; outer, inner)
        constexpr int N = decltype(size)::value;
        // a warp has every sixteenth row, a lane every 32nd group; kBatch of them are loaded before any is stored
        constexpr int kBatch = N == 4 ? 4 : 12;
        const int groups = inners / N, chunks = (groups + 31) / 32;
        int o = warp, c = 0;
        while (o < outers && chunks > 0) {
            float u[kBatch][N], mo[kBatch][N];
            int outer[kBatch], inner[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int g = c * 32 + lane;
                outer[i] = o < outers && g < groups ? o : -1;
                inner[i] = g * N;
                if (++c == chunks) {
                    c = 0;
                    o += kSmallThreads / 32;
                }
#pragma unroll
                for (int e = 0; e < N; ++e) u[i][e] = mo[i][e] = 0.f;
                if (outer[i] < 0) continue;
                const int64_t at = place(outer[i], inner[i]);
                if constexpr (N == 4) {
                    const float4 a = __ldg(reinterpret_cast<const float4*>(G + at));
                    u[i][0] = a.x, u[i][1] = a.y, u[i][2] = a.z, u[i][3] = a.w;
                    if (mom != nullptr) {
                        const float4 b = *reinterpret_cast<const float4*>(mom + at);
                        mo[i][0] = b.x, mo[i][1] = b.y, mo[i][2] = b.z, mo[i][3] = b.w;
                    }
                } else {
                    u[i][0] = __ldg(G + at);
                    if (mom != nullptr) mo[i][0] = mom[at];
                }
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (outer[i] >= 0) f(u[i], mo[i], outer[i], inner[i]);
        }
    };
    auto visit = [&](auto f) {                                       // (where cols is a multiple of four, so is every block's share)
        if (p.cols % 4 == 0) visit_by(std::integral_constant<int, 4>(), f);
        else visit_by(std::integral_constant<int, 1>(), f);
    };
    double squares = 0.0;
    if (ok) {
        visit([&](auto& u, auto& mo, int outer, int inner) {
            constexpr int N = sizeof(u) / sizeof(float);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (mom != nullptr) {
                    mo[e] = fmaf(p.beta, mo[e], u[e]);
                    u[e] = p.nesterov ? fmaf(p.beta, mo[e], u[e]) : mo[e];
                }
                squares = fma((double)u[e], (double)u[e], squares);
            }
            if (mom == nullptr) return;
            const int64_t at = place(outer, inner);
            if constexpr (N == 4) *reinterpret_cast<float4*>(mom + at) = make_float4(mo[0], mo[1], mo[2], mo[3]);
            else mom[at] = mo[0];
        });
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
    if (lane == 0) warp_squares[warp] = squares;
    ptx::cluster_sync_all();                                         // (a barrier of the block, and every block has begun)
    if (tid < (int)blocks) {
        double s = 0.0;
        for (int w = 0; w < kSmallThreads / 32; ++w) s += warp_squares[w];
        if (skip) s = -1.0;
        st_cluster(ptx::map_to_cta(ptx::smem_addr(&block_squares[rank]), (uint32_t)tid), s);
    }
    ptx::cluster_sync_all();
    {
        double s = 0.0;
        for (uint32_t b = 0; b < blocks; ++b) {
            s += block_squares[b];
            if (block_squares[b] < 0.0) ok = false;                  // some block has seen an error: none goes on
        }
        float power, factor;
        inverse_norm(sqrt(s) + p.eps, power, factor);
        if (ok) {
            visit([&](auto& u, auto& mo, int outer, int inner) {
                constexpr int N = sizeof(u) / sizeof(float);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (mom != nullptr) u[e] = p.nesterov ? fmaf(p.beta, mo[e], u[e]) : mo[e];
                    const float x = u[e] * power * factor;
                    const uint32_t at = p.tall ? small_at(inner + e, outer) : small_at(outer, inner + e);
                    const __half h = __float2half_rn(x);
                    *reinterpret_cast<__half*>(X + at) = h;
                    *reinterpret_cast<__half*>(X + kSmallX + at) = __float2half_rn(x - __half2float(h));
                }
            });
        }
    }

    // ---- the steps ----
    const int quad = warp & 3, row = quad * 32 + lane, cols0 = (warp >> 2) * 32;       // epilogues: a lane's row, a warp's columns
    const uint32_t lane_tmem = tmem + ((uint32_t)(quad * 32) << 16);
    // tensor memory: A and its polynomial in columns 0 .. 127, the next X in 256 ..; the small products of the three, first x second
    // and second x first, 128 columns further on (an instruction that adds to the place of the one before it waits for it),
    // where a slice of over 128 positions does not need them.  A and its square use the next X's columns too: their products go to three
    // places in turns (see the head: short chains).
    const bool narrow = p.slice <= 128;
    const uint32_t d_sym = 0, d_step = 256, d_more = 256;
    const int m16 = (p.m + 15) / 16 * 16, deep_m = (p.m + kDeep - 1) / kDeep, deep_n = p.slice / kDeep;
    uint32_t phase = 0;
    // products of a and b (reduction along their rows, or down b's: across), the small ones to `two` where that is another place
    auto multiply = [&](bool symmetric, uint32_t d, uint32_t two, uint32_t a, uint32_t a_plane, uint32_t b, uint32_t b_plane, bool across, int width_n,
                        int blocks_k) {
        asm volatile("fence.proxy.async;" ::: "memory");             // what this thread wrote to shared memory, for the tensor core
        ptx::tc_fence_before_sync();
        __syncthreads();
        if (warp == 0 && ok) {
            ptx::tc_fence_after_sync();
            const bool leader = ptx::elect_one();
            const uint32_t idesc = ptx::umma_idesc_f16(kTile, width_n, false, across);
            const uint32_t a_lo = ptx::umma_desc_lo(a, 16u), b_lo = ptx::umma_desc_lo(b, across ? kSmallBlock : 16u);
            uint32_t place_at = 0u;
#pragma unroll 1
            for (int k = 0; k < blocks_k; ++k) {
#pragma unroll
                for (uint32_t u = 0; u < kDeep / kUmmaDeep; ++u) {
                    // along: 32 bytes of a row, the next 64 in the next block; across: 16 rows down, 64 rows in a deep block
                    const uint32_t au = a_lo + ((k * kSmallBlock + u * kUmmaDeep * 2) >> 4);
                    const uint32_t bu = b_lo + ((across ? k * kHalfOperand + u * kUmmaDeep * kRow : k * kSmallBlock + u * kUmmaDeep * 2) >> 4);
                    const bool more = k != 0 || u != 0u;
                    const bool fresh = k == 0 && u < (symmetric ? 3u : 1u);
                    const uint32_t dk = tmem + d + place_at;
                    if (symmetric) place_at = place_at == 0u ? d_more : place_at == d_more ? d_more + 128u : 0u;
                    ptx::umma_bf16_warp<false>(tmem + two, ptx::umma_desc_of(au + (a_plane >> 4)), ptx::umma_desc_of(bu), idesc, more, leader);
                    ptx::umma_bf16_warp<false>(dk, ptx::umma_desc_of(au), ptx::umma_desc_of(bu), idesc, !fresh || two == d, leader);
                    ptx::umma_bf16_warp<false>(tmem + two, ptx::umma_desc_of(au), ptx::umma_desc_of(bu + (b_plane >> 4)), idesc, true, leader);
                }
            }
            if (leader) ptx::umma_commit(ptx::smem_addr(&product_done));
            __syncwarp();
        }
        if (ok) ok = ptx::mbar_wait(ptx::smem_addr(&product_done), phase & 1u, abort_flag, p.status_word);
        ok = __all_sync(0xffffffffu, ok);
        ++phase;
        ptx::tc_fence_after_sync();
    };
    auto sums = [&](uint32_t d, uint32_t two, float (&v)[32]) {      // of this lane's row, 32 columns from d on
        ptx::tmem_ld_32x32(lane_tmem + d, v);
        if (two != d) {
            float w[32];
            ptx::tmem_ld_32x32(lane_tmem + two, w);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] += w[e];
        } else {
            ptx::tmem_ld_wait();
        }
    };
    auto symmetric_sums = [&](float (&v)[32]) {                      // 32 columns from cols0 on
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            float w[4][16];
            const uint32_t from = lane_tmem + d_sym + cols0 + h;
            ptx::tmem_ld_32x16(from, w[0]);
            ptx::tmem_ld_32x16(from + d_more, w[1]);
            ptx::tmem_ld_32x16(from + d_more + 128, w[2]);
            ptx::tmem_ld_32x16(from + 128, w[3]);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) v[h + e] = ((w[0][e] + w[1][e]) + w[2][e]) + w[3][e];
        }
    };
    // 32 numbers of a row, times 2^12, as two fp16 numbers each
    auto put = [&](uint8_t* plane, uint32_t second, int r, int c, float (&v)[32]) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t at = small_at(r, c + 8 * g);
            *reinterpret_cast<uint4*>(plane + at) = pack_half(&v[8 * g]);
            *reinterpret_cast<uint4*>(plane + second + at) = pack_half(&v[8 * g]);
        }
    };
    for (int step = 0; step < p.steps; ++step) {
        // A: every block's share of the sum
        multiply(true, d_sym, d_sym + 128, x_addr, kSmallX, x_addr, kSmallX, false, m16, deep_n);
        float v[32];
        symmetric_sums(v);
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = cols0 + e < m16 ? v[e] * kDown : 0.f;      // (columns that no product wrote)
        if (blocks == 1) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
                if (cols0 + e == row) diag_a[row] = v[e] * kDown;
            put(S, kSmallS, row, cols0, v);
        } else {
            const int own = kSmallSide / (int)blocks;                // rows a block owns
            // the partial rows go where X has no positions, or else to the place of A and B, once no block reads them any more
            auto partial = [&](int r) { return narrow ? (uint32_t)(r < 64 ? 0 : kSmallX) + kSmallX / 2 + (uint32_t)(r & 63) * 512 : 2 * kSmallX + (uint32_t)r * 512; };
            const uint32_t to = ptx::map_to_cta(x_addr, (uint32_t)(row / own)) + partial((int)rank * own + row % own);
            if (step > 0 && !narrow) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // no block reads its A or B any more
#pragma unroll
            for (int g = 0; g < 8; ++g)
                st_cluster(to + (((uint32_t)(cols0 / 4 + g) ^ ((uint32_t)row & 7u)) << 4), make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]));
            ptx::cluster_sync_all();
            float4 a[4];
            const int items = own * 32;                              // (row, four columns) of the owned rows
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int item = tid + i * kSmallThreads;
                a[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (item >= items) continue;
                const int r = item >> 5;
                for (uint32_t b = 0; b < blocks; ++b) {              // (own is a multiple of eight: the swizzle is the row's)
                    const float4 q = *reinterpret_cast<const float4*>(X + partial((int)b * own + r) + (((item & 31) ^ (r & 7)) << 4));
                    a[i].x += q.x;
                    a[i].y += q.y;
                    a[i].z += q.z;
                    a[i].w += q.w;
                }
            }
            if (!narrow) ptx::cluster_sync_all();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int item = tid + i * kSmallThreads;
                if (item >= items) continue;
                const int r = (int)rank * own + (item >> 5), c = (item & 31) * 4;
                const float q[4] = {a[i].x, a[i].y, a[i].z, a[i].w};
                __half2 h[2], l[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    h[e] = __floats2half2_rn(q[2 * e], q[2 * e + 1]);
                    const float2 f = __half22float2(h[e]);
                    l[e] = __floats2half2_rn(q[2 * e] - f.x, q[2 * e + 1] - f.y);
                }
                const uint2 first = make_uint2(*reinterpret_cast<uint32_t*>(&h[0]), *reinterpret_cast<uint32_t*>(&h[1]));
                const uint2 second = make_uint2(*reinterpret_cast<uint32_t*>(&l[0]), *reinterpret_cast<uint32_t*>(&l[1]));
                float diagonal = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e == r) diagonal = q[e] * kDown;
                for (uint32_t b = 0; b < blocks; ++b) {
                    const uint32_t at = ptx::map_to_cta(s_addr + small_at(r, c), b);
                    st_cluster(at, first);
                    st_cluster(at + kSmallS, second);
                    if (r >= c && r < c + 4) st_cluster(ptx::map_to_cta(ptx::smem_addr(&diag_a[r]), b), diagonal);
                }
            }
            ptx::cluster_sync_all();
        }
        // B = b A + c A^2, its diagonal apart in fp32
        multiply(true, d_sym, d_sym + 128, s_addr, kSmallS, s_addr, kSmallS, false, m16, deep_m);
        symmetric_sums(v);
        const float d = diag_a[row];
        float on_diagonal = 0.f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t at = small_at(row, cols0 + 8 * g);
            float first[8], second[8];
            unpack_half(*reinterpret_cast<const uint4*>(S + at), first);
            unpack_half(*reinterpret_cast<const uint4*>(S + kSmallS + at), second);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a2 = cols0 + 8 * g + e < m16 ? v[8 * g + e] * (kDown * kDown) : 0.f;
                v[8 * g + e] = fmaf(kNsB, first[e] + second[e], kNsC * a2 * kUp);
                if (cols0 == quad * 32) {                            // (the same in the whole warp)
                    const float h = first[e] * kDown, l = second[e] * kDown, b = kNsB * d + kNsC * (a2 + (d - h) * (d + h) - 2.f * h * l);
                    on_diagonal = 8 * g + e == lane ? b : on_diagonal;
                    v[8 * g + e] = 8 * g + e == lane ? 0.f : v[8 * g + e];
                }
            }
        }
        if (cols0 == quad * 32) diag_b[row] = on_diagonal;
        put(S, kSmallS, row, cols0, v);
        // X <- a X + B X
        const uint32_t d_two = narrow ? d_step + 128 : d_step;
        multiply(false, d_step, d_two, s_addr, kSmallS, x_addr, kSmallX, true, p.slice, deep_m);
        const float f = kNsA + diag_b[row];
        const bool last = step == p.steps - 1;
        if (blocks > 1 && !narrow && !last) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        for (int pass = 0; pass < p.slice; pass += 128) {
            const int c0 = cols0 + pass;
            if (c0 < p.slice) {                                      // (the same in the whole warp)
                sums(d_step + c0, d_two + c0, v);
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint32_t at = small_at(row, c0 + 8 * g);
                    float first[8], second[8];
                    unpack_half(*reinterpret_cast<const uint4*>(X + at), first);
                    unpack_half(*reinterpret_cast<const uint4*>(X + kSmallX + at), second);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * g + e] = fmaf(f, second[e], fmaf(f, first[e], v[8 * g + e] * kDown));
                }
                if (!last) {
                    put(X, kSmallX, row, c0, v);
                } else {                                             // to the place of B: fp32 rows of 128, 16-byte pieces swizzled
#pragma unroll
                    for (int g = 0; g < 8; ++g)
                        *reinterpret_cast<float4*>(S + row * 512 + (((cols0 / 4 + g) ^ (row & 7)) << 4)) =
                            make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
                }
            }
            if (!last) continue;
            __syncthreads();
            const int have = width - pass < 128 ? width - pass : 128;
            auto out = [&](int r, int c) {                           // consecutive lanes write consecutive numbers
                const float x = *reinterpret_cast<const float*>(S + r * 512 + (((c >> 2) ^ (r & 7)) << 4) + (c & 3) * 4) * (p.scale * kDown);
                const int64_t o = matrix * elements + (p.tall ? place(pass + c, r) : place(r, pass + c));
                if (p.out_bf16) static_cast<__nv_bfloat16*>(p.out)[o] = __float2bfloat16_rn(x);
                else static_cast<float*>(p.out)[o] = x;
            };
            if (ok && p.tall) {
                for (int c = warp; c < have; c += kSmallThreads / 32)
                    for (int r = lane; r < p.m; r += 32) out(r, c);
            } else if (ok) {
                for (int r = warp; r < p.m; r += kSmallThreads / 32)
                    for (int c = lane; c < have; c += 32) out(r, c);
            }
            __syncthreads();
        }
        ptx::tc_fence_before_sync();
    }
    __syncthreads();
    ptx::cluster_sync_all();                                         // no block leaves while another may write to it
    if (warp == 0) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
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
    int s_planes, b_plane, start_blocks, width, cuts;
    uint32_t sym_tiles;
    bool exact;
    size_t S, diag_a, diag_b, partial, counters, share, bytes;       // offsets behind the planes of X
};
OrthoLayout ortho_layout(sbp_dtype dt, int64_t count, int64_t rows, int64_t cols) {
    OrthoLayout l;
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    l.m = rows < cols ? rows : cols;
    l.ldx = (cols + 7) / 8 * 8;
    l.ldm = (l.m + 7) / 8 * 8;
    l.exact = dt == SBP_F32 || l.m <= kExactSide;
    l.s_planes = l.exact ? 4 : 3;
    l.b_plane = l.exact ? 2 : 1;
    l.x_plane = rows * l.ldx;
    l.s_plane = l.m * l.ldm;
    const int64_t want = (rows * cols / 4 + 4 * kStartThreads - 1) / (4 * kStartThreads), most = kStartBlocks / count > 1 ? kStartBlocks / count : 1;
    l.start_blocks = (int)(want < 1 ? 1 : want < most ? want : most);
    // 256 wide tiles take half as much of their operands from the L2 for a product, but there are half as many: from about three 128
    // wide ones an SM on.  (Whole calls without momentum, 256 wide and 128 wide, us: 4 x 2048 x 2048, 1024 tiles of 128, 705 and 818;
    // 24 x 768 x 768, 864, 380 and 397; 2 x 2048 x 2048, 512, 499 and 492 to 520; 12 x 768 x 768, 432, 231 and 219; 4 x 2304 x 768,
    // 432, 274 and 242; 8 x 1261 x 222, 160, 254 to 300 and 236.)
    l.width = !l.exact && (rows + kTile - 1) / kTile * ((cols + kTile - 1) / kTile) * count > 3 * kNumSMs ? 256 : 128;
    const uint32_t tiles = (uint32_t)((l.m + kTile - 1) / kTile), wide = (uint32_t)((l.m + l.width - 1) / l.width), f = (uint32_t)l.width / kTile;
    l.sym_tiles = f * wide * (wide + 1) / 2 - (f * wide - tiles);
    // A's tiles are few, and their reduction is the longer side: it is cut into up to four shares of eight blocks at least while the
    // SMs have room for them
    const int64_t blocks = ((rows > cols ? rows : cols) + kDeep - 1) / kDeep;
    l.cuts = 1;
    // (waiting for the other shares costs some 4 us: 1024 x 1024, 16 blocks, 165 us whole and 217 cut in bf16, 289 and 309 in fp32;
    // 1024 x 4096 422 and 302 in bf16, 568 and 408 in fp32)
    while (l.width == kTile && blocks * (l.exact ? 2 : 1) >= 48 && l.cuts < 4 && (int64_t)(l.cuts + 1) * l.sym_tiles * count <= kNumSMs && blocks / (l.cuts + 1) >= 8) ++l.cuts;
    l.S = up((size_t)(4 * count * l.x_plane) * 2);
    l.diag_a = l.S + up((size_t)(l.s_planes * count * l.s_plane) * 2);
    l.diag_b = l.diag_a + up((size_t)(count * l.ldm) * 4);
    l.partial = l.diag_b + up((size_t)(count * l.ldm) * 4);
    l.counters = l.partial + up((size_t)count * l.start_blocks * 8);
    l.share = l.counters + up((size_t)(1 + count + (l.cuts > 1 ? count * l.sym_tiles : 0)) * 4);
    l.bytes = l.share + (size_t)(l.cuts - 1) * count * l.sym_tiles * kTile * kTile * 4;
    return l;
}

template <bool kExact, int kWidth>
cudaError_t launch_products(const CUtensorMap& x_rows, const CUtensorMap& x_across, const CUtensorMap& s_rows, OrthoParams& p, cudaStream_t stream) {
    const cudaError_t e = opt_in_dynamic_smem<ortho_kernel<kExact, kWidth>>((int)kOrthoSmem);
    if (e != cudaSuccess) return e;
    p.step_cols = (uint32_t)((p.cols + kWidth - 1) / kWidth);
    p.step_tiles = (uint32_t)((p.rows + kTile - 1) / kTile) * p.step_cols;
    const uint32_t grams = p.sym_tiles * (uint32_t)p.cuts;
    const int64_t most = (int64_t)p.count * (p.step_tiles > grams ? p.step_tiles : grams);
    return launch_pdl(ortho_kernel<kExact, kWidth>, dim3((unsigned)(most < kNumSMs ? most : kNumSMs)), dim3(ortho_threads(kExact)), kOrthoSmem, stream,
                      x_rows, x_across, s_rows, p);
}

// Blocks of a matrix's cluster, and the positions of the longer side each has; 0 where the other kernels take the matrix.  A step is
// 6.5 us without other blocks (128 positions; 10 with 256) and 12.4 with: 100 x 257, momentum included, 80 us on four blocks and 89
// on two, 100 x 256 67 us on one and 71 on two.  Without momentum, one matrix and twenty: 100 x 256 66 and 66 us on one block, 73 and 155
// on eight; 100 x 400 73 and 77 on four, 73 and 156 on eight; 100 x 513 85 and 179 on eight, 93 and 97 on four; 100 x 1000 80 and 169
// on eight, 93 and 99 on four (eight blocks a matrix fill the device twice from 19 matrices on: the rule is made for few).
int ortho_small_blocks(int64_t n) { return n <= 256 ? 1 : n <= 512 ? 4 : 8; }
int ortho_small_slice(int64_t rows, int64_t cols) {
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (m > kSmallSide || n > kSmallCluster * kSmallSlice) return 0;
    const int64_t blocks = ortho_small_blocks(n);
    return (int)((n + blocks * kDeep - 1) / (blocks * kDeep) * kDeep);
}
cudaError_t launch_small(sbp_dtype dt, const float* G, float* momentum, float beta, bool nesterov, int64_t count, int64_t rows, int64_t cols, int steps,
                         double eps, float scale, void* O, int32_t* status_word, cudaStream_t stream) {
    const cudaError_t e = opt_in_dynamic_smem<ortho_small_kernel>((int)kSmallSmem);
    if (e != cudaSuccess) return e;
    SmallParams p = {};
    p.G = G;
    p.momentum = momentum;
    p.out = O;
    p.rows = (int)rows;
    p.cols = (int)cols;
    p.tall = rows > cols;
    p.m = (int)(p.tall ? cols : rows);
    p.n = (int)(p.tall ? rows : cols);
    p.slice = ortho_small_slice(rows, cols);
    p.steps = steps;
    p.nesterov = nesterov;
    p.out_bf16 = dt == SBP_BF16;
    p.beta = beta;
    p.scale = scale;
    p.eps = eps;
    p.status_word = status_word;
    const unsigned blocks = (unsigned)ortho_small_blocks(p.n);
    return launch_pdl_cluster(ortho_small_kernel, dim3((unsigned)count * blocks), dim3(kSmallThreads), kSmallSmem, blocks, stream, p);
}

}  // namespace

size_t orthogonalize_workspace_bytes(sbp_dtype dt, int64_t count, int64_t rows, int64_t cols) {
    return ortho_small_slice(rows, cols) > 0 ? 256 : ortho_layout(dt, count, rows, cols).bytes;
}

// the items of a launch (A's in four shares, two more products of at most this many tiles, up to 32 times) and the planes a tensor map counts are 32-bit numbers
bool orthogonalize_supported(int64_t count, int64_t rows, int64_t cols) {
    const int64_t tiles = (rows + kTile - 1) / kTile * ((cols + kTile - 1) / kTile);
    return rows <= (1 << 16) && cols <= (1 << 16) && count <= (1 << 16) - 1 && 6 * 32 * tiles * count < (1ll << 31);
}

cudaError_t launch_orthogonalize(sbp_dtype dt, const float* G, float* momentum, float beta, bool nesterov, int64_t count, int64_t rows, int64_t cols,
                                 int steps, double eps, float scale, void* O, void* workspace, int32_t* status_word, cudaStream_t stream) {
    if (ortho_small_slice(rows, cols) > 0)
        return launch_small(dt, G, momentum, beta, nesterov, count, rows, cols, steps, eps, scale, O, status_word, stream);
    const OrthoLayout l = ortho_layout(dt, count, rows, cols);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    StartParams s = {};
    s.G = G;
    s.momentum = momentum;
    s.partial = reinterpret_cast<double*>(ws + l.partial);
    s.X = reinterpret_cast<__half*>(ws);
    s.counters = reinterpret_cast<uint32_t*>(ws + l.counters);
    s.counters_each = l.cuts > 1 ? (int)l.sym_tiles : 0;
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
    p.b_plane = l.b_plane;
    p.tall = rows > cols;
    p.out_bf16 = dt == SBP_BF16;
    p.scale = scale;
    p.status_word = status_word;
    CUtensorMap x_rows, x_across, s_rows;
    if (!plane_map(&x_rows, p.X, 4 * count, rows, cols, l.ldx, kTile) || !plane_map(&x_across, p.X, 4 * count, rows, cols, l.ldx, 64) ||
        !plane_map(&s_rows, p.S, l.s_planes * count, l.m, l.m, l.ldm, kTile))
        return cudaErrorUnknown;
    p.gram_blocks = (int)(((p.tall ? rows : cols) + kDeep - 1) / kDeep);
    p.m_blocks = (int)((l.m + kDeep - 1) / kDeep);
    p.steps = steps;
    p.out = O;
    p.sym_tiles = l.sym_tiles;
    p.cuts = l.cuts;
    p.drawn = s.counters;
    p.done = reinterpret_cast<int32_t*>(s.counters) + 1;
    p.shares = p.done + count;
    p.share = reinterpret_cast<float4*>(ws + l.share);
    if (l.exact) return launch_products<true, 128>(x_rows, x_across, s_rows, p, stream);
    return l.width == 256 ? launch_products<false, 256>(x_rows, x_across, s_rows, p, stream) : launch_products<false, 128>(x_rows, x_across, s_rows, p, stream);
}

}  // namespace sbp
