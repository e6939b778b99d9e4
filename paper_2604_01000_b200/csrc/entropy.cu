// Softmax cross entropy of x W^T + b over many classes, and its gradient; the logits only ever exist a piece at a time.
//
//     l = x W^T + b;   lse = log sum_c exp l_c;   row_loss = lse - l_target;   loss = mean of row_loss over the rows that count
//     G = (exp(l - lse) - [c = target]) g,  g = dloss / rows + drow;   dx = G W;   dW = G^T x;   db = column sums of G
//
// Of 16-bit inputs a tile of logits never leaves the tensor memory: the threads that read it there keep a running maximum
// and sum for each row (forward), or make a tile of G of it (backward), in the operands' type, for two more products.  G exists a
// piece at a time (some rows by some classes, small enough to stay in the L2 until both products have read it).
// fp32 inputs are split into three bf16 numbers as in linear.cu; a piece of their logits is made by the products' own tile
// kernel, and row kernels go over it to the same ends; few of them, and few 16-bit ones' gradients, go without either (small problems, below).
// Logits of more than 256 16-bit elements are summed in runs (sums_log2e, below).
//
// Measured, on the device.  Forward of 169343 x 128 -> 4096 bf16: 231 us; the product alone would need 109 us at 1625 TFLOP/s, its 694
// million exponentials 154 us at 16 a clock and SM: bound by the issue of what is around them (0.44 a clock and scheduler; the tensor pipe
// is 33 % busy).  Backward: 691 us, of three products 328 us and of the exponentials, made for either gradient, 308 us; 4096 x 256 -> 169343
// fp16: 1291 us of 656 us: bound by the hand-over of tiles between the tensor core and the 16 warps that make G (tensor pipe 40 to
// 48 % busy, issue 0.24 to 0.47).  fp32: forward of 128 x 64 -> 32 8.4 us: latency; backward of
// 2999 x 65 -> 257 33 us, of which its multiply-adds, fed from shared memory, 26.
#include "ep_common.cuh"
#include "rows.cuh"
#include "tile_device.cuh"

#include <algorithm>
#include <cfloat>
#include <type_traits>

using namespace eprow;
using namespace eptile;
using ep::Matrix;
using ep::Operand;
using ep::Packed;

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// What is known of a row's softmax: exponentials sum to s with the maximum m taken out.
struct Running {
    float m, s;
};
__device__ __forceinline__ Running join(Running a, Running b) {
    const float m = fmaxf(a.m, b.m), shift = m == -INFINITY ? 0.f : m;
    return {m, a.s * exp_fast(a.m - shift) + b.s * exp_fast(b.m - shift)};
}

// A row's target class, or -1 where it has none.  (One outside the classes raises the status and counts as none.)
__device__ __forceinline__ int target_of(const int32_t *targets, int64_t row, int classes, int *status) {
    const int t = targets[row];
    if (t >= -1 && t < classes) return t;
    ep_raise(status, EP_ERR_BAD_INDEX);
    return -1;
}

// ---------------------------------------------------------------------------------------------- logits by tiles
//
// A pair of blocks works on 256 rows x 256 classes at a time (see linear.cu, whose pipeline this is: one warp loads, one of
// the first block multiplies, 16 finish a tile, or take a run's sums, while the next is being summed).  Workers share out the tiles evenly, in
// one long line: row tile after row tile in the forward (a thread keeps its row's statistics from tile to tile), class tile after
// class tile in the backward (a thread keeps its classes' sums), each worker a stretch of it.  What a worker has when its
// stretch or its row (class) tile ends is a partial result, number `worker - first worker of that tile`.
constexpr int TILE = 256;
constexpr int BLOCK_ROWS = 128, PIECE_COLS = 64;   // a block's rows; the columns of a warp that finishes tiles
constexpr int EPI_WARPS = 16, TILE_THREADS = 32 * (EPI_WARPS + 2);
constexpr int STAGE_BYTES = 2 * BLOCK_ROWS * 128, SLOT_BYTES = 4096;

struct TileShared {
    uint64_t full[8], empty[8], t_full[2], t_empty[2], drain;
    uint32_t tmem_base;
    int abort;
};
template <bool GRAD>
struct TileMemory {
    static constexpr int STAGING = GRAD ? EPI_WARPS * SLOT_BYTES : 0;
    static constexpr int STAGES = GRAD ? 5 : 6;
    static constexpr int RING = STAGES * STAGE_BYTES;
    static constexpr size_t TOTAL = 1024 + RING + STAGING + sizeof(TileShared);
    static_assert(TOTAL <= 227 * 1024, "shared memory of a block");
};

// tiles = outer x inner, in a line with `inner` fastest; worker w of n has [tiles w / n, tiles (w + 1) / n).
struct Line {
    int64_t tiles;
    int inner, workers;
    __host__ __device__ int64_t begin(int w) const { return tiles * w / workers; }   // (below 2^47)
    __host__ __device__ int worker_of(int64_t tile) const { return (int)(((tile + 1) * workers - 1) / tiles); }
    __host__ __device__ int first_worker(int64_t outer) const { return worker_of(outer * inner); }
    __host__ __device__ int last_worker(int64_t outer) const { return worker_of(outer * inner + inner - 1); }
};
struct Stretch {
    int64_t left;
    int outer, inner;
    const int inners;
    __device__ __forceinline__ Stretch(const Line &l, int worker) : inners(l.inner) {
        const int64_t from = l.begin(worker);
        left = l.begin(worker + 1) - from;
        outer = (int)(from / l.inner);
        inner = (int)(from - (int64_t)outer * l.inner);
    }
    __device__ __forceinline__ bool more() const { return left > 0; }
    __device__ __forceinline__ void next() {
        --left;
        if (++inner == inners) {
            inner = 0;
            ++outer;
        }
    }
};

// What the blocks of entropy_weights have found, together.  G is rounded to 16 bits, so what it is measured in matters.
// The gradient of a mean (no weights of the rows' own) has the same g in every row, and -g where the target is unlikely: rounded, all of
// a gradient would be off by the same up to 2^-8 in bf16.  There G is measured in |g|, 2^14 of which are 1 in fp16, and the products' sums are
// multiplied by |g|: -1 is exact, and what is rounded are chances (of a target less likely than 2^-9, p is lost beside 1).  255 x 64 rows of 3000
// classes, bf16: gradients were off by 3.6e-3 in common, now by p = 3.3e-4; in all by 0.0017 of themselves, as their own rounding leaves.
// Otherwise fp16, which holds nothing below 2^-25, takes the power of two that brings the largest |g| to [2^14, 2^15) (|p - 1| is at
// most 1), and the sums its inverse.
// up: what g and the slopes still have to be multiplied by.
struct Scale {
    float up, down;
    int unclean;
};
// What the backward knows of each row, padded by a tile.  Rows that take no part, and those past the end: -infinity, 0, -1.
struct RowInfo {
    float *shift;   // -lse / log 2 + log2 |g|: the slope of a class that is not the target is 2^(l / log 2 + shift), or minus that
    float *g;       // in what G is measured in
    int *target;
    __host__ __device__ RowInfo from(int64_t row) const { return RowInfo{shift + row, g + row, target + row}; }
};
// The tensor cores cut a sum off after every 16 products, toward zero, they do not round it.  What that costs depends on what is summed:
// nothing where the sum fits fp32 (rows of one element, or of few bits), 1e-7 of the sum a step where all products have one sign, and
// of dense rows of either sign, on average and within a fifth, (2.5 + 1.5 steps) 1e-8 of the sum in bf16, (5 + 1.9 steps) 1e-8 in fp16.
// So a logit of more than 256 elements is summed in runs of 16 such steps, as fp32 products are in linear.cu, which are added up to nearest
// in registers: however long it is, it loses what one run does.  (Forward and backward, us, in one run -> in such: 169343 x 512 -> 4096 bf16
// 440 -> 501 and 2162 -> 2503, 20000 x 1024 -> 4096 107 -> 119 and 472 -> 532, 8192 x 4096 -> 4096 197 -> 213 and 581 -> 626: a run is handed
// over while there is room for one more.  Runs of 8 steps would lose half as much and take 612, 138 and 223; 2794, 549 and 628.)
// Up to 256 elements a logit is one run, of up to 16 steps.  Many rows' sums (dbias) would keep the part of its loss that has always the same
// sign (100000 x 256 -> 10 in bf16: dbias off by 1.4e-5 of itself, so by 1.1e-6); what dense rows lose on average is therefore given back there
// with the factor 1 / log 2: at most 3.6e-7 of the logit, three units of fp32's last place, by which a sum that lost nothing is too large.
constexpr int ONE_RUN = 256, RUN_KB = ONE_RUN / 64;   // elements of a run, and its k-blocks
float sums_log2e(int n_in, int type) {
    const double steps = (n_in + 15) / 16, lost = n_in > ONE_RUN ? 0.0 : type == EP_BF16 ? 2.5 + 1.5 * steps : 5.0 + 1.9 * steps;
    return (float)(1.4426950408889634 * (1.0 + 1e-8 * lost));
}
struct TileWork {
    int64_t M;
    int N, class0, kb;
    Line line;
    uint32_t idesc;
    float log2e;              // of sums_log2e
    const float *bias;        // / log 2, of all classes, padded by a tile; or NULL
    const int32_t *targets;
    float2 *partial;          // forward: [number * 4 + piece][M], over log 2
    float *at_target;
    unsigned *ticket;
    RowInfo rows;             // backward
    const Scale *scale;
    float *sums;              // [number * 8 + block's and warp's rows][stride], or NULL
    int64_t stride;
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// One column of this warp's lanes.
__device__ __forceinline__ float tmem_ld_column(uint32_t taddr) {
    uint32_t v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\ntcgen05.wait::ld.sync.aligned;" : "=r"(v) : "r"(taddr) : "memory");
    return __uint_as_float(v);
}
// 16 lanes of 32 accumulator columns, waited for in the same statement: lane l holds rows l / 4 and l / 4 + 8, of each 8 columns two
// from 2 (l % 4) on: v[4 c + 2 r + i] is column 8 c + 2 (l % 4) + i of row l / 4 + 8 r.
__device__ __forceinline__ void tmem_ld_rows16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}
// Four 8 x 8 matrices of 16-bit elements in the layout above, lane l's address that of row l % 8 of matrix l / 8.
__device__ __forceinline__ void store_matrices(void *at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(smem_u32(at)), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}
template <typename T>
__device__ __forceinline__ uint32_t packed(float lo, float hi) {
    if constexpr (std::is_same_v<T, __half>) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    } else {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
}

// RUNS: rows of more than ONE_RUN elements, which those of the backward always are.  (BIASED: of the forward alone)
template <bool GRAD, bool BIASED, bool RUNS, typename T>
__global__ void __launch_bounds__(TILE_THREADS, 1) entropy_tiles(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                                                                 const __grid_constant__ CUtensorMap map_g, const __grid_constant__ CUtensorMap map_clean,
                                                                 const TileWork e, int *status) {
    using Mem = TileMemory<GRAD>;
    constexpr int STAGES = Mem::STAGES;
    static_assert(RUNS || !GRAD, "the backward of shorter rows is entropy_fused");
    extern __shared__ char smem_raw[];
    char *ring = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    char *staging = ring + Mem::RING;
    TileShared *sh = reinterpret_cast<TileShared *>(staging + Mem::STAGING);
    const uint32_t rank = cluster_rank();     // rank 0 issues the MMAs
    const int worker = blockIdx.x >> 1;
    volatile int *abort_flag = &sh->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&sh->full[s], 1);
            mbar_init(&sh->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sh->t_full[b], 1);
            mbar_init(&sh->t_empty[b], 2 * EPI_WARPS);   // (of both blocks, at the first one's)
        }
        mbar_init(&sh->drain, 1);
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(2 * TILE)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_meet();   // the other block's barriers are ready
    tc_fence_after();
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    const uint32_t tmem_base = sh->tmem_base;
    if (!GRAD && blockIdx.x == 0 && threadIdx.x == 0) *e.ticket = 0;   // of entropy_finish
    auto row_tile = [](const Stretch &t) { return GRAD ? t.inner : t.outer; };
    auto class_tile = [](const Stretch &t) { return GRAD ? t.outer : t.inner; };
    // columns that the MMAs compute: the last tile's are cut to what there is
    auto columns = [&](int n) { return min(TILE, (e.N - n * TILE + 31) & ~31); };

    if (warp == EPI_WARPS) {
        uint32_t it = 0, s = 0, ph = 0;
        bool ok = true;
        const uint32_t ring_base = smem_u32(ring);
        const CUtensorMap *const from_x = GRAD && e.scale->unclean ? &map_clean : &map_x;
        for (Stretch t(e.line, worker); ok && t.more(); t.next()) {
            const int m = row_tile(t) * TILE + (int)rank * BLOCK_ROWS, n = class_tile(t) * TILE + (int)rank * (columns(class_tile(t)) / 2);
            for (int kb = 0; kb < e.kb; ++kb, ++it) {
                if (!(ok = mbar_wait_warp(&sh->empty[s], ph ^ 1u, abort_flag))) break;
                if (rank == 0) mbar_expect_tx_elected(&sh->full[s], 2 * STAGE_BYTES);
                const uint32_t bar = in_block(smem_u32(&sh->full[s]), 0), dst = ring_base + s * (uint32_t)STAGE_BYTES;
                load_tile_elected<true>(dst, from_x, kb * 64, m, 0, bar);
                load_tile_elected<true>(dst + BLOCK_ROWS * 128, &map_w, kb * 64, n, 0, bar);
                if (++s == (uint32_t)STAGES) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
        // after an abort the loads already issued get time to land before the block leaves
        if (rank == 0 && lane == 0 && (!ok || *abort_flag))
#pragma unroll 1
            for (uint32_t j = it > (uint32_t)STAGES ? it - (uint32_t)STAGES : 0u; j < it; ++j)
                mbar_wait_quiet(&sh->full[j % (uint32_t)STAGES], (j / (uint32_t)STAGES) & 1u, DRAIN_LIMIT_CLOCKS);
    } else if (warp == EPI_WARPS + 1) {
        uint32_t acc = 0, s = 0, ph = 0;
        bool ok = true;
        const uint32_t ring_base = smem_u32(ring);
        for (Stretch t(e.line, worker); rank == 0 && ok && t.more(); t.next()) {
            const uint32_t idesc = e.idesc | (uint32_t)(columns(class_tile(t)) >> 3) << 17;
            int kb = 0;
            do {
                const uint32_t buf = acc & 1u;
                if (!(ok = mbar_wait_warp(&sh->t_empty[buf], ((acc >> 1) & 1u) ^ 1u, abort_flag))) break;
                tc_fence_after();
                const int first = kb, end = RUNS ? min(kb + RUN_KB, e.kb) : e.kb;
                for (; kb < end; ++kb) {
                    if (!(ok = mbar_wait_warp(&sh->full[s], ph, abort_flag))) break;
                    tc_fence_after();
                    const uint32_t a = ring_base + s * (uint32_t)STAGE_BYTES;
                    umma_kblock_elected<HALF, true>(tmem_base + buf * TILE, operand_desc(a, false), operand_desc(a + BLOCK_ROWS * 128, false), 2,
                                                    2, idesc, kb > first);
                    commit_elected<true>(&sh->empty[s]);
                    if (++s == (uint32_t)STAGES) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                if (ok) commit_elected<true>(&sh->t_full[buf]);
                ++acc;
            } while (RUNS && ok && kb < e.kb);
        }
        if (rank == 0 && __any_sync(FULL, !ok || *abort_flag)) {
            commit_elected<true>(&sh->drain);
            if (lane == 0) mbar_wait_quiet(&sh->drain, 0u, DRAIN_LIMIT_CLOCKS);
        }
    } else {
        const int quad = warp & 3, piece = warp >> 2;   // TMEM lanes 32 quad.. and 64 columns are this warp's
        const uint32_t t_empty = in_block(smem_u32(&sh->t_empty[0]), 0);
        const uint32_t from = tmem_base + ((uint32_t)(quad * 32) << 16) + piece * PIECE_COLS;
        auto give_back = [&](uint32_t buf) {   // the accumulator, once every column of it is in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(t_empty + buf * 8);
        };
        uint32_t acc = 0;   // accumulators so far, a run's each
        const float log2e = e.log2e;
        // take(buffer) of each run of a tile's sums, if there is any of it that is wanted; false after an abort
        auto each_run = [&](bool wanted, auto take) {
            for (int run = 0; run < e.kb; run += RUN_KB, ++acc) {
                if (!mbar_wait_warp(&sh->t_full[acc & 1u], (acc >> 1) & 1u, abort_flag)) return false;
                tc_fence_after();
                if (wanted) take(from + (acc & 1u) * TILE);
                give_back(acc & 1u);
            }
            return true;
        };
        if constexpr (!GRAD) {
            float top = -FLT_MAX, sum = 0.f;   // (finite from the start: what is closed is below it)
            int target = -1;
            for (Stretch t(e.line, worker); t.more(); t.next()) {
                const int64_t row = (int64_t)t.outer * TILE + rank * BLOCK_ROWS + quad * 32 + lane;
                const int col = t.inner * TILE + piece * PIECE_COLS;
                if (acc == 0 || t.inner == 0) target = row < e.M ? e.targets[row] : -1;
                // these logits into the row's statistics; mine: the target's column, if it is one of these, found: its logit
                auto count = [&](float (&f)[64], int mine, float found) {
                    if ((unsigned)mine < 64u) e.at_target[row] = BIASED ? fmaf(found, log2e, e.bias[target]) : found * log2e;
                    if (BIASED) {
#pragma unroll
                        for (int j = 0; j < 64; j += 4) {
                            const float4 add = *reinterpret_cast<const float4 *>(e.bias + col + j);
                            fma2(Pair(f[j], f[j + 1]), Pair(log2e), Pair(add.x, add.y)).get(f[j], f[j + 1]);
                            fma2(Pair(f[j + 2], f[j + 3]), Pair(log2e), Pair(add.z, add.w)).get(f[j + 2], f[j + 3]);
                        }
                    }
                    if (col + PIECE_COLS > e.N) {
#pragma unroll
                        for (int j = 0; j < 64; ++j) f[j] = col + j < e.N ? f[j] : -INFINITY;
                    }
                    const float scale = BIASED ? 1.f : log2e;
                    auto sum_below = [&](float shift) {   // of 2^(f - shift)
                        Pair s0(0.f), s1(0.f);
#pragma unroll
                        for (int j = 0; j < 64; j += 4) {
                            float x0, x1, x2, x3;
                            fma2(Pair(f[j], f[j + 1]), Pair(scale), Pair(-shift)).get(x0, x1);
                            fma2(Pair(f[j + 2], f[j + 3]), Pair(scale), Pair(-shift)).get(x2, x3);
                            s0 = add2(s0, Pair(exp2_fast(x0), exp2_fast(x1)));
                            s1 = add2(s1, Pair(exp2_fast(x2), exp2_fast(x3)));
                        }
                        float lo, hi;
                        add2(s0, s1).get(lo, hi);
                        return lo + hi;
                    };
                    // What is taken out of the exponents need not be the maximum, only near it: the largest so far does unless this
                    // tile goes above it by 2^64, and its exponentials need not wait for the maximum to be known.
                    float more = sum_below(top);
                    float high = f[0];
#pragma unroll
                    for (int j = 1; j + 1 < 64; j += 2) high = max3(high, f[j], f[j + 1]);
                    high = fmaxf(high, f[63]) * scale;
                    if (__any_sync(FULL, high > top + 64.f)) {
                        const float now = fmaxf(top, high);
                        sum *= exp2_fast(top - now);
                        top = now;
                        more = sum_below(top);
                    }
                    sum += more;
                };
                if constexpr (RUNS) {
                    const bool wanted = col < e.N && row - lane < e.M;
                    float f[64], found = 0.f;
#pragma unroll
                    for (int j = 0; j < 64; ++j) f[j] = 0.f;
                    if (!each_run(wanted, [&](uint32_t at) {
#pragma unroll
                            for (int q = 0; q < 64; q += 16) {
                                uint32_t a[16];
                                tmem_ld16(at + q, a);
#pragma unroll
                                for (int j = 0; j < 16; j += 2)
                                    add2(Pair(f[q + j], f[q + j + 1]), Pair(__uint_as_float(a[j]), __uint_as_float(a[j + 1])))
                                        .get(f[q + j], f[q + j + 1]);
                            }
                        }))
                        break;
                    if (wanted) {
                        const int mine = target >= 0 ? target - col : -1;
                        if (__any_sync(FULL, (unsigned)mine < 64u)) {
#pragma unroll
                            for (int j = 0; j < 64; ++j) found = j == mine ? f[j] : found;
                        }
                        count(f, mine, found);
                    }
                } else {
                    const uint32_t buf = acc & 1u;
                    if (!mbar_wait_warp(&sh->t_full[buf], (acc >> 1) & 1u, abort_flag)) break;
                    tc_fence_after();
                    if (col < e.N && row - lane < e.M) {
                        const uint32_t at = from + buf * TILE;
                        uint32_t a[64];
                        tmem_ld32_issue(at, reinterpret_cast<uint32_t(&)[32]>(a[0]));
                        tmem_ld32_issue(at + 32, reinterpret_cast<uint32_t(&)[32]>(a[32]));
                        // The logits of targets among these columns: a column to each, read once more.
                        const int mine = target >= 0 ? target - col : -1;
                        unsigned hits = __ballot_sync(FULL, (unsigned)mine < 64u);
                        const bool few = __popc(hits) <= 4;
                        float found = 0.f;
                        for (; few && hits; hits &= hits - 1) {
                            const int who = __ffs(hits) - 1;
                            const float v = tmem_ld_column(at + __shfl_sync(FULL, mine, who));
                            if (lane == who) found = v;
                        }
                        tmem_ld_wait(reinterpret_cast<uint32_t(&)[32]>(a[0]));
                        tmem_ld_wait(reinterpret_cast<uint32_t(&)[32]>(a[32]));
                        give_back(buf);
                        float f[64];
#pragma unroll
                        for (int j = 0; j < 64; ++j) f[j] = __uint_as_float(a[j]);
                        if (!few) {
#pragma unroll
                            for (int j = 0; j < 64; ++j) found = j == mine ? f[j] : found;
                        }
                        count(f, mine, found);
                    } else
                        give_back(buf);
                    ++acc;
                }
                if (t.left == 1 || t.inner + 1 == t.inners) {
                    if (row < e.M) e.partial[((int64_t)(worker - e.line.first_worker(t.outer)) * 4 + piece) * e.M + row] = make_float2(top, sum);
                    top = -FLT_MAX;
                    sum = 0.f;
                }
            }
        } else {
            char *slot = staging + warp * SLOT_BYTES;
            const float up = e.scale->up, down = e.scale->down;
            Pair sums[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) sums[c] = Pair(0.f);
            for (Stretch t(e.line, worker); t.more(); t.next()) {
                const int64_t row0 = (int64_t)t.inner * TILE + rank * BLOCK_ROWS + quad * 32;
                const int col = t.outer * TILE + piece * PIECE_COLS;
                const bool wanted = col < e.N && row0 < e.M;
                float v[2][32];   // 16 rows each, as tmem_ld_rows16 has them
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int q = 0; q < 32; ++q) v[h][q] = 0.f;
                if (!each_run(wanted, [&](uint32_t at) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int q = 0; q < 32; q += 16) {
                                uint32_t a[16];
                                tmem_ld_rows16(at + ((uint32_t)(16 * h) << 16) + 2 * q, a);
#pragma unroll
                                for (int j = 0; j < 16; j += 2)
                                    add2(Pair(v[h][q + j], v[h][q + j + 1]), Pair(__uint_as_float(a[j]), __uint_as_float(a[j + 1])))
                                        .get(v[h][q + j], v[h][q + j + 1]);
                            }
                    }))
                    break;
                if (wanted) {
                    stores_read<0>();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float shift[2], weight[2], sign[2];
                        int target[2];
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const int64_t row = row0 + 16 * h + 8 * r + (lane >> 2);
                            const float g = e.rows.g[row];
                            shift[r] = e.rows.shift[row];
                            weight[r] = fabsf(g);
                            sign[r] = g < 0.f ? -up : up;
                            target[r] = e.rows.target[row];
                        }
                        float(&f)[32] = v[h];
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const float2 b = e.bias ? *reinterpret_cast<const float2 *>(e.bias + e.class0 + col + 8 * c + 2 * (lane & 3)) : float2{};
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                Pair l = fma2(Pair(f[4 * c + 2 * r], f[4 * c + 2 * r + 1]), Pair(log2e), Pair(shift[r]));
                                if (e.bias) l = add2(l, Pair(b.x, b.y));
                                l.get(f[4 * c + 2 * r], f[4 * c + 2 * r + 1]);
                            }
                        }
#pragma unroll
                        for (int q = 0; q < 32; ++q) f[q] = exp2_fast(f[q]);
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const int at = target[r] - e.class0 - col;
                            const bool mine = target[r] >= 0 && (unsigned)at < 64u && ((at >> 1) & 3) == (lane & 3);
                            const int index = mine ? (at >> 3) * 2 + (at & 1) : -1;
                            if (__any_sync(FULL, mine)) {
#pragma unroll
                                for (int q = 0; q < 16; ++q) f[4 * (q >> 1) + 2 * r + (q & 1)] -= q == index ? weight[r] : 0.f;
                            }
                        }
                        uint32_t out[16];
#pragma unroll
                        for (int c = 0; c < 8; ++c)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const Pair g = mul2(Pair(f[4 * c + 2 * r], f[4 * c + 2 * r + 1]), Pair(sign[r]));
                                if (e.sums) sums[c] = add2(sums[c], g);
                                float lo, hi;
                                g.get(lo, hi);
                                out[2 * c + r] = packed<T>(lo, hi);
                            }
                        const int r = 16 * h + (lane & 15);   // the row whose address this lane gives
#pragma unroll
                        for (int c = 0; c < 8; c += 2)
                            store_matrices(slot + r * 128 + (((c + (lane >> 4)) ^ (r & 7)) << 4), out[2 * c], out[2 * c + 1], out[2 * c + 2],
                                           out[2 * c + 3]);
                    }
                    before_stores();
                    tma_store_3d_elected(&map_g, slot, col, (int)row0, 0);
                }
                if (e.sums && (t.left == 1 || t.inner + 1 == t.inners)) {
                    float *to = e.sums + ((int64_t)(worker - e.line.first_worker(t.outer)) * 8 + rank * 4 + quad) * e.stride + col;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        float lo, hi;
                        sums[c].get(lo, hi);
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) {
                            lo += __shfl_xor_sync(FULL, lo, o);
                            hi += __shfl_xor_sync(FULL, hi, o);
                        }
                        const int at = 8 * c + 2 * (lane & 3);
                        if (lane < 4 && col + at < e.N) to[at] = lo * down;
                        if (lane < 4 && col + at + 1 < e.N) to[at + 1] = hi * down;
                        sums[c] = Pair(0.f);
                    }
                }
            }
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // what has been stored is written before the block ends
    }
    __syncthreads();
    cluster_meet();   // neither block leaves while the other may still signal it
    if (sh->abort && threadIdx.x == 0) ep_raise(status, EP_ERR_TIMEOUT);
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(2 * TILE) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------- backward of narrow rows
//
// Rows of up to 256 elements leave room in the tensor memory for 128 rows of a gradient beside the logits, so G need not
// leave the SM either.  One kernel serves both gradients, the roles of x and W exchanged: 128 rows P of one stay in
// shared memory, tiles Q of 128 rows of the other go by;
//     S = P Q^T;   G = slopes of S, in the operands' type;   acc += G Q
// with all three in the tensor memory and G multiplied from there (a product whose first operand is in the tensor memory
// reads half as much of the shared memory, which otherwise could not keep up).  P = rows of x gives dx, P = classes gives dW
// and dbias; the logits are so made twice, four products in all where three would do, but G (two bytes for 4 n_in operations, written
// once and read twice) is not moved (169343 x 128 -> 4096 bf16: 1548 us with G written and read, 691 so).  Of 19 warps one loads, one makes S, one adds up, 16 make G: groups of
// them take tiles in turn, a thread a row of S and 64 columns.
// Workers (SMs) share out the tiles as in entropy_tiles; who has only a part of a P tile leaves its sums for entropy_join.
constexpr int FUSED_WIDTH = ONE_RUN;   // the widest rows
constexpr int P_ROWS = 128, FUSED_THREADS = 32 * (EPI_WARPS + 3);
struct FusedShared {
    uint64_t full[8], empty[8], p_full[2], p_empty[2], s_full[2], s_empty[2], g_full[2], g_empty[2], acc_full, acc_empty, sums_full, drain[2];
    uint32_t tmem_base;
    int abort;
    double sums[2][4][P_ROWS];   // of a class's slopes, by each of its row's four warps; of P tiles in turn
};
constexpr int Q_ROWS = 128;
// WIDE: rows of more than 128 elements.
template <bool DW, bool WIDE>
struct FusedMemory {
    static constexpr int BOXES = WIDE ? 4 : 2;                   // of 64 elements, of a row at most
    static constexpr int P_BUFFERS = WIDE ? 1 : 2;
    static constexpr int P_BYTES = BOXES * P_ROWS * 128;
    static constexpr int EXTRA = (DW ? 3 : 1) * Q_ROWS * 4;      // what is known of Q's rows: shift, g, target; or the classes' bias
    static constexpr int Q_BYTES = BOXES * Q_ROWS * 128, STAGE = Q_BYTES + 2048;
    static constexpr int STAGES = WIDE ? 2 : 4;
    // The tensor memory: a tile or two of S, two of G (two of its numbers to a column), the sums.  (G has columns of its own, so that
    // beside sums of 256 columns there is room for one S.  Tiles of 64 rows of Q, two of which fit, need twice the instructions of S
    // and have the shared memory read P twice as often: 4096 x 256 -> 169343 in 1340 us.)
    static constexpr int LOGITS = WIDE ? 1 : 2, SLOPES = 2;
    static constexpr int G_AT = LOGITS * Q_ROWS, ACC = G_AT + SLOPES * Q_ROWS / 2;
    static constexpr size_t TOTAL = 1024 + P_BUFFERS * P_BYTES + STAGES * STAGE + sizeof(FusedShared);
    static_assert(TOTAL <= 227 * 1024 && ACC + BOXES * 64 <= 512, "a block's shared and tensor memory");
};
struct FusedWork {
    int64_t P, Q;             // rows of either
    int ragged;               // the tile of Q that has classes past the last, or -1
    int width, boxes;         // of a row, and its boxes
    Line line;
    uint32_t idesc_s, idesc_acc;
    float log2e;              // of sums_log2e
    const float *bias;        // of the classes, over log 2, padded; or NULL
    RowInfo rows;
    const Scale *scale;
    void *out;                // or NULL
    float *dbias;             // of DW, or NULL
    bool vec;                 // out can be written by 16 bytes
    float *share;             // [2 worker + segment][P_ROWS][share_ld]: sums of part of a P tile; then its dbias [..][P_ROWS]
    double *share_bias;
    int share_ld;             // (behind share, too: [worker][share_ld / 4][P_ROWS][4], the runs so far of a worker's P tile)
};
// Where a worker's part of P tile `tile` lies: its first segment's place, or its last one's.
__host__ __device__ __forceinline__ int64_t share_of(const Line &l, int worker, int64_t tile) {
    return 2 * worker + (l.begin(worker) / l.inner == tile ? 0 : 1);
}

__device__ __forceinline__ void bulk_load_elected(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                 "@pe cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n}" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
// acc += G Q over 64 columns of G: four steps of 16, G in the tensor memory, two of its numbers to a column.
__device__ __forceinline__ void umma_from_tmem_elected(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate_first) {
    const uint64_t b1 = b + (2048 >> 4), b2 = b1 + (2048 >> 4), b3 = b2 + (2048 >> 4);
    asm volatile("{\n.reg .pred pe, pa, pt;\n"
                 "elect.sync _|pe, 0xffffffff;\n"
                 "setp.ne.b32 pa, %10, 0;\nsetp.eq.b32 pt, 0, 0;\n"
                 "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %5, %9, pa;\n"
                 "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [%2], %6, %9, pt;\n"
                 "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [%3], %7, %9, pt;\n"
                 "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [%4], %8, %9, pt;\n}" ::"r"(d_tmem),
                 "r"(a_tmem), "r"(a_tmem + 8), "r"(a_tmem + 16), "r"(a_tmem + 24), "l"(b), "l"(b1), "l"(b2), "l"(b3), "r"(idesc),
                 "r"(accumulate_first)
                 : "memory");
}

// The sums of a run, or of the last one of a P tile or of this worker's part of it (over): put away, or with the earlier runs' to the gradient or this
// worker's share.  By the 16 warps that make G, 32 columns of 32 rows each at a time.  false after an abort.  (What is put away lies so that a warp's
// rows are side by side: 4096 x 256 -> 169343 in fp16, whose sums are put away after each 64 tiles, 1290 us; in rows as they are shared 1335; never 1290.)
template <bool DW, bool WIDE, typename T>
__device__ __forceinline__ bool put_away(const FusedWork &e, FusedShared *sh, int worker, int outer, int inner, bool over, int run) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = warp & 3, column = warp >> 2;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const int64_t p = (int64_t)outer * P_ROWS + quad * 32 + lane;
    const float down = e.scale->down;
    tc_fence_after();
    const bool whole = e.line.first_worker(outer) == e.line.last_worker(outer);
    const int64_t place = share_of(e.line, worker, outer), begin = e.line.begin(worker);
    const int before = (int)(begin / e.line.inner);   // the P tile that this worker begins in
    const bool kept = inner / run > (outer == before ? (int)(begin - (int64_t)before * e.line.inner) : 0) / run;   // earlier runs' sums
    // (this thread's own: four columns of its row at a time, those of a warp's rows side by side)
    float4 *const away = reinterpret_cast<float4 *>(e.share + (int64_t)(2 * e.line.workers + worker) * P_ROWS * e.share_ld) + quad * 32 + lane;
#pragma unroll 1
    for (int c0 = column * 32; c0 < e.width && e.out; c0 += 128) {
        uint32_t a[32];
        tmem_ld32_issue(lanes + FusedMemory<DW, WIDE>::ACC + c0, a);
        tmem_ld_wait(a);
        float v[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) v[c] = __uint_as_float(a[c]);
        if (kept) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
                const float4 k = away[(c0 + c) / 4 * P_ROWS];
                v[c] += k.x, v[c + 1] += k.y, v[c + 2] += k.z, v[c + 3] += k.w;
            }
        }
        if (!over) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) away[(c0 + c) / 4 * P_ROWS] = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
        } else if (!whole) {
            float *to = e.share + (place * P_ROWS + quad * 32 + lane) * e.share_ld + c0;
#pragma unroll
            for (int c = 0; c < 32; c += 4) *reinterpret_cast<float4 *>(to + c) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
        } else if (p < e.P) {
            T *to = static_cast<T *>(e.out) + p * e.width;
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = v[c + i] * down;
                store_chunk(to, c0 + c, e.width, e.vec, w);
            }
        }
    }
    if constexpr (DW) {
        if (e.dbias && over) {   // a class's sums are those of its row's four warps, in order
            const uint32_t turn = (uint32_t)(outer - before) & 1u;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->sums_full);
            if (column == 0) {   // (the others write there again only after these have given the sums of products back)
                if (!mbar_wait_warp(&sh->sums_full, turn, &sh->abort)) return false;
                const int c = quad * 32 + lane;
                const double(&part)[4][P_ROWS] = sh->sums[turn];
                const double sum = ((part[0][c] + part[1][c]) + (part[2][c] + part[3][c])) * (double)down;
                if (!whole)
                    e.share_bias[place * P_ROWS + c] = sum;
                else if (p < e.P)
                    e.dbias[p] = (float)sum;
            }
        }
    }
    return true;
}

template <bool DW, bool BIASED, bool WIDE, typename T>
__global__ void __launch_bounds__(FUSED_THREADS, 1) entropy_fused(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q,
                                                                 const __grid_constant__ CUtensorMap map_clean, const __grid_constant__ FusedWork e, int *status) {
    using Mem = FusedMemory<DW, WIDE>;
    constexpr int STAGES = Mem::STAGES, LOGITS = Mem::LOGITS, SLOPES = Mem::SLOPES;
    // Warps to a row of S; groups of warps that take tiles in turn.  What a group waits for has barriers of its own (a barrier that
    // went on by two phases meanwhile could not be told from one that has not moved).
    constexpr int BQ = Q_ROWS, COLUMN_WARPS = BQ / 64, GROUPS = 4 / COLUMN_WARPS;
    static_assert(STAGES % GROUPS == 0 && SLOPES % GROUPS == 0 && GROUPS <= 2, "a group's stages and slopes are its own");
    // Long sums are put away after 512 steps of 16 products (fp16) or 4096 (bf16), as in linear.cu: at tiles of Q whose number RUN divides.
    // (In one go of 10584 steps a column of fp16 gradients that should be 0 came out as 3.8e-4 of its terms.)
    constexpr int RUN = (std::is_same_v<T, __half> ? 512 : 4096) / (BQ / 16);
    auto ends_run = [](const Stretch &t) { return t.left == 1 || t.inner + 1 == t.inners || (t.inner + 1) % RUN == 0; };
    extern __shared__ char smem_raw[];
    char *p_room = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    char *ring = p_room + Mem::P_BUFFERS * Mem::P_BYTES;               // [STAGES] of Q
    char *extras = ring + STAGES * Mem::Q_BYTES;                       // [STAGES][2048]
    FusedShared *sh = reinterpret_cast<FusedShared *>(extras + STAGES * 2048);
    const int worker = blockIdx.x;
    volatile int *abort_flag = &sh->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&sh->full[s], 1);
            mbar_init(&sh->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sh->p_full[b], 1);
            mbar_init(&sh->p_empty[b], 1);
        }
        for (int b = 0; b < GROUPS; ++b) {
            mbar_init(&sh->s_full[b], 1);
            mbar_init(&sh->s_empty[b], 4 * COLUMN_WARPS);
        }
        for (int b = 0; b < SLOPES; ++b) {
            mbar_init(&sh->g_full[b], 4 * COLUMN_WARPS);
            mbar_init(&sh->g_empty[b], 1);
        }
        mbar_init(&sh->acc_full, 1);
        mbar_init(&sh->acc_empty, EPI_WARPS);
        mbar_init(&sh->sums_full, EPI_WARPS);
        mbar_init(&sh->drain[0], 1);
        mbar_init(&sh->drain[1], 1);
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    constexpr uint32_t tmem_base = 0;   // of an allocation of all 512 columns (known as such, addresses need no registers of a lane)

    if (warp == EPI_WARPS) {
        const bool unclean = e.scale->unclean;
        const CUtensorMap *const from_p = !DW && unclean ? &map_clean : &map_p, *const from_q = DW && unclean ? &map_clean : &map_q;
        uint32_t it = 0, s = 0, ph = 0, pb = 0, pph = 0, p_loads = 0;
        bool ok = true;
        for (Stretch t(e.line, worker); ok && t.more(); t.next(), ++it) {
            if (it == 0 || t.inner == 0) {
                if (!(ok = mbar_wait_warp(&sh->p_empty[pb], pph ^ 1u, abort_flag))) break;
                mbar_expect_tx_elected(&sh->p_full[pb], e.boxes * P_ROWS * 128);
                for (int b = 0; b < e.boxes; ++b)
                    load_tile_elected<false>(smem_u32(p_room) + pb * Mem::P_BYTES + b * P_ROWS * 128, from_p, b * 64, t.outer * P_ROWS, 0,
                                             smem_u32(&sh->p_full[pb]));
                ++p_loads;
                if (++pb == Mem::P_BUFFERS) {
                    pb = 0;
                    pph ^= 1u;
                }
            }
            if (!(ok = mbar_wait_warp(&sh->empty[s], ph ^ 1u, abort_flag))) break;
            const int q0 = t.inner * BQ;
            constexpr bool extra = DW || BIASED;
            mbar_expect_tx_elected(&sh->full[s], e.boxes * BQ * 128 + (extra ? Mem::EXTRA : 0));
            for (int b = 0; b < e.boxes; ++b)
                load_tile_elected<false>(smem_u32(ring) + s * Mem::Q_BYTES + b * BQ * 128, from_q, b * 64, q0, 0, smem_u32(&sh->full[s]));
            const uint32_t known = smem_u32(extras) + s * 2048;
            if (DW) {
                bulk_load_elected(known, e.rows.shift + q0, BQ * 4, &sh->full[s]);
                bulk_load_elected(known + BQ * 4, e.rows.g + q0, BQ * 4, &sh->full[s]);
                bulk_load_elected(known + 2 * BQ * 4, e.rows.target + q0, BQ * 4, &sh->full[s]);
            } else if (extra)
                bulk_load_elected(known, e.bias + q0, BQ * 4, &sh->full[s]);
            if (++s == (uint32_t)STAGES) {
                s = 0;
                ph ^= 1u;
            }
        }
        // after an abort the loads already issued get time to land before the block leaves
        if (lane == 0 && (!ok || *abort_flag)) {
#pragma unroll 1
            for (uint32_t j = it > (uint32_t)STAGES ? it - (uint32_t)STAGES : 0u; j < it; ++j)
                mbar_wait_quiet(&sh->full[j % (uint32_t)STAGES], (j / (uint32_t)STAGES) & 1u, DRAIN_LIMIT_CLOCKS);
#pragma unroll 1
            for (uint32_t j = p_loads > (uint32_t)Mem::P_BUFFERS ? p_loads - (uint32_t)Mem::P_BUFFERS : 0u; j < p_loads; ++j)
                mbar_wait_quiet(&sh->p_full[j % (uint32_t)Mem::P_BUFFERS], (j / (uint32_t)Mem::P_BUFFERS) & 1u, DRAIN_LIMIT_CLOCKS);
        }
    } else if (warp == EPI_WARPS + 1) {
        bool ok = true;
        const uint32_t p_base = smem_u32(p_room), q_base = smem_u32(ring);
        uint32_t j = 0, s = 0, ph = 0, buf = 0, pb = 0, pph = 0;
        for (Stretch t(e.line, worker); t.more(); t.next(), ++j) {
            if ((j == 0 || t.inner == 0) && !(ok = mbar_wait_warp(&sh->p_full[pb], pph, abort_flag))) break;
            if (!(ok = mbar_wait_warp(&sh->full[s], ph, abort_flag))) break;
            if (j >= (uint32_t)LOGITS) {
                const uint32_t before = j - LOGITS;
                if (!(ok = mbar_wait_warp(&sh->s_empty[before % GROUPS], (before / GROUPS) & 1u, abort_flag))) break;
            }
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < Mem::BOXES; ++b)
                if (b < e.boxes) umma_kblock_elected<HALF, false>(tmem_base + buf * BQ, operand_desc(p_base + pb * Mem::P_BYTES + b * P_ROWS * 128, false),
                                                 operand_desc(q_base + s * Mem::Q_BYTES + b * BQ * 128, false), 2, 2, e.idesc_s, b > 0);
            commit_elected<false>(&sh->s_full[j % GROUPS]);
            if (t.left == 1 || t.inner + 1 == t.inners) {
                commit_elected<false>(&sh->p_empty[pb]);
                if (++pb == Mem::P_BUFFERS) {
                    pb = 0;
                    pph ^= 1u;
                }
            }
            if (++s == (uint32_t)STAGES) {
                s = 0;
                ph ^= 1u;
            }
            if (++buf == (uint32_t)LOGITS) buf = 0;
        }
        if (__any_sync(FULL, !ok || *abort_flag)) {
            commit_elected<false>(&sh->drain[0]);
            if (lane == 0) mbar_wait_quiet(&sh->drain[0], 0u, DRAIN_LIMIT_CLOCKS);
        }
    } else if (warp == EPI_WARPS + 2) {
        bool ok = true;
        const uint32_t q_base = smem_u32(ring);
        uint32_t j = 0, s = 0, buf = 0, lap = 0, segment = 0;
        for (Stretch t(e.line, worker); t.more(); t.next(), ++j) {
            const bool first = j == 0 || t.inner % RUN == 0;
            if (!(ok = mbar_wait_warp(&sh->g_full[buf], lap, abort_flag))) break;
            if (first && !(ok = mbar_wait_warp(&sh->acc_empty, (segment & 1u) ^ 1u, abort_flag))) break;
            tc_fence_after();
            // (Q read along its rows: boxes of 64 elements lie BQ rows apart)
            const uint64_t q = ((uint64_t)((q_base + s * Mem::Q_BYTES) & 0x3FFFFu) >> 4) | ((uint64_t)(BQ * 128 >> 4) << 16) |
                               ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
#pragma unroll
            for (int k = 0; k < BQ / 64; ++k)
                umma_from_tmem_elected(tmem_base + Mem::ACC, tmem_base + Mem::G_AT + buf * (BQ / 2) + k * 32, q + k * (4 * 2048 >> 4), e.idesc_acc,
                                       !first || k > 0);
            commit_elected<false>(&sh->empty[s]);
            commit_elected<false>(&sh->g_empty[buf]);
            if (ends_run(t)) {
                commit_elected<false>(&sh->acc_full);
                ++segment;
            }
            if (++s == (uint32_t)STAGES) s = 0;
            if (++buf == (uint32_t)SLOPES) {
                buf = 0;
                lap ^= 1u;
            }
        }
        if (__any_sync(FULL, !ok || *abort_flag)) {
            commit_elected<false>(&sh->drain[1]);
            if (lane == 0) mbar_wait_quiet(&sh->drain[1], 0u, DRAIN_LIMIT_CLOCKS);
        }
    } else {
        const int quad = warp & 3, column = warp >> 2;   // TMEM lanes 32 quad.., and which of the warps that share them
        const int piece = column % COLUMN_WARPS, group = column / COLUMN_WARPS;
        const uint32_t lanes = tmem_base + ((uint32_t)(quad * 32) << 16);
        const float up = e.scale->up;
        uint32_t j = 0, segment = 0;
        int64_t p = 0;
        // of dx: what is known of this thread's row; of dW: its class's bias, and the scale of fp16
        int target = -1;
        float shift = 0.f, weight = 0.f, bias = 0.f;
        bool negative = false;                                 // some row's g is
        const float log_up = std::is_same_v<T, __half> ? log2f(up) : 0.f, log2e = e.log2e;
        double *total = nullptr;                               // (a class's slopes, of up to 2^31 rows; fp32 within a tile)
        uint32_t tiles = 0;
        for (Stretch t(e.line, worker); t.more(); t.next(), ++j) {
            if (j == 0 || t.inner == 0) {
                p = (int64_t)t.outer * P_ROWS + quad * 32 + lane;
                if constexpr (DW) {
                    if (BIASED) bias = (e.bias ? e.bias[p] : 0.f) + log_up;   // (padded)
                    total = &sh->sums[tiles++ & 1u][column][quad * 32 + lane];
                    *total = 0.0;
                } else {
                    shift = e.rows.shift[p] + log_up;
                    weight = e.rows.g[p] * up;
                    target = e.rows.target[p];
                    negative = __any_sync(FULL, weight < 0.f);
                }
            }
            if (j % GROUPS == (uint32_t)group) {
                const uint32_t s = j % STAGES, buf = j % LOGITS, gbuf = j % SLOPES;
                if (!mbar_wait_warp(&sh->s_full[group], (j / GROUPS) & 1u, abort_flag)) break;
                // (long since: what came with Q is there to read)
                if ((DW || BIASED) && !mbar_wait_warp(&sh->full[s], (j / STAGES) & 1u, abort_flag)) break;
                tc_fence_after();
                const float *known = reinterpret_cast<const float *>(extras + s * 2048) + piece * 64;
                const uint32_t at = lanes + buf * BQ + piece * 64, to = lanes + Mem::G_AT + gbuf * (BQ / 2) + piece * 32;
                uint32_t a[2][32];
                tmem_ld32_issue(at, a[0]);
                tmem_ld32_issue(at + 32, a[1]);
                // Where a row's class is among these columns, its slope is its share less all of g; and slopes may be negative.
                // Both are rare and out of the way of what is not.
                int mine = -1;
                bool special[2];
                if constexpr (DW) {
                    const int class0 = (int)p - lane;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        special[h] = __any_sync(FULL, (unsigned)(reinterpret_cast<const int *>(known)[2 * BQ + 32 * h + lane] - class0) < 32u ||
                                                          known[BQ + 32 * h + lane] < 0.f);
                } else {
                    mine = target >= 0 ? target - t.inner * BQ - piece * 64 : -1;
                    special[0] = negative || __any_sync(FULL, (unsigned)mine < 32u);
                    special[1] = negative || __any_sync(FULL, (unsigned)(mine - 32) < 32u);
                }
                tmem_ld_wait(a[0]);
                tmem_ld_wait(a[1]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->s_empty[group]);
                // Columns past the last class, which fill the last tile up, have no slope.  (Their logit of 0 may be far above all others:
                // 2^shift then passes the operands' type, and infinity times the zeros of W there is NaN.  Done here, not with the slopes
                // below, it costs the other tiles nothing; there it cost a tenth of dx.)
                if (!DW && t.inner == e.ragged) {
                    const int classes = (int)e.Q - t.inner * BQ - piece * 64;
#pragma unroll
                    for (int c = 0; c < 64; ++c)
                        if (c >= classes) a[c / 32][c % 32] = __float_as_uint(-INFINITY);
                }
                // (what was there has long been multiplied)
                if (!mbar_wait_warp(&sh->g_empty[gbuf], ((j / SLOPES) & 1u) ^ 1u, abort_flag)) break;
                tc_fence_after();
                Pair here(0.f);
                auto half = [&](int h, auto rare) {
                    [[maybe_unused]] const float *k = known + 32 * h;
                    float x[32];
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        Pair v0(__uint_as_float(a[h][c]), __uint_as_float(a[h][c + 1])), v1(__uint_as_float(a[h][c + 2]), __uint_as_float(a[h][c + 3]));
                        if constexpr (DW) {
                            const float4 z = *reinterpret_cast<const float4 *>(k + c);
                            v0 = fma2(v0, Pair(log2e), Pair(z.x, z.y));
                            v1 = fma2(v1, Pair(log2e), Pair(z.z, z.w));
                            if constexpr (BIASED) {
                                v0 = add2(v0, Pair(bias));
                                v1 = add2(v1, Pair(bias));
                            }
                        } else {
                            v0 = fma2(v0, Pair(log2e), Pair(shift));
                            v1 = fma2(v1, Pair(log2e), Pair(shift));
                            if constexpr (BIASED) {
                                const float4 b = *reinterpret_cast<const float4 *>(k + c);
                                v0 = add2(v0, Pair(b.x, b.y));
                                v1 = add2(v1, Pair(b.z, b.w));
                            }
                        }
                        v0.get(x[c], x[c + 1]);
                        v1.get(x[c + 2], x[c + 3]);
                    }
#pragma unroll
                    for (int c = 0; c < 32; ++c) x[c] = exp2_fast(x[c]);
                    if constexpr (decltype(rare)::value) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            if constexpr (DW) {
                                const float g = k[BQ + c];
                                x[c] = copysignf(1.f, g) * x[c] - (reinterpret_cast<const int *>(k)[2 * BQ + c] == (int)p ? g * up : 0.f);
                            } else
                                x[c] = copysignf(1.f, weight) * x[c] - (32 * h + c == mine ? weight : 0.f);
                        }
                    }
                    uint32_t out[16];
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        if (DW) here = add2(here, Pair(x[c], x[c + 1]));
                        out[c / 2] = packed<T>(x[c], x[c + 1]);
                    }
                    tmem_st16(to + 16 * h, out);
                };
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (special[h])
                        half(h, std::true_type{});
                    else
                        half(h, std::false_type{});
                }
                if constexpr (DW) {
                    float lo, hi;
                    here.get(lo, hi);
                    *total += (double)(lo + hi);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->g_full[gbuf]);
            }
            if (!ends_run(t)) continue;
            // the end of a run; of a P tile, or of this worker's part of it
            if (!mbar_wait_warp(&sh->acc_full, segment & 1u, abort_flag)) break;
            ++segment;
            if (!put_away<DW, WIDE, T>(e, sh, worker, t.outer, t.inner, t.left == 1 || t.inner + 1 == t.inners, RUN)) break;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->acc_empty);
        }
    }
    __syncthreads();
    if (sh->abort && threadIdx.x == 0) ep_raise(status, EP_ERR_TIMEOUT);
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh->tmem_base), "r"(512) : "memory");
    }
}

// The sums of P tiles that several workers had a part of, in the workers' order.  The tile that worker blockIdx.x begins inside
// of, if it is the first to do so (the second of those that share it); `rows` rows a block.
template <typename T>
__global__ void __launch_bounds__(256) entropy_join(const FusedWork e, int rows) {
    ep_wait_for_launch_before();
    const int64_t tile = e.line.begin(blockIdx.x) / e.line.inner;
    const int w0 = e.line.first_worker(tile), w1 = e.line.last_worker(tile);
    if (w0 == w1 || (int)blockIdx.x != w0 + 1) return;
    const float down = e.scale->down;
    const int row0 = blockIdx.y * rows, chunks = e.share_ld / 4;
    // (the first worker has it as its last segment unless that is its only one, the others as their first)
    const int64_t first = share_of(e.line, w0, tile);
    auto place = [&](int w) { return w == w0 ? first : 2 * (int64_t)w; };
    for (int i = threadIdx.x; i < rows * chunks && e.out; i += 256) {
        const int row = row0 + i / chunks, c = (i - i / chunks * chunks) * 4;
        const int64_t p = tile * P_ROWS + row;
        if (p >= e.P) break;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int w = w0; w <= w1; ++w) {
            const float4 v = *reinterpret_cast<const float4 *>(e.share + (place(w) * P_ROWS + row) * e.share_ld + c);
            sum[0] += v.x, sum[1] += v.y, sum[2] += v.z, sum[3] += v.w;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) sum[q] *= down;
        store_chunk(static_cast<T *>(e.out) + p * e.width, c, e.width, e.vec, sum);
    }
    if (e.dbias && threadIdx.x < rows && tile * P_ROWS + row0 + threadIdx.x < e.P) {
        double sum = 0.0;
        for (int w = w0; w <= w1; ++w) sum += e.share_bias[place(w) * P_ROWS + row0 + threadIdx.x];
        e.dbias[tile * P_ROWS + row0 + threadIdx.x] = (float)sum;
    }
}

// The classes' bias over log 2, padded to whole tiles (a finite bias stays finite: only -infinity closes a class; see entropy_finish).
__device__ __forceinline__ float padded_bias(const void *bias, int type, int c, int classes) {
    const float b = c < classes ? load_param(bias, type, c) : 0.f;
    return fabsf(b) < INFINITY ? fminf(fmaxf(b * LOG2E, -FLT_MAX), FLT_MAX) : b;
}
__global__ void __launch_bounds__(256) entropy_bias(const void *bias, int type, int classes, int padded, float *out) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < padded) out[c] = padded_bias(bias, type, c, classes);
}

// ---------------------------------------------------------------------------------------------- forward
// The statistics of rows over one piece of classes, added to those of the pieces before (first: there are none).
// WARPS warps to a row.
template <int WARPS>
__global__ void __launch_bounds__(256) entropy_rows(const float *__restrict__ logits, int ld, int64_t rows, int classes, int class0,
                                                    const void *__restrict__ bias, int bias_type, const int32_t *__restrict__ targets,
                                                    bool first, float2 *running, float *at_target, unsigned *ticket) {
    __shared__ Running part[8];
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;   // of entropy_finish
    const int lane = threadIdx.x % (32 * WARPS), warp = threadIdx.x >> 5;
    const int64_t row = (int64_t)blockIdx.x * (8 / WARPS) + warp / WARPS;
    Running r{-INFINITY, 0.f};
    if (row < rows) {
        const float *l = logits + row * ld;
        const int mine = targets[row] - class0;
        for (int c = lane * 4; c < classes; c += 32 * WARPS * 4) {
            float v[4];
            load_chunk(l, c, 1 << 30, true, 0.f, v);   // (rows are padded to whole chunks)
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (c + i < classes) {
                    if (bias) v[i] += load_param(bias, bias_type, class0 + c + i);
                    if (c + i == mine) at_target[row] = v[i];
                } else
                    v[i] = -INFINITY;
                top = fmaxf(top, v[i]);
            }
            const float m = fmaxf(r.m, top), shift = m == -INFINITY ? 0.f : m;
            r.s *= exp_fast(r.m - shift);
            r.m = m;
#pragma unroll
            for (int i = 0; i < 4; ++i) r.s += exp_fast(v[i] - shift);
        }
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        const Running other{__shfl_xor_sync(FULL, r.m, o), __shfl_xor_sync(FULL, r.s, o)};
        r = join(r, other);
    }
    if constexpr (WARPS > 1) {
        if ((threadIdx.x & 31) == 0) part[warp] = r;
        __syncthreads();
        if (lane == 0)
            for (int w = 1; w < WARPS; ++w) r = join(r, part[warp + w]);
    }
    if (lane == 0 && row < rows) {
        if (!first) r = join(Running{running[row].x, running[row].y}, r);
        running[row] = make_float2(r.m, r.s);
    }
}

// Where the statistics of a row are: one pair, or as many as the tile kernel's workers left.
struct Statistics {
    const float2 *all;
    int64_t M;
    bool tiled;      // [4 number + piece][M], over log 2
    Line line;
    int lists;       // not tiled: [lists][M]
    __device__ __forceinline__ Running of(int64_t row) const {
        if (!tiled) {
            Running r{all[row].x, all[row].y};
#pragma unroll 4
            for (int i = 1; i < lists; ++i) {
                const float2 v = all[(int64_t)i * M + row];
                r = join(r, Running{v.x, v.y});
            }
            return r;
        }
        const int64_t tile = row / TILE;
        const int n = 4 * (line.last_worker(tile) - line.first_worker(tile) + 1);
        float top = -FLT_MAX, sum = 0.f;
        for (int i = 0; i < n; i += 4) {
            float2 v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = all[(int64_t)(i + q) * M + row];
            const float now = fmaxf(max3(v[0].x, v[1].x, v[2].x), fmaxf(v[3].x, top));
            sum *= exp2_fast(top - now);
#pragma unroll
            for (int q = 0; q < 4; ++q) sum = fmaf(v[q].y, exp2_fast(v[q].x - now), sum);
            top = now;
        }
        return Running{sum == 0.f ? -INFINITY : top * LN2, sum};
    }
};

// lse and loss of each row from its statistics, and each block's sum of losses and count of rows that take part; the block
// that finishes last (the ticket tells) makes the mean of them.
constexpr int FINISH_ROWS = 256;   // a block's
struct Finish {
    double *sums;
    long long *counts;
    unsigned *ticket;
    float *loss;
    long long *counted;
};
__device__ __forceinline__ void sum_block(double &total, long long &live, double (&sum)[8], long long (&count)[8]) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        total += __shfl_xor_sync(FULL, total, o);
        live += __shfl_xor_sync(FULL, live, o);
    }
    if ((threadIdx.x & 31) == 0) {
        sum[threadIdx.x >> 5] = total;
        count[threadIdx.x >> 5] = live;
    }
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < 8; ++w) {
            total += sum[w];
            live += count[w];
        }
}
__global__ void __launch_bounds__(256) entropy_finish(const Statistics stats, const float *at_target, const int32_t *targets, int64_t rows,
                                                      int classes, const void *bias, int bias_type, float *lse, float *row_loss, const Finish f,
                                                      int *status) {
    __shared__ double sum[8];
    __shared__ long long count[8];
    __shared__ bool last;
    ep_wait_for_launch_before();
    double total = 0.0;
    long long live = 0;
    const int64_t row = (int64_t)blockIdx.x * FINISH_ROWS + threadIdx.x;
    if (row < rows) {
        float z = 0.f, loss = 0.f;
        if (target_of(targets, row, classes, status) >= 0) {
            const Running r = stats.of(row);
            z = r.m + logf(r.s);
            if (r.m == -INFINITY && r.s == 0.f)   // every class is closed: the row takes no part
                z = -INFINITY;
            else {
                float at = at_target[row] * (stats.tiled ? LN2 : 1.f);
                // (over log 2 a bias near fp32's lowest value was cut off at that value: beside other classes the logit is the bias)
                if (stats.tiled && bias && at_target[row] == -FLT_MAX && z > at) at = load_param(bias, bias_type, targets[row]);
                loss = z - at;
                live = 1;
            }
        }
        lse[row] = z;
        row_loss[row] = loss;
        total = (double)loss;
    }
    sum_block(total, live, sum, count);
    if (threadIdx.x == 0) {
        f.sums[blockIdx.x] = total;
        f.counts[blockIdx.x] = live;
        __threadfence();
        last = atomicAdd(f.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    total = 0.0;
    live = 0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 256) {
        total += __ldcg(f.sums + i);
        live += __ldcg(f.counts + i);
    }
    sum_block(total, live, sum, count);
    if (threadIdx.x == 0) {
        *f.loss = (float)(total / (double)(live > 0 ? live : 1));
        *f.counted = live;
    }
}

// ---------------------------------------------------------------------------------------------- backward
// What is known of each row, and each block's largest finite |g|, in what G is measured in.  A row that takes no part counts for nothing, whatever x holds
// there; but 0 times an infinity or a NaN is NaN, so such rows of x are looked through: a block's `unclean` is 1 where one
// holds any (or numbers so large that a logit might overflow), and the products then read a copy of x with zeros there.
constexpr int WEIGHT_THREADS = 512;
// How G of 16 bits is measured: in |g| of all rows, or, with weights of their own, by a power of two; `log2_unit`: what 1 becomes.
struct Measure {
    const float *dloss;
    const long long *counted;
    bool mean;        // no row has a weight of its own
    bool scaled;      // by a power of two, where not by |g|
    int log2_unit;
};
__device__ __forceinline__ double mean_weight(const Measure &m) {
    return m.dloss ? (double)*m.dloss / (double)(*m.counted > 0 ? *m.counted : 1) : 0.0;
}
// |g| of all rows, or 0 (which leaves what is measured in it and its inverse far from the ends of fp32).
__device__ __forceinline__ float common_weight(const Measure &m, double mean) {
    const float g = fabsf((float)mean);
    return m.mean && g >= 7.9e-31f && g <= 1.2e30f ? g : 0.f;
}
__device__ __forceinline__ Scale scale_of(float common, float top, const Measure &m, int unclean) {
    if (common > 0.f) return Scale{1.f, scalbnf(common, -m.log2_unit), unclean};
    const int up = m.scaled && top > 0.f ? min(14 - ilogbf(top), 126) : 0;
    return Scale{scalbnf(1.f, up), scalbnf(1.f, -up), unclean};
}
template <typename T>
__global__ void __launch_bounds__(WEIGHT_THREADS) entropy_weights(const float *__restrict__ lse, const int32_t *__restrict__ targets, int64_t rows,
                                                                  int classes, const Measure measure, const float *__restrict__ drow,
                                                                  const void *__restrict__ x, int64_t ldx, int n_in,
                                                                  const void *__restrict__ bias, int bias_type, float *padded, RowInfo info,
                                                                  float *peaks, int *unclean, Scale *scale, int *status) {
    __shared__ int bad_rows;
    __shared__ float tops[WEIGHT_THREADS / 32];
    const double mean = mean_weight(measure);   // (it and a row's own may cancel)
    const float common = common_weight(measure, mean), unit = scalbnf(1.f, measure.log2_unit);
    const int lane = threadIdx.x & 31;
    if (bias)   // (on the way: the bias as the tile kernels read it)
        for (int c = blockIdx.x * WEIGHT_THREADS + threadIdx.x; c < (classes + TILE - 1) / TILE * TILE; c += gridDim.x * WEIGHT_THREADS)
            padded[c] = padded_bias(bias, bias_type, c, classes);
    if (threadIdx.x == 0) bad_rows = 0;
    __syncthreads();
    float top = 0.f;
    for (int64_t row0 = (int64_t)blockIdx.x * WEIGHT_THREADS; row0 < rows; row0 += (int64_t)gridDim.x * WEIGHT_THREADS) {
        const int64_t row = row0 + threadIdx.x;
        bool dead = false;
        if (row < rows) {
            dead = target_of(targets, row, classes, status) < 0 || lse[row] == -INFINITY;
            const float g = dead ? 0.f : common > 0.f ? copysignf(unit, (float)mean) : (float)(mean + (drow ? (double)drow[row] : 0.0));
            const float z = lse[row];
            // (rounded once: a g that all rows share would else be off by the same in all of them, and their sums with it)
            info.shift[row] = dead ? -INFINITY : (float)(log2((double)fabsf(g)) - (double)z * 1.44269504088896340736);
            info.g[row] = z != z ? z : g;
            info.target[row] = dead ? -1 : targets[row];
            if (fabsf(g) < INFINITY) top = fmaxf(top, fabsf(g));
        }
        else if (row < (rows + TILE - 1) / TILE * TILE) {
            info.shift[row] = -INFINITY;
            info.g[row] = 0.f;
            info.target[row] = -1;
        }
        if (!x) continue;
        // four rows at a time, 8 lanes to each
        for (unsigned left = __ballot_sync(FULL, dead); left;) {
            unsigned mine = left;
            for (int i = 0; i < (lane >> 3); ++i) mine &= mine - 1;
            if (mine) {
                const T *from = static_cast<const T *>(x) + (row0 + (threadIdx.x & ~31) + __ffs(mine) - 1) * ldx;
                bool bad = false;
#pragma unroll 8
                for (int c = lane & 7; c < n_in; c += 8) bad |= !(fabsf(to_f32(from[c])) < 1e18f);
                if (bad) bad_rows = 1;
            }
            for (int i = 0; i < 4; ++i) left &= left - 1;
        }
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
    if (lane == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < WEIGHT_THREADS / 32; ++w) top = fmaxf(top, tops[w]);
        if (gridDim.x == 1)   // nobody to wait for
            *scale = scale_of(common, top, measure, bad_rows);
        else {
            peaks[blockIdx.x] = top;
            unclean[blockIdx.x] = bad_rows;
        }
    }
}

__global__ void __launch_bounds__(256) entropy_scale(const float *peaks, const int *unclean, int n, const Measure measure, Scale *out) {
    __shared__ float tops[8];
    float top = 0.f;
    bool bad = false;
    ep_wait_for_launch_before();
    for (int i = threadIdx.x; i < n; i += 256) {
        top = fmaxf(top, peaks[i]);
        bad |= unclean[i] != 0;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) top = fmaxf(top, tops[w]);
        *out = scale_of(common_weight(measure, mean_weight(measure)), top, measure, any);
    }
}

// x with zeros in the rows that take no part (see entropy_weights).  from: x, copied only if a row needs it; NULL: `to` is a
// copy of x already, of `parts` matrices.
template <typename E>
__global__ void __launch_bounds__(256) entropy_clean(const E *from, int64_t ld, int64_t rows, int cols, const RowInfo info, const Scale *scale,
                                                     E *to, int ld_to, int parts, int64_t part_stride) {
    ep_wait_for_launch_before();
    if (!scale->unclean) return;
    const int lane = threadIdx.x & 31;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows; row += (int64_t)gridDim.x * 8) {
        const bool dead = info.target[row] < 0;
        if (from)
            for (int c = lane; c < cols; c += 32) to[row * ld_to + c] = dead ? E{} : from[row * ld + c];
        else if (dead)
            for (int p = 0; p < parts; ++p)
                for (int c = lane; c < cols; c += 32) to[p * part_stride + row * ld_to + c] = E{};
    }
}

// G of one piece from its logits, in the operands' type (fp32 as three bf16 parts; zero past the classes), and the sums of its
// columns over the block's rows: part[blockIdx.y][stride].
constexpr int G_CHUNKS = 16, G_ROWS = 16;   // a block covers 128 classes, 16 rows at a time
template <typename T>
__global__ void __launch_bounds__(256) entropy_slopes(const float *__restrict__ logits, int ld, int64_t rows, int classes, int class0,
                                                      const void *__restrict__ bias, int bias_type,
                                                      const float *__restrict__ lse, const RowInfo info,
                                                      const Scale *__restrict__ scale, void *to_raw, int64_t part_stride, float *part,
                                                      int64_t stride) {
    constexpr bool SPLIT = sizeof(T) == 4;
    __shared__ float fold[G_ROWS][G_CHUNKS * 8];
    const int cx = threadIdx.x % G_CHUNKS, r0 = threadIdx.x / G_CHUNKS;
    const int col = (blockIdx.x * G_CHUNKS + cx) * 8;
    const float up = scale->up;
    float b[8], sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        b[i] = bias && col + i < classes ? load_param(bias, bias_type, class0 + col + i) : 0.f;
        sum[i] = 0.f;
    }
    if (col < ld)
        for (int64_t row = (int64_t)blockIdx.y * G_ROWS + r0; row < rows; row += (int64_t)gridDim.y * G_ROWS) {
            float v[8];
            load_chunk(logits + row * ld, col, 1 << 30, true, 0.f, v);
            const float g = info.g[row], z = lse[row];
            const int target = info.target[row];
            const bool live = target >= 0;
            const int mine = live ? target - class0 : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = exp_fast(v[i] + b[i] - z) - (col + i == mine ? 1.f : 0.f);
                v[i] = live && col + i < classes ? p * g : 0.f;
                sum[i] += v[i];
                v[i] *= up;
            }
            if (!to_raw) continue;
            if constexpr (SPLIT) {
                __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(to_raw) + row * ld + col;
                __nv_bfloat16 p[8][3];
#pragma unroll
                for (int q = 0; q < 8; ++q) split3(v[q], p[q]);
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    alignas(16) __nv_bfloat16 o[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) o[q] = p[q][k];
                    *reinterpret_cast<uint4 *>(to + k * part_stride) = *reinterpret_cast<const uint4 *>(o);
                }
            } else
                store_chunk(static_cast<T *>(to_raw) + row * ld, col, ld, true, v);
        }
    if (!part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) fold[r0][cx * 8 + i] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < G_CHUNKS * 8; c += 256) {
        const int to = blockIdx.x * G_CHUNKS * 8 + c;
        if (to >= classes) continue;
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < G_ROWS; ++q) t += fold[q][c];
        part[(size_t)blockIdx.y * stride + to] = t;
    }
}

// Sums over all pieces, rounded once.
template <typename T>
__global__ void __launch_bounds__(256) entropy_round(const float *__restrict__ sums, int64_t n, const Scale *__restrict__ scale, T *out) {
    const float down = scale->down;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (i + q < n) out[i + q] = from_f32<T>(sums[i + q] * down);
    }
}

// ---------------------------------------------------------------------------------------------- small problems
//
// A few products cost the tile kernels mostly launches and passes (fp32 operands split in three, logits written and read back,
// statistics or G, joins: ten launches of a backward).  Then fp32 multiply-adds of tiles of 64 x 64 take the operands as they are: the
// forward is two launches, the backward two to four.  Bound by latency, then by what the shared memory gives the multiply-adds: a thread
// has 4 x 4 logits (8 16-byte reads to 64 multiply-adds) or 4 rows of n_in / 16 columns of the second product.
// fp32, tiles -> here, us.  Forward: 128 x 64 -> 32 12.2 -> 8.5, 500 x 64 -> 500 13.2 -> 9.8, 3000 x 65 -> 257 16.2 -> 13.0, 50000 x 16 -> 40
// 30 -> 16, 200000 x 16 -> 10 109 -> 45; but 2000 x 128 -> 257 14.8 -> 18.0, 40 x 128 -> 4000 16 -> 27 (statistics of many classes).  Backward:
// 128 x 64 -> 32 24.8 -> 11.5, 500 x 64 -> 500 34.9 -> 14.1, 40 x 128 -> 4000 31.8 -> 18.4, 3000 x 65 -> 257 41.6 -> 32.7, 18 x 42 -> 77887
// 123 -> 77; but 2000 x 128 -> 257 37.8 -> 45.7, 64 x 128 -> 16384 45 -> 57, 2000 x 64 -> 1000 44 -> 56.
// In 16 bits, where nothing is split, the tiles' forward is as quick or quicker everywhere.  Backward, bf16: 128 x 64 -> 32 15.8 -> 11.5,
// 16 x 100 -> 456 35.5 -> 15.1, 500 x 64 -> 500 23.3 -> 14.3, 3000 x 65 -> 257 46 -> 32, 1000 x 64 -> 1000 31.8 -> 29.1; but 2000 x 64 -> 1000 33,
// fp32 here 56.  G stays fp32 here, in all types.
constexpr int ST = 64;            // a block's rows of either operand
constexpr int SMALL_BLOCKS = 1;   // to an SM, of either gradient's
constexpr int SMALL_WIDTH = 128;  // elements of a row at most
// 64 rows on their way to shared memory, LD floats apart, zero past their n_in elements and past the last row.
// (Asynchronously of fp32; 16-bit elements become fp32 on the way.)
template <int LD, typename T, typename Wanted>
__device__ __forceinline__ void small_rows(float *to, const T *from, int64_t ld, int64_t row0, int64_t rows, int n_in, Wanted wanted) {
    const int lane = threadIdx.x & 31;
    if constexpr (sizeof(T) == 2) {
        constexpr int COLUMNS = (LD - 4 + 31) / 32;
#pragma unroll
        for (int q0 = 0; q0 < ST / 8; q0 += 4) {
            T v[4][COLUMNS];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t row = row0 + (threadIdx.x >> 5) + 8 * (q0 + q);
                const bool there = row < rows && wanted(row);
#pragma unroll
                for (int i = 0; i < COLUMNS; ++i) v[q][i] = there && 32 * i + lane < n_in ? from[row * ld + 32 * i + lane] : from_f32<T>(0.f);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < COLUMNS; ++i)
                    if (32 * i + lane < LD - 4) to[((threadIdx.x >> 5) + 8 * (q0 + q)) * LD + 32 * i + lane] = to_f32(v[q][i]);
        }
    } else {
#pragma unroll
        for (int q = 0; q < ST / 8; ++q) {
            const int r = (threadIdx.x >> 5) + 8 * q;
            const bool there = row0 + r < rows && wanted(row0 + r);
#pragma unroll
            for (int c0 = 0; c0 < LD - 4; c0 += 32) {
                const int c = c0 + lane;
                if (c < LD - 4) {
                    const bool in = there && c < n_in;
                    const float *src = in ? from + (row0 + r) * ld + c : from;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(to + r * LD + c)), "l"(src), "r"(in ? 4 : 0) : "memory");
                }
            }
        }
    }
}
// s[i][j] = p_(4 ty + i) . q_(tx + 16 j); rows LD floats apart, which keeps the lanes of a 16-byte access in different banks.
template <int LD>
__device__ __forceinline__ void small_products(const float *p, const float *q, int n_in, int tx, int ty, float (&s)[4][4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 2
    for (int k = 0; k < n_in; k += 4) {
        float4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = *reinterpret_cast<const float4 *>(p + (4 * ty + i) * LD + k);
            b[i] = *reinterpret_cast<const float4 *>(q + (tx + 16 * i) * LD + k);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = fmaf(a[i].x, b[j].x, s[i][j]);
                s[i][j] = fmaf(a[i].y, b[j].y, s[i][j]);
                s[i][j] = fmaf(a[i].z, b[j].z, s[i][j]);
                s[i][j] = fmaf(a[i].w, b[j].w, s[i][j]);
            }
    }
}

struct SmallWork {
    const void *x;
    int64_t ldx;
    const void *w;
    int64_t ldw;
    const void *bias;
    int bias_type;
    const int32_t *targets;
    int64_t rows;
    int n_in, classes, class_tiles;
    float2 *stats;            // forward: [class tile][rows]
    float *at_target;
    unsigned *ticket;
    const float *lse;         // backward
    RowInfo info;
    int dx_splits, dw_splits; // shares of the sums over classes and over rows
    int64_t dx_blocks;
    float *dx_part, *dw_part, *db_part;   // [share][..], or the outputs themselves are written
    void *dx, *dweight;
    float *dbias;
};
// What the tile kernels make of an infinity among fp32 operands, which split into NaN: an infinite logit is no logit.
template <typename T>
__device__ __forceinline__ float small_logit(float v) { return sizeof(T) == 4 && isinf(v) ? CUDART_NAN_F : v; }
// Statistics of a tile's rows.  J = ceil(n_in / 16).
template <int J>
__global__ void __launch_bounds__(256) entropy_small_forward(const SmallWork e) {
    constexpr int LD = 16 * J + 4;
    extern __shared__ float4 small_memory[];
    float *const p = reinterpret_cast<float *>(small_memory), *const q = p + ST * LD;
    const int64_t row0 = (int64_t)blockIdx.y * ST;
    const int class0 = blockIdx.x * ST, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    auto all = [](int64_t) { return true; };
    ep_wait_for_launch_before();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *e.ticket = 0;
    small_rows<LD>(p, static_cast<const float *>(e.x), e.ldx, row0, e.rows, e.n_in, all);
    small_rows<LD>(q, static_cast<const float *>(e.w), e.ldw, class0, e.classes, e.n_in, all);
    copies_end_group();
    float bias[4];
    int target[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = class0 + tx + 16 * j;
        bias[j] = e.bias && c < e.classes ? load_param(e.bias, e.bias_type, c) : 0.f;
        target[j] = row0 + 4 * ty + j < e.rows ? e.targets[row0 + 4 * ty + j] : -1;
    }
    copies_wait<0>();
    __syncthreads();
    float s[4][4];
    small_products<LD>(p, q, e.n_in, tx, ty, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + 4 * ty + i;
        Running r{-INFINITY, 0.f};
        float l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = class0 + tx + 16 * j;
            l[j] = c < e.classes ? small_logit<float>(s[i][j]) + bias[j] : -INFINITY;
            if (c == target[i] && c < e.classes) e.at_target[row] = l[j];
            r.m = fmaxf(r.m, l[j]);
        }
        const float shift = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
        for (int j = 0; j < 4; ++j) r.s += exp_fast(l[j] - shift);
#pragma unroll
        for (int o = 8; o >= 1; o >>= 1) r = join(r, Running{__shfl_xor_sync(FULL, r.m, o), __shfl_xor_sync(FULL, r.s, o)});
        if (tx == 0 && row < e.rows) e.stats[(int64_t)blockIdx.x * e.rows + row] = make_float2(r.m, r.s);
    }
}
// Gradient of 64 rows of x (P = x, Q = W), or of W (P = W, Q = x): over its share of Q, 64 rows at a time, the logits, G of them, G Q.
// (Either makes all logits: it needs a third more multiply-adds than G written and read back, and two launches less.)
template <typename T, bool DW, int J>
__device__ __forceinline__ void small_gradient(const SmallWork &e, int64_t block, float *memory) {
    constexpr int LD = 16 * J + 4, LDG = ST + 4;
    float *const p = memory, *const q = p + ST * LD, *const g = q + 2 * ST * LD;   // q: two tiles; g[row of Q][row of P]
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int splits = DW ? e.dw_splits : e.dx_splits, share = (int)(block % splits);
    const int64_t P = DW ? e.classes : e.rows, Q = DW ? e.rows : e.classes, p0 = block / splits * ST, tiles = (Q + ST - 1) / ST;
    const int64_t t0 = tiles * share / splits, t1 = tiles * (share + 1) / splits;
    auto bring = [&](int64_t tile) {
        // (a row that takes no part counts for nothing, whatever it holds)
        small_rows<LD>(q + (tile & 1) * ST * LD, static_cast<const T *>(DW ? e.x : e.w), DW ? e.ldx : e.ldw, tile * ST, Q, e.n_in,
                       [&](int64_t r) { return !DW || e.info.target[r] >= 0; });
    };
    small_rows<LD>(p, static_cast<const T *>(DW ? e.w : e.x), DW ? e.ldw : e.ldx, p0, P, e.n_in, [](int64_t) { return true; });
    if (t0 < t1) bring(t0);
    copies_end_group();
    // what is known of rows of x (target, g, lse) and of classes (bias), of either operand
    struct Known {
        int target[4];
        float g[4], z[4], bias[4];
    };
    auto known = [&](bool rows, int64_t first, int step, Known &k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t at = first + i * step;
            if (rows) {
                k.target[i] = at < e.rows ? e.info.target[at] : -1;
                k.g[i] = k.target[i] >= 0 ? e.info.g[at] : 0.f;
                k.z[i] = k.target[i] >= 0 ? e.lse[at] : 0.f;
            } else
                k.bias[i] = e.bias && at < e.classes ? load_param(e.bias, e.bias_type, at) : 0.f;
        }
    };
    Known k;
    known(!DW, p0 + 4 * ty, 1, k);
    float total[4][J];
    double column[4] = {};   // of dbias
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) total[i][j] = 0.f;
    for (int64_t tile = t0; tile < t1; ++tile) {
        const int64_t q0 = tile * ST;
        const float *const mine = q + (tile & 1) * ST * LD;
        known(DW, q0 + tx, 16, k);
        copies_wait<0>();
        __syncthreads();
        if (tile + 1 < t1) {
            bring(tile + 1);
            copies_end_group();
        }
        float s[4][4];
        small_products<LD>(p, mine, e.n_in, tx, ty, s);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = DW ? j : i, c = DW ? i : j;
                const int64_t one_class = DW ? p0 + 4 * ty + i : q0 + tx + 16 * j;
                const float share_of_class = exp_fast(small_logit<T>(s[i][j]) + k.bias[c] - k.z[r]) - (one_class == k.target[r] ? 1.f : 0.f);
                s[i][j] = k.target[r] >= 0 && one_class < e.classes ? share_of_class * k.g[r] : 0.f;
            }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *reinterpret_cast<float4 *>(g + (tx + 16 * j) * LDG + 4 * ty) = make_float4(s[0][j], s[1][j], s[2][j], s[3][j]);
        if (DW)
#pragma unroll
            for (int i = 0; i < 4; ++i) column[i] += (double)((s[i][0] + s[i][1]) + (s[i][2] + s[i][3]));
        __syncthreads();
        float acc[4][J];   // of this tile: a long sum of fp32 would lose bits
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) acc[i][j] = 0.f;
#pragma unroll 4
        for (int r = 0; r < ST; ++r) {
            const float4 a = *reinterpret_cast<const float4 *>(g + r * LDG + 4 * ty);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const float b = mine[r * LD + tx + 16 * j];
                acc[0][j] = fmaf(a.x, b, acc[0][j]);
                acc[1][j] = fmaf(a.y, b, acc[1][j]);
                acc[2][j] = fmaf(a.z, b, acc[2][j]);
                acc[3][j] = fmaf(a.w, b, acc[3][j]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) total[i][j] += acc[i][j];
    }
    copies_wait<0>();
    float *const part = DW ? e.dw_part : e.dx_part;
    T *const out = static_cast<T *>(DW ? e.dweight : e.dx);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = p0 + 4 * ty + i;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int n = tx + 16 * j;
            if (m >= P || n >= e.n_in) continue;
            if (splits > 1)
                part[((int64_t)share * P + m) * e.n_in + n] = total[i][j];
            else if (out)
                out[m * e.n_in + n] = from_f32<T>(total[i][j]);
        }
        if (DW && e.dbias) {
#pragma unroll
            for (int o = 8; o >= 1; o >>= 1) column[i] += __shfl_xor_sync(FULL, column[i], o);
            if (tx == 0 && m < P) {
                if (splits > 1)
                    e.db_part[(int64_t)share * P + m] = (float)column[i];
                else
                    e.dbias[m] = (float)column[i];
            }
        }
    }
}
template <typename T, int J>
__global__ void __launch_bounds__(256, 2) entropy_small_backward(const SmallWork e) {
    extern __shared__ float4 small_memory[];
    float *const memory = reinterpret_cast<float *>(small_memory);
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    if ((int64_t)blockIdx.x < e.dx_blocks)
        small_gradient<T, false, J>(e, blockIdx.x, memory);
    else
        small_gradient<T, true, J>(e, blockIdx.x - e.dx_blocks, memory);
}
// The shares: LANES lanes to an element, each every LANES-th share in order, then the lanes (in a fixed order).
template <typename T, int LANES>
__global__ void __launch_bounds__(256) entropy_small_fold(const float *part, int splits, int64_t n, T *out, const float *more_part,
                                                          int64_t more, float *more_out) {
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
    if (at >= n + more) return;   // (a warp's lanes leave together: LANES is 1 or 32)
    const bool rest = at >= n;
    const int64_t i = rest ? at - n : at, all = rest ? more : n;
    const float *from = rest ? more_part : part;
    double sum = 0.0;
#pragma unroll 8
    for (int s = threadIdx.x % LANES; s < splits; s += LANES) sum += (double)from[(int64_t)s * all + i];
    if constexpr (LANES > 1) {
#pragma unroll
        for (int o = LANES / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
        if (threadIdx.x % LANES) return;
    }
    if (rest)
        more_out[i] = (float)sum;
    else if (out)
        out[i] = from_f32<T>((float)sum);
}

// ---------------------------------------------------------------------------------------------- host side
constexpr int MAX_WIDTH = 65536, MAX_CLASSES = 1 << 24;
// Elements of a piece: of fp32 logits, of which G is made beside them; of G alone.
constexpr int64_t LOGITS_PIECE = 1 << 24, SLOPES_PIECE = 1 << 25;

// Rows x classes in pieces; of the shorter side as much as goes, so that little of what is summed over pieces is large.
struct Pieces {
    int64_t rows;
    int classes;
    int64_t across;   // pieces along the rows
    int down;         // and along the classes
};
Pieces make_pieces(int64_t rows, int classes, int64_t piece) {
    Pieces p;
    auto up = [](int64_t v) { return std::max<int64_t>(1, (v + 255) / 256) * 256; };
    if (rows >= classes) {
        p.classes = std::min(classes, 16384);
        p.rows = std::min(rows, std::max<int64_t>(256, piece / up(p.classes) / 256 * 256));
    } else {
        p.rows = std::min<int64_t>(rows, 16384);
        p.classes = (int)std::min<int64_t>(classes, std::max<int64_t>(256, piece / up(p.rows) / 256 * 256));
    }
    p.across = rows ? ep::ceil_div(rows, p.rows) : 0;
    p.down = (int)ep::ceil_div(classes, p.classes);
    return p;
}
int padded(int classes) { return (classes + 7) & ~7; }

// The most that f(rows, classes) takes for any piece.
template <typename F>
size_t most_of(const Pieces &p, int64_t rows, int classes, F f) {
    size_t most = 0;
    for (int64_t r : {p.rows, rows - (p.across - 1) * p.rows})
        for (int c : {p.classes, classes - (p.down - 1) * p.classes}) most = std::max<size_t>(most, f(r, c));
    return most;
}

bool entropy_shape_ok(int64_t rows, int n_in, int classes) {
    return rows >= 0 && rows <= (1ll << 31) - 256 && n_in >= 1 && n_in <= MAX_WIDTH && classes >= 1 && classes <= MAX_CLASSES;
}

Line line_of(const ep_ctx *ctx, int64_t outer, int64_t inner) {
    Line l;
    l.tiles = outer * inner;
    l.inner = (int)inner;
    l.workers = (int)std::min<int64_t>(l.tiles, ctx->sm_count / 2);
    return l;
}
// The most workers that share a tile of the outer kind.
int64_t most_workers(const Line &l) {
    return std::min<int64_t>(l.workers, ep::ceil_div(l.inner, std::max<int64_t>(1, l.tiles / l.workers)) + 1);
}

struct Inputs {
    const void *x;
    int64_t ldx;
    const void *w;
    int64_t ldw;
    int type;
    const void *bias;
    int bias_type;
    const int32_t *targets;
    int64_t rows;
    int n_in, classes;
    bool aligned;
    cudaStream_t stream;
    int kernels;
};

// Blocks of entropy_weights: one alone, for few rows, needs no other launch to join what it found.
int weight_blocks(const ep_ctx *ctx, int64_t rows) {
    return rows <= 2 * WEIGHT_THREADS ? 1 : (int)std::min<int64_t>(ep::ceil_div(rows, WEIGHT_THREADS), ctx->sm_count);
}

// Copies of the operands, and the bias as the tile kernel reads it.
struct Copies {
    void *x, *w;
    float *bias;
};
Copies copies_space(ep::Arena &a, int64_t rows, int n_in, int classes, int type, bool aligned, bool x_always) {
    Copies c{};
    const bool copy = type == EP_F32 || !aligned;
    if (copy || x_always) c.x = a.take<char>(ep::packed_form(rows, n_in, type).bytes);
    if (copy) c.w = a.take<char>(ep::packed_form(classes, n_in, type).bytes);
    if (type != EP_F32) c.bias = a.take<float>(ep::ceil_div(classes, TILE) * TILE);
    return c;
}

// `rows` of an operand from row `first` on.
Operand rows_of(Operand o, int64_t first, int64_t rows) {
    o.base = static_cast<const char *>(o.base) + first * o.ld * ep::type_size(o.type);
    o.rows = rows;
    return o;
}

int operands(ep_ctx *ctx, Inputs &in, const Copies &c, bool with_bias, Operand *x, Operand *w) {
    if (with_bias && c.bias && in.bias) {
        const int n = (int)ep::ceil_div(in.classes, TILE) * TILE;
        entropy_bias<<<n / 256, 256, 0, in.stream>>>(in.bias, in.bias_type, in.classes, n, c.bias);
        EP_CUDA(ctx, cudaGetLastError());
        ++in.kernels;
    }
    *x = Operand{in.x, in.type, in.rows, in.n_in, in.ldx, 1, 0};
    *w = Operand{in.w, in.type, in.classes, in.n_in, in.ldw, 1, 0};
    if (in.type != EP_F32 && in.aligned) return EP_OK;
    return ep::make_operands(ctx, Matrix{in.x, in.ldx, in.rows, in.n_in, c.x}, Matrix{in.w, in.ldw, in.classes, in.n_in, c.w}, in.type,
                             in.stream, x, w, &in.kernels);
}

int logits_of(ep_ctx *ctx, Inputs &in, const Operand &x, const Operand &w, int64_t row0, int64_t rows, int class0, int classes,
              float *logits, float *share) {
    return ep::product(ctx, rows_of(x, row0, rows), false, rows_of(w, class0, classes), false, rows, padded(classes), in.n_in, logits,
                       EP_F32, false, nullptr, share, in.stream, &in.kernels);
}

template <bool GRAD, bool BIASED, bool RUNS, typename T>
int launch_tiles_of(ep_ctx *ctx, const CUtensorMap &x, const CUtensorMap &w, const CUtensorMap &g, const CUtensorMap &clean,
                    const TileWork &e, cudaStream_t stream) {
    auto kernel = entropy_tiles<GRAD, BIASED, RUNS, T>;
    constexpr size_t smem = TileMemory<GRAD>::TOTAL;
    EP_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(2 * e.line.workers));
    cfg.blockDim = dim3(TILE_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2] = {};
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = 2;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = 2;
    EP_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, x, w, g, clean, e, ctx->d_status));
    return EP_OK;
}
// g: of the backward, [rows][ld].
template <bool GRAD>
int launch_tiles(ep_ctx *ctx, const Operand &x, const Operand &w, void *g, int64_t ld, const Operand &clean, TileWork &e,
                 cudaStream_t stream, int *kernels) {
    const uint32_t fmt = x.type == EP_BF16 ? 1u : 0u;
    e.idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(TILE >> 4) << 24);
    e.kb = (int)ep::ceil_div(x.cols, 64);
    e.log2e = sums_log2e((int)x.cols, x.type);
    CUtensorMap mx{}, mw{}, mg{}, mc{};
    if (!encode_operand(&mx, x, false, BLOCK_ROWS) || !encode_operand(&mw, w, false, BLOCK_ROWS) ||
        (GRAD && !(encode_result(&mg, g, x.type, 1, e.M, e.N, ld, TILE) && encode_operand(&mc, clean, false, BLOCK_ROWS))))
        return ep::fail(ctx, EP_ERR_CUDA, "cuTensorMapEncodeTiled failed for %lld rows of %d classes", (long long)e.M, e.N);
    ++*kernels;
    auto launch = [&](auto biased, auto runs, auto type) {
        return launch_tiles_of<GRAD, decltype(biased)::value, decltype(runs)::value, decltype(type)>(ctx, mx, mw, mg, mc, e, stream);
    };
    auto of_type = [&](auto biased, auto runs) {
        return x.type == EP_BF16 ? launch(biased, runs, __nv_bfloat16{}) : launch(biased, runs, __half{});
    };
    const std::true_type yes;
    const std::false_type no;
    if constexpr (GRAD)
        return of_type(no, yes);
    else if (x.cols > ONE_RUN)
        return e.bias ? of_type(yes, yes) : of_type(no, yes);
    else
        return e.bias ? of_type(yes, no) : of_type(no, no);
}

struct ForwardSpace {
    Copies copies;
    float *logits, *share, *at_target;
    float2 *stats;
    Finish finish;
    Pieces pieces;   // of fp32
    Line line;       // of 16 bits
    size_t bytes;
};
ForwardSpace forward_space(const ep_ctx *ctx, int64_t rows, int n_in, int classes, int type, bool aligned, void *base) {
    ep::Arena a(base);
    ForwardSpace s{};
    s.copies = copies_space(a, rows, n_in, classes, type, aligned, false);
    if (rows && type == EP_F32) {
        s.pieces = make_pieces(rows, classes, LOGITS_PIECE);
        s.logits = a.take<float>(s.pieces.rows * padded(s.pieces.classes));
        s.share = a.take<float>(most_of(s.pieces, rows, classes, [&](int64_t r, int c) { return ep::product_bytes(ctx, r, padded(c), n_in, type, EP_F32); }) / 4);
        s.stats = a.take<float2>(rows);
    } else if (rows) {
        s.line = line_of(ctx, ep::ceil_div(rows, TILE), ep::ceil_div(classes, TILE));
        s.stats = a.take<float2>((size_t)most_workers(s.line) * 4 * rows);
    }
    s.at_target = a.take<float>(rows);
    s.finish.sums = a.take<double>(ep::ceil_div(rows, FINISH_ROWS));
    s.finish.counts = a.take<long long>(ep::ceil_div(rows, FINISH_ROWS));
    s.finish.ticket = a.take<unsigned>(1);
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
}

int forward_run(ep_ctx *ctx, Inputs &in, const ForwardSpace &s, float *loss, float *row_loss, float *lse, long long *counted) {
    Operand x, w;
    int rc = operands(ctx, in, s.copies, true, &x, &w);
    if (rc != EP_OK) return rc;
    Statistics stats{s.stats, in.rows, in.type != EP_F32, s.line, 1};
    if (stats.tiled) {
        TileWork e{};
        e.M = in.rows;
        e.N = in.classes;
        e.line = s.line;
        e.bias = in.bias ? s.copies.bias : nullptr;
        e.targets = in.targets;
        e.partial = s.stats;
        e.at_target = s.at_target;
        e.ticket = s.finish.ticket;
        rc = launch_tiles<false>(ctx, x, w, nullptr, 0, x, e, in.stream, &in.kernels);
        if (rc != EP_OK) return rc;
    }
    const Pieces &p = s.pieces;
    for (int64_t row0 = 0; !stats.tiled && row0 < in.rows; row0 += p.rows)
        for (int class0 = 0; class0 < in.classes; class0 += p.classes) {
            const int64_t rows = std::min(p.rows, in.rows - row0);
            const int classes = std::min(p.classes, in.classes - class0);
            rc = logits_of(ctx, in, x, w, row0, rows, class0, classes, s.logits, s.share);
            if (rc != EP_OK) return rc;
            const bool wide = classes > 2048 || rows < 8 * ctx->sm_count;
            auto kernel = wide ? entropy_rows<8> : entropy_rows<1>;
            kernel<<<(unsigned)ep::ceil_div(rows, wide ? 1 : 8), 256, 0, in.stream>>>(
                s.logits, padded(classes), rows, classes, class0, in.bias, in.bias_type, in.targets + row0, class0 == 0,
                s.stats + row0, s.at_target + row0, s.finish.ticket);
            EP_CUDA(ctx, cudaGetLastError());
            ++in.kernels;
        }
    Finish f = s.finish;
    f.loss = loss;
    f.counted = counted;
    EP_CUDA(ctx, ep::launch_early(entropy_finish, dim3((unsigned)ep::ceil_div(in.rows, FINISH_ROWS)), dim3(256), 0, in.stream, stats, s.at_target,
                                  in.targets, in.rows, in.classes, in.bias, in.bias_type, lse, row_loss, f, ctx->d_status));
    ++in.kernels;
    return EP_OK;
}

// The columns' sums of this many pieces of rows are kept before they are joined to one: 2^20 rows of 2^17 classes would need 6 GB.
constexpr int JOINED_PIECES = 16;
struct Backward {
    Copies copies;
    void *g;
    float *logits, *share, *dx, *dweight, *part, *peaks;
    RowInfo rows;
    int *unclean;
    Scale *scale;
    Pieces pieces;
    int blocks;           // of entropy_weights
    int64_t slabs;        // partial sums of a piece's columns
    int64_t kept;         // and how many of all pieces are kept before they are joined
    size_t bytes;
};
Backward backward_space(const ep_ctx *ctx, int64_t rows, int n_in, int classes, int type, bool aligned, void *base) {
    ep::Arena a(base);
    Backward s{};
    const bool f32 = type == EP_F32;
    s.copies = copies_space(a, rows, n_in, classes, type, aligned, true);   // (x: see entropy_clean)
    if (rows) {
        s.pieces = make_pieces(rows, classes, f32 ? LOGITS_PIECE : SLOPES_PIECE);
        const Pieces &p = s.pieces;
        s.g = a.take<char>(ep::packed_form(p.rows, p.classes, type).bytes);
        if (f32) s.logits = a.take<float>(p.rows * padded(p.classes));
        s.share = a.take<float>(most_of(p, rows, classes, [&](int64_t r, int c) {
                                    size_t most = f32 ? ep::product_bytes(ctx, r, padded(c), n_in, type, EP_F32) : 0;
                                    for (int out : {type, (int)EP_F32}) {
                                        most = std::max(most, ep::product_bytes(ctx, r, n_in, c, type, out));
                                        most = std::max(most, ep::product_bytes(ctx, c, n_in, r, type, out));
                                    }
                                    return most;
                                }) / 4);
        if (!f32 && p.down > 1) s.dx = a.take<float>(p.rows * n_in);
        if (!f32 && p.across > 1) s.dweight = a.take<float>((int64_t)classes * n_in);
        if (f32) {
            const int want = std::max(1, ctx->sm_count * 4 / (int)ep::ceil_div(p.classes, G_CHUNKS * 8));
            s.slabs = std::max<int64_t>(1, std::min<int64_t>(want, ep::ceil_div(p.rows, 2 * G_ROWS)));
        } else
            s.slabs = 8 * (int64_t)most_of(p, rows, classes, [&](int64_t r, int c) {
                          return most_workers(line_of(ctx, ep::ceil_div(c, TILE), ep::ceil_div(r, TILE)));
                      });
        s.kept = p.across <= JOINED_PIECES ? p.across * s.slabs : JOINED_PIECES * s.slabs + 1;
        s.part = a.take<float>((size_t)s.kept * classes);
    }
    const int64_t all = ep::ceil_div(rows, TILE) * TILE;
    s.rows = RowInfo{a.take<float>(all), a.take<float>(all), a.take<int>(all)};
    s.blocks = weight_blocks(ctx, rows);
    s.peaks = a.take<float>(s.blocks);
    s.unclean = a.take<int>(s.blocks);
    s.scale = a.take<Scale>(1);
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
}

struct Given {
    const float *lse, *dloss, *drow;
    const long long *counted;
};
struct Wanted {
    void *dx, *dweight;
    float *dbias;
};

// What is known of the rows, and the operands: x, x without what rows that take no part hold, and W.
template <typename Space>
int prepare(ep_ctx *ctx, Inputs &in, const Space &s, const Given &g, Operand *x, Operand *clean, Operand *w) {
    auto weights = in.type == EP_F32    ? entropy_weights<float>
                   : in.type == EP_BF16 ? entropy_weights<__nv_bfloat16>
                                        : entropy_weights<__half>;
    const Measure measure{g.dloss, g.counted, in.type != EP_F32 && !g.drow, in.type == EP_F16, in.type == EP_F16 ? 14 : 0};
    weights<<<s.blocks, WEIGHT_THREADS, 0, in.stream>>>(g.lse, in.targets, in.rows, in.classes, measure, g.drow, in.x, in.ldx, in.n_in,
                                                        s.copies.bias ? in.bias : nullptr, in.bias_type, s.copies.bias, s.rows, s.peaks,
                                                        s.unclean, s.scale, ctx->d_status);
    ++in.kernels;
    if (s.blocks > 1) {
        EP_CUDA(ctx, ep::launch_early(entropy_scale, dim3(1), dim3(256), 0, in.stream, s.peaks, s.unclean, s.blocks, measure, s.scale));
        ++in.kernels;
    }
    EP_CUDA(ctx, cudaGetLastError());
    const int rc = operands(ctx, in, s.copies, false, x, w);
    if (rc != EP_OK) return rc;
    const bool direct = x->base == in.x;
    const Packed f = ep::packed_form(in.rows, in.n_in, in.type);
    const int grid = (int)std::min<int64_t>(ep::ceil_div(in.rows, 8), (int64_t)ctx->sm_count * 8);
    EP_CUDA(ctx, ep::launch_early(entropy_clean<uint16_t>, dim3((unsigned)grid), dim3(256), 0, in.stream,
                                  direct ? (const uint16_t *)in.x : nullptr, in.ldx, in.rows, in.n_in, s.rows, s.scale, (uint16_t *)s.copies.x,
                                  f.ld, f.parts, f.part_stride));
    ++in.kernels;
    *clean = direct ? Operand{s.copies.x, in.type, in.rows, in.n_in, f.ld, 1, 0} : *x;
    return EP_OK;
}

int launch_round(ep_ctx *ctx, Inputs &in, const float *sums, int64_t n, const Scale *scale, void *out) {
    const int grid = (int)std::min<int64_t>(ep::ceil_div(n, 1024), (int64_t)ctx->sm_count * 8);
    if (in.type == EP_BF16)
        entropy_round<<<grid, 256, 0, in.stream>>>(sums, n, scale, static_cast<__nv_bfloat16 *>(out));
    else
        entropy_round<<<grid, 256, 0, in.stream>>>(sums, n, scale, static_cast<__half *>(out));
    EP_CUDA(ctx, cudaGetLastError());
    ++in.kernels;
    return EP_OK;
}

// G of one piece, and its columns' partial sums.
int slopes_of(ep_ctx *ctx, Inputs &in, const Backward &s, const Given &given, const Operand &x, const Operand &clean, const Operand &w, int64_t row0, int64_t rows,
              int class0, int classes, const Packed &f, bool wanted, float *part) {
    if (in.type == EP_F32) {
        const int rc = logits_of(ctx, in, x, w, row0, rows, class0, classes, s.logits, s.share);
        if (rc != EP_OK) return rc;
        entropy_slopes<float><<<dim3((unsigned)ep::ceil_div(f.ld, G_CHUNKS * 8), (unsigned)s.slabs), 256, 0, in.stream>>>(
            s.logits, f.ld, rows, classes, class0, in.bias, in.bias_type, given.lse + row0, s.rows.from(row0), s.scale, wanted ? s.g : nullptr,
            f.part_stride, part, in.classes);
        EP_CUDA(ctx, cudaGetLastError());
        ++in.kernels;
        return EP_OK;
    }
    TileWork e{};
    e.M = rows;
    e.N = classes;
    e.class0 = class0;
    e.line = line_of(ctx, ep::ceil_div(classes, TILE), ep::ceil_div(rows, TILE));
    e.bias = in.bias ? s.copies.bias : nullptr;
    e.rows = s.rows.from(row0);
    e.scale = s.scale;
    e.sums = part;
    e.stride = in.classes;
    return launch_tiles<true>(ctx, rows_of(x, row0, rows), rows_of(w, class0, classes), s.g, f.ld, rows_of(clean, row0, rows), e, in.stream, &in.kernels);
}

int backward_run(ep_ctx *ctx, Inputs &in, const Backward &s, const Given &given, const Wanted &out) {
    Operand x, clean, w;
    int rc = prepare(ctx, in, s, given, &x, &clean, &w);
    if (rc != EP_OK) return rc;
    const Pieces &p = s.pieces;
    const bool f32 = in.type == EP_F32;
    const size_t size = ep::type_size(in.type);
    const float *factor = f32 ? nullptr : &s.scale->down;
    if (out.dbias && !f32)   // (not every piece has as many partial sums)
        EP_CUDA(ctx, cudaMemsetAsync(s.part, 0, sizeof(float) * s.kept * in.classes, in.stream));
    int64_t slab = 0;
    for (int64_t row0 = 0; row0 < in.rows; row0 += p.rows) {
        const int64_t rows = std::min(p.rows, in.rows - row0);
        const Operand xr = rows_of(x, row0, rows);
        char *dx_rows = out.dx ? static_cast<char *>(out.dx) + row0 * in.n_in * size : nullptr;
        for (int class0 = 0; class0 < in.classes; class0 += p.classes) {
            const int classes = std::min(p.classes, in.classes - class0);
            const Packed f = ep::packed_form(rows, classes, in.type);
            rc = slopes_of(ctx, in, s, given, x, clean, w, row0, rows, class0, classes, f, out.dx || out.dweight,
                           out.dbias ? s.part + slab * in.classes + class0 : nullptr);
            if (rc != EP_OK) return rc;
            const Operand g{s.g, f.type, rows, classes, f.ld, f.parts, f.part_stride};
            if (out.dx) {
                const bool add = p.down > 1;
                rc = ep::product(ctx, g, false, rows_of(w, class0, classes), true, rows, in.n_in, classes,
                                 add && !f32 ? (void *)s.dx : dx_rows, add ? EP_F32 : in.type, class0 > 0, add ? nullptr : factor, s.share,
                                 in.stream, &in.kernels);
                if (rc != EP_OK) return rc;
            }
            if (out.dweight) {
                const bool add = p.across > 1;
                const int64_t at = (int64_t)class0 * in.n_in;
                rc = ep::product_of_either(ctx, g, xr, rows_of(clean, row0, rows), &s.scale->unclean, classes, in.n_in, rows,
                                           add && !f32 ? (void *)(s.dweight + at) : static_cast<char *>(out.dweight) + at * size,
                                           add ? EP_F32 : in.type, row0 > 0, add ? nullptr : factor, s.share, in.stream, &in.kernels);
                if (rc != EP_OK) return rc;
            }
        }
        if (out.dx && p.down > 1 && !f32) {
            rc = launch_round(ctx, in, s.dx, rows * in.n_in, s.scale, dx_rows);
            if (rc != EP_OK) return rc;
        }
        slab += s.slabs;
        if (out.dbias && row0 + p.rows < in.rows && slab + s.slabs > s.kept) {
            rc = ep::sum_partials(ctx, s.part, (int)slab, in.classes, s.part, in.stream);   // (a block reads its columns before it writes them)
            if (rc != EP_OK) return rc;
            ++in.kernels;
            if (!f32) EP_CUDA(ctx, cudaMemsetAsync(s.part + in.classes, 0, sizeof(float) * (s.kept - 1) * in.classes, in.stream));
            slab = 1;
        }
    }
    if (out.dweight && p.across > 1 && !f32) {
        rc = launch_round(ctx, in, s.dweight, (int64_t)in.classes * in.n_in, s.scale, out.dweight);
        if (rc != EP_OK) return rc;
    }
    if (out.dbias) {
        rc = ep::sum_partials(ctx, s.part, (int)slab, in.classes, out.dbias, in.stream);
        if (rc != EP_OK) return rc;
        ++in.kernels;
    }
    return EP_OK;
}

// ---- the backward of narrow rows
bool narrow(int n_in, int type) { return type != EP_F32 && n_in <= FUSED_WIDTH; }
Line fused_line(const ep_ctx *ctx, int64_t p, int64_t q) {
    Line l;
    l.inner = (int)ep::ceil_div(q, Q_ROWS);
    l.tiles = ep::ceil_div(p, P_ROWS) * l.inner;
    // Where there are not four tiles to each SM, workers have whole P tiles, or four tiles each: parts of a P tile have to be written and
    // joined, which takes as long as a few tiles.
    const int64_t outer = ep::ceil_div(p, P_ROWS), parts = ep::ceil_div(l.inner, 4);
    l.workers = (int)std::min<int64_t>(ctx->sm_count, l.tiles <= 4 * ctx->sm_count ? outer * parts : l.tiles);
    return l;
}
int share_width(int n_in) { return (n_in + 31) & ~31; }

struct NarrowSpace {
    Copies copies;
    RowInfo rows;
    float *peaks, *share;
    double *share_bias;
    int *unclean;
    Scale *scale;
    int blocks;
    size_t bytes;
};
NarrowSpace narrow_space(const ep_ctx *ctx, int64_t rows, int n_in, int classes, int type, bool aligned, void *base) {
    ep::Arena a(base);
    NarrowSpace s{};
    s.copies = copies_space(a, rows, n_in, classes, type, aligned, true);
    const int64_t all = ep::ceil_div(rows, TILE) * TILE;
    s.rows = RowInfo{a.take<float>(all), a.take<float>(all), a.take<int>(all)};
    s.share = a.take<float>((size_t)ctx->sm_count * 3 * P_ROWS * share_width(n_in));
    s.share_bias = a.take<double>((size_t)ctx->sm_count * 2 * P_ROWS);
    s.blocks = weight_blocks(ctx, rows);
    s.peaks = a.take<float>(s.blocks);
    s.unclean = a.take<int>(s.blocks);
    s.scale = a.take<Scale>(1);
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
}

// Whether no worker begins inside a P tile.
bool whole_tiles(const Line &l) {
    for (int w = 1; w < l.workers; ++w)
        if (l.begin(w) % l.inner) return false;
    return true;
}
template <bool DW, bool BIASED, bool WIDE, typename T>
int launch_fused_of(ep_ctx *ctx, const CUtensorMap &p, const CUtensorMap &q, const CUtensorMap &clean, const FusedWork &e, cudaStream_t stream) {
    auto kernel = entropy_fused<DW, BIASED, WIDE, T>;
    constexpr size_t smem = FusedMemory<DW, WIDE>::TOTAL;
    EP_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    EP_CUDA(ctx, ep::launch_early(kernel, dim3((unsigned)e.line.workers), dim3(FUSED_THREADS), smem, stream, p, q, clean, e, ctx->d_status));
    // Many workers to a tile: long sums, so fewer of them to a block (rows of 29 in fp16 against 27668 classes: 8 us sooner); else few
    // blocks, most of which have nothing to do (5322 rows against 2723 classes: 13 us sooner).
    const int rows = e.line.workers >= 8 * (e.line.tiles / e.line.inner) ? 4 : 16;
    if (!whole_tiles(e.line))
        EP_CUDA(ctx, ep::launch_early(entropy_join<T>, dim3((unsigned)e.line.workers, P_ROWS / rows), dim3(256), 0, stream, e, rows));
    return EP_OK;
}
// Gradient of x (P = x, Q = W) or of W (P = W, Q = x).
template <bool DW>
int launch_fused(ep_ctx *ctx, Inputs &in, const NarrowSpace &s, const Operand &x, const Operand &clean, const Operand &w, void *out,
                 float *dbias) {
    FusedWork e{};
    e.P = DW ? in.classes : in.rows;
    e.Q = DW ? in.rows : in.classes;
    e.ragged = DW || e.Q % Q_ROWS == 0 ? -1 : (int)(e.Q / Q_ROWS);
    e.width = in.n_in;
    e.boxes = (int)ep::ceil_div(in.n_in, 64);
    e.line = fused_line(ctx, e.P, e.Q);
    const int columns = (in.n_in + 15) & ~15;
    const uint32_t fmt = in.type == EP_BF16 ? 1u : 0u, common = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(P_ROWS >> 4) << 24);
    e.log2e = sums_log2e(in.n_in, in.type);
    e.idesc_s = common | ((uint32_t)(Q_ROWS >> 3) << 17);
    e.idesc_acc = common | (1u << 16) | ((uint32_t)(columns >> 3) << 17);
    e.bias = in.bias ? s.copies.bias : nullptr;
    e.rows = s.rows;
    e.scale = s.scale;
    e.out = out;
    e.dbias = dbias;
    e.vec = in.n_in % 8 == 0 && ep::aligned(out, 16);
    e.share = s.share;
    e.share_bias = s.share_bias;
    e.share_ld = share_width(in.n_in);
    CUtensorMap mp{}, mq{}, mc{};
    if (!encode_operand(&mp, DW ? w : x, false, P_ROWS) || !encode_operand(&mq, DW ? x : w, false, Q_ROWS) ||
        !encode_operand(&mc, clean, false, DW ? Q_ROWS : P_ROWS))
        return ep::fail(ctx, EP_ERR_CUDA, "cuTensorMapEncodeTiled failed for %lld rows of %d classes", (long long)in.rows, in.classes);
    in.kernels += whole_tiles(e.line) ? 1 : 2;
    // (dW of fp16 takes the power of two that G is scaled by with the bias)
    const bool biased = e.bias || (DW && in.type == EP_F16);
    auto launch = [&](auto biased, auto type) {
        using T = decltype(type);
        return in.n_in <= 128 ? launch_fused_of<DW, decltype(biased)::value, false, T>(ctx, mp, mq, mc, e, in.stream)
                              : launch_fused_of<DW, decltype(biased)::value, true, T>(ctx, mp, mq, mc, e, in.stream);
    };
    if (in.type == EP_BF16)
        return biased ? launch(std::true_type{}, __nv_bfloat16{}) : launch(std::false_type{}, __nv_bfloat16{});
    return biased ? launch(std::true_type{}, __half{}) : launch(std::false_type{}, __half{});
}

int narrow_backward_run(ep_ctx *ctx, Inputs &in, const NarrowSpace &s, const Given &given, const Wanted &out) {
    Operand x, clean, w;
    int rc = prepare(ctx, in, s, given, &x, &clean, &w);
    if (rc == EP_OK && out.dx) rc = launch_fused<false>(ctx, in, s, x, clean, w, out.dx, nullptr);
    if (rc == EP_OK && (out.dweight || out.dbias)) rc = launch_fused<true>(ctx, in, s, x, clean, w, out.dweight, out.dbias);
    return rc;
}

// ---- small problems
// (What was measured on both sides stands at the kernels.)  Tiles of 64 x 64 cost the same however little of them there is, and the tile
// kernels' k-blocks of 64 elements and tiles of 128 or 256 rows as much for fewer.
bool small_problem(bool grad, int64_t rows, int n_in, int classes, int type) {
    if ((type != EP_F32 && !grad) || n_in > SMALL_WIDTH || rows > 1 << 20 || (!grad && classes > 512)) return false;
    // (backward, fp32, tiles -> here: 200000 x 16 -> 10 212 -> 183, 18 x 42 -> 77887 121 -> 77; but 39224 x 24 -> 237 101 -> 154)
    const bool empty_tiles = n_in <= 48 && (!grad || std::min<int64_t>(rows, classes) <= ST);
    return ep::ceil_div(rows, ST) * ST * (ep::ceil_div(classes, ST) * ST) * n_in <= (type == EP_F32 && empty_tiles ? 1 << 28 : 1 << 26);
}
// f(J) with J = ceil(n_in / 16).
template <int J = 1, typename F>
int small_width(int n_in, F f) {
    if constexpr (J < SMALL_WIDTH / 16)
        if (n_in > 16 * J) return small_width<J + 1>(n_in, f);
    return f(std::integral_constant<int, J>{});
}
// Shares of a sum over `all` rows of the other operand, so that `tiles` tiles make about two blocks an SM.
int small_splits(const ep_ctx *ctx, int64_t tiles, int64_t all) {
    return (int)std::max<int64_t>(1, std::min<int64_t>(ctx->sm_count * SMALL_BLOCKS / std::max<int64_t>(tiles, 1), ep::ceil_div(all, ST)));
}
struct SmallSpace {
    float2 *stats;
    float *at_target, *dx_part, *dw_part, *db_part, *peaks;
    Finish finish;
    RowInfo rows;
    int *unclean;
    Scale *scale;
    int dx_splits, dw_splits;
    int64_t dx_tiles, dw_tiles;
    size_t bytes;
};
SmallSpace small_space(const ep_ctx *ctx, bool grad, int64_t rows, int n_in, int classes, void *base) {
    ep::Arena a(base);
    SmallSpace s{};
    if (!grad) {
        s.stats = a.take<float2>(ep::ceil_div(classes, ST) * rows);
        s.at_target = a.take<float>(rows);
        s.finish.sums = a.take<double>(ep::ceil_div(rows, FINISH_ROWS));
        s.finish.counts = a.take<long long>(ep::ceil_div(rows, FINISH_ROWS));
        s.finish.ticket = a.take<unsigned>(1);
    } else {
        const int64_t all = ep::ceil_div(rows, TILE) * TILE;
        s.rows = RowInfo{a.take<float>(all), a.take<float>(all), a.take<int>(all)};
        s.peaks = a.take<float>(weight_blocks(ctx, rows));
        s.unclean = a.take<int>(weight_blocks(ctx, rows));
        s.scale = a.take<Scale>(1);
        s.dx_tiles = ep::ceil_div(rows, ST);
        s.dw_tiles = ep::ceil_div(classes, ST);
        s.dx_splits = small_splits(ctx, s.dx_tiles, classes);
        s.dw_splits = small_splits(ctx, s.dw_tiles, rows);
        s.dx_part = a.take<float>(s.dx_splits > 1 ? (size_t)s.dx_splits * rows * n_in : 0);
        s.dw_part = a.take<float>(s.dw_splits > 1 ? (size_t)s.dw_splits * classes * n_in : 0);
        s.db_part = a.take<float>(s.dw_splits > 1 ? (size_t)s.dw_splits * classes : 0);
    }
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
}
SmallWork small_work(const Inputs &in) {
    SmallWork e{};
    e.x = in.x;
    e.ldx = in.ldx;
    e.w = in.w;
    e.ldw = in.ldw;
    e.bias = in.bias;
    e.bias_type = in.bias_type;
    e.targets = in.targets;
    e.rows = in.rows;
    e.n_in = in.n_in;
    e.classes = in.classes;
    e.class_tiles = (int)ep::ceil_div(in.classes, ST);
    return e;
}
int small_forward(ep_ctx *ctx, Inputs &in, const SmallSpace &s, float *loss, float *row_loss, float *lse, long long *counted) {
    SmallWork e = small_work(in);
    e.stats = s.stats;
    e.at_target = s.at_target;
    e.ticket = s.finish.ticket;
    const int rc = small_width(in.n_in, [&](auto j) {
        constexpr int J = decltype(j)::value;
        constexpr size_t smem = sizeof(float) * 2 * ST * (16 * J + 4);
        EP_CUDA(ctx, cudaFuncSetAttribute(entropy_small_forward<J>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        EP_CUDA(ctx, ep::launch_early(entropy_small_forward<J>, dim3((unsigned)e.class_tiles, (unsigned)ep::ceil_div(in.rows, ST)), dim3(256), smem,
                                      in.stream, e));
        return (int)EP_OK;
    });
    if (rc != EP_OK) return rc;
    Finish f = s.finish;
    f.loss = loss;
    f.counted = counted;
    EP_CUDA(ctx, ep::launch_early(entropy_finish, dim3((unsigned)ep::ceil_div(in.rows, FINISH_ROWS)), dim3(256), 0, in.stream,
                                  Statistics{s.stats, in.rows, false, Line{}, e.class_tiles}, s.at_target, in.targets, in.rows, in.classes, in.bias,
                                  in.bias_type, lse, row_loss, f, ctx->d_status));
    in.kernels += 2;
    return EP_OK;
}
template <typename T>
int small_backward(ep_ctx *ctx, Inputs &in, const SmallSpace &s, const Given &g, const Wanted &out) {
    const int blocks = weight_blocks(ctx, in.rows);
    entropy_weights<float><<<blocks, WEIGHT_THREADS, 0, in.stream>>>(g.lse, in.targets, in.rows, in.classes, Measure{g.dloss, g.counted}, g.drow, nullptr,
                                                                     0, 0, nullptr, 0, nullptr, s.rows, s.peaks, s.unclean, s.scale, ctx->d_status);
    EP_CUDA(ctx, cudaGetLastError());
    const bool over_rows = out.dweight || out.dbias;
    SmallWork e = small_work(in);
    e.lse = g.lse;
    e.info = s.rows;
    e.dx_splits = s.dx_splits;
    e.dw_splits = s.dw_splits;
    e.dx_blocks = out.dx ? s.dx_tiles * s.dx_splits : 0;
    e.dx_part = s.dx_part;
    e.dw_part = s.dw_part;
    e.db_part = s.db_part;
    e.dx = out.dx;
    e.dweight = out.dweight;
    e.dbias = out.dbias;
    const int64_t grid = e.dx_blocks + (over_rows ? s.dw_tiles * s.dw_splits : 0);
    const int rc = small_width(in.n_in, [&](auto j) {
        constexpr int J = decltype(j)::value;
        constexpr size_t smem = sizeof(float) * (3 * ST * (16 * J + 4) + ST * (ST + 4));
        EP_CUDA(ctx, cudaFuncSetAttribute(entropy_small_backward<T, J>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        EP_CUDA(ctx, ep::launch_early(entropy_small_backward<T, J>, dim3((unsigned)grid), dim3(256), smem, in.stream, e));
        return (int)EP_OK;
    });
    if (rc != EP_OK) return rc;
    in.kernels += 2;
    // many shares: a warp to an element
    auto fold = [&](const float *part, int splits, int64_t n, void *to, const float *more_part, int64_t more, float *more_to) {
        if (splits == 1 || n + more == 0) return cudaSuccess;
        ++in.kernels;
        const int lanes = splits > 16 ? 32 : 1;
        auto kernel = lanes > 1 ? entropy_small_fold<T, 32> : entropy_small_fold<T, 1>;
        return ep::launch_early(kernel, dim3((unsigned)ep::ceil_div((n + more) * lanes, 256)), dim3(256), 0, in.stream, part, splits, n,
                                static_cast<T *>(to), more_part, more, more_to);
    };
    EP_CUDA(ctx, fold(e.dx_part, e.dx_splits, out.dx ? in.rows * in.n_in : 0, e.dx, nullptr, 0, nullptr));
    EP_CUDA(ctx, fold(e.dw_part, e.dw_splits, out.dweight ? (int64_t)in.classes * in.n_in : 0, e.dweight, e.db_part, out.dbias ? in.classes : 0,
                      out.dbias));
    return EP_OK;
}

}  // namespace

using namespace ep;

namespace {
bool element_aligned(const void *p, int type) { return !p || aligned(p, (size_t)type_size(type)); }
bool can_be_read_by_tma(const void *p, int64_t ld, int type) { return aligned(p, 16) && ld * type_size(type) % 16 == 0; }

int check_inputs(ep_ctx *ctx, const Inputs &in) {
    if (!entropy_shape_ok(in.rows, in.n_in, in.classes))
        return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld, n_in %d or classes %d out of range", (long long)in.rows, in.n_in, in.classes);
    if (!float_type(in.type) || (in.bias && !float_type(in.bias_type)))
        return fail(ctx, EP_ERR_INVALID_ARG, "no cross entropy of type %d", in.type);
    if (in.ldx < in.n_in || in.ldw < in.n_in) return fail(ctx, EP_ERR_INVALID_ARG, "a row stride is shorter than its row");
    if (!element_aligned(in.x, in.type) || !element_aligned(in.w, in.type) || !element_aligned(in.bias, in.bias ? in.bias_type : EP_E4M3) ||
        !aligned(in.targets, 4) || !in.w || (in.rows && (!in.x || !in.targets)))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    return EP_OK;
}
}  // namespace

extern "C" {

size_t ep_cross_entropy_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t n_in, int32_t classes, int32_t in_type,
                                        int32_t is_aligned) {
    if (!ctx || !entropy_shape_ok(rows, n_in, classes) || !float_type(in_type)) return 0;
    if (small_problem(false, rows, n_in, classes, in_type)) return small_space(ctx, false, rows, n_in, classes, nullptr).bytes;
    return forward_space(ctx, rows, n_in, classes, in_type, is_aligned != 0, nullptr).bytes;
}

int ep_cross_entropy(ep_ctx *ctx, const void *x, int64_t ldx, const void *w, int64_t ldw, int32_t in_type, const void *bias,
                     int32_t bias_type, const int32_t *targets, int64_t rows, int32_t n_in, int32_t classes, float *loss,
                     float *row_loss, float *lse, int64_t *counted, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    Inputs in{x, ldx, w, ldw, in_type, bias, bias_type, targets, rows, n_in, classes, false, static_cast<cudaStream_t>(cuda_stream), 0};
    int rc = check_inputs(ctx, in);
    if (rc != EP_OK) return rc;
    if (!loss || !counted || !aligned(loss, 4) || !aligned(counted, 8) || !aligned(row_loss, 4) || !aligned(lse, 4) ||
        (rows && (!row_loss || !lse)))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    DeviceGuard guard(ctx->device);
    if (rows == 0) {
        EP_CUDA(ctx, cudaMemsetAsync(loss, 0, sizeof(float), in.stream));
        EP_CUDA(ctx, cudaMemsetAsync(counted, 0, sizeof(int64_t), in.stream));
        return EP_OK;
    }
    in.aligned = can_be_read_by_tma(x, ldx, in_type) && can_be_read_by_tma(w, ldw, in_type);
    const bool small = small_problem(false, rows, n_in, classes, in_type);
    const SmallSpace few = small ? small_space(ctx, false, rows, n_in, classes, workspace) : SmallSpace{};
    const ForwardSpace s = small ? ForwardSpace{} : forward_space(ctx, rows, n_in, classes, in_type, in.aligned, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < std::max(few.bytes, s.bytes))
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    long long *count = reinterpret_cast<long long *>(counted);
    Timed tm(ctx, in.stream, EP_TIMER_ENTROPY);
    rc = small ? small_forward(ctx, in, few, loss, row_loss, lse, count) : forward_run(ctx, in, s, loss, row_loss, lse, count);
    tm.end(in.kernels);
    return rc;
}

size_t ep_cross_entropy_backward_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t n_in, int32_t classes, int32_t in_type,
                                                 int32_t is_aligned) {
    if (!ctx || !entropy_shape_ok(rows, n_in, classes) || !float_type(in_type)) return 0;
    if (small_problem(true, rows, n_in, classes, in_type)) return small_space(ctx, true, rows, n_in, classes, nullptr).bytes;
    return narrow(n_in, in_type) ? narrow_space(ctx, rows, n_in, classes, in_type, is_aligned != 0, nullptr).bytes
                                 : backward_space(ctx, rows, n_in, classes, in_type, is_aligned != 0, nullptr).bytes;
}

int ep_cross_entropy_backward(ep_ctx *ctx, const void *x, int64_t ldx, const void *w, int64_t ldw, int32_t in_type, const void *bias,
                              int32_t bias_type, const int32_t *targets, const float *lse, const int64_t *counted, const float *dloss,
                              const float *drow_loss, int64_t rows, int32_t n_in, int32_t classes, void *dx, void *dweight,
                              float *dbias, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    Inputs in{x, ldx, w, ldw, in_type, bias, bias_type, targets, rows, n_in, classes, false, static_cast<cudaStream_t>(cuda_stream), 0};
    int rc = check_inputs(ctx, in);
    if (rc != EP_OK) return rc;
    if (!element_aligned(dx, in_type) || !element_aligned(dweight, in_type) || !aligned(dbias, 4) || !aligned(lse, 4) ||
        !aligned(counted, 8) || !aligned(dloss, 4) || !aligned(drow_loss, 4) || (rows && (!lse || !counted)))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    DeviceGuard guard(ctx->device);
    if (rows == 0) {
        if (dweight) EP_CUDA(ctx, cudaMemsetAsync(dweight, 0, (size_t)classes * n_in * type_size(in_type), in.stream));
        if (dbias) EP_CUDA(ctx, cudaMemsetAsync(dbias, 0, sizeof(float) * (size_t)classes, in.stream));
        return EP_OK;
    }
    if (!dx && !dweight && !dbias) return EP_OK;
    in.aligned = can_be_read_by_tma(x, ldx, in_type) && can_be_read_by_tma(w, ldw, in_type);
    const bool small = small_problem(true, rows, n_in, classes, in_type), in_tmem = !small && narrow(n_in, in_type);
    const SmallSpace few = small ? small_space(ctx, true, rows, n_in, classes, workspace) : SmallSpace{};
    const NarrowSpace n = in_tmem ? narrow_space(ctx, rows, n_in, classes, in_type, in.aligned, workspace) : NarrowSpace{};
    const Backward s = small || in_tmem ? Backward{} : backward_space(ctx, rows, n_in, classes, in_type, in.aligned, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < std::max({few.bytes, n.bytes, s.bytes}))
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    const Given given{lse, dloss, drow_loss, reinterpret_cast<const long long *>(counted)};
    const Wanted out{dx, dweight, dbias};
    Timed tm(ctx, in.stream, EP_TIMER_ENTROPY);
    rc = small     ? (in_type == EP_F32    ? small_backward<float>(ctx, in, few, given, out)
                      : in_type == EP_BF16 ? small_backward<__nv_bfloat16>(ctx, in, few, given, out)
                                           : small_backward<__half>(ctx, in, few, given, out))
         : in_tmem ? narrow_backward_run(ctx, in, n, given, out)
                   : backward_run(ctx, in, s, given, out);
    tm.end(in.kernels);
    return rc;
}

}  // extern "C"
