// Product with a weight matrix, with bias, activation and residual in its epilogue, and its backward pass.
//
// One tile kernel (linear_tiles) serves the forward product and both gradients: D[M, N] = sum_k A[m, k] B[n, k] with
// either operand stored along k ("K-major") or along its own rows ("MN-major", 16-bit types), so that no operand is
// ever transposed in memory:
//     z  = x W^T     A = x  (K-major)     B = W (K-major)
//     dx = dz W      A = dz (K-major)     B = W (MN-major)
//     dW = dz^T x    A = dz (MN-major)    B = x (MN-major)
// Beside it: a dot-product kernel for the fewest rows (serving), the kernel that makes dz and sums dbias, one that
// copies unaligned operands or splits fp32 ones into three bf16 numbers, and one that joins the shares of a sum over k
// that was split between blocks.
//
// Measured: 8192 x 4096 x 4096 fp16 193 us, 1430 TFLOP/s (tensor pipe 90 % busy; cuBLAS alone reaches 1669 in short bursts);
// 2000 x 4096 x 4096 in 8 bits 31 us, 2150 TFLOP/s (1.7 waves of tiles, so 2); 169343 x 128 -> 512 bf16 41 us, 5.3 TB/s of
// 6.5, with z kept 76 us, 5.2 TB/s; backward of 232965 x 256 x 256 bf16 through GELU 155 us: dz 62, dx 44, dW 46 and its
// join 7, against 74 us for reading and writing everything once; one row of 1024 x 1024 3 us.  fp32 by six bf16 products:
// 8192 x 4096 x 4096 1266 us, 217 TFLOP/s of 278 (a sixth of bf16's); 169343 x 128 -> 512 219 us.
#include "ep_common.cuh"
#include "rows.cuh"
#include "tc_device.cuh"

#include <algorithm>
#include <initializer_list>
#include <mutex>
#include <type_traits>

using namespace eprow;
using namespace eptc;

namespace {

// ---------------------------------------------------------------------------------------------- epilogue
struct Epilogue {
    const float *x_scale, *w_scale;   // of 8-bit inputs
    const void *bias;
    int bias_type, act;
    const void *residual;
    int64_t ldr;
    void *out, *preact;
    int out_type;
    int64_t M;
    int N;
    bool vec;                         // out, preact, residual, bias, scales: 16-byte rows of whole 8-column chunks
    bool tma;                         // out and preact can be written by TMA, the residual read by 16 bytes
    const float *factor;              // of fp16 results: what the sums are multiplied by first (one value), or NULL
    float *share;                     // where a block's share of a split sum goes: [split][M][ld_share] fp32
    int ld_share;
};

// The upper tail of the normal distribution at |z|, over exp(-z^2 / 2): a polynomial in t = 1 / (1 + 0.35 |z|), fitted
// (weighted least squares, reweighted towards the largest error) to 1.1e-7 (1 + z^2) of the tail itself up to |z| = 14,
// where fp32 loses as much by rounding the exponential's argument.  The gradient needs the same exponential, and where the
// slope of z Phi(z) crosses zero the exponential is a common factor of the terms that cancel.
// For z = (z0, z1): the bell exp(-z^2 / 2), |z| and that tail.
__device__ __forceinline__ void normal_parts(float z0, float z1, Pair &bell, Pair &size, Pair &tail) {
    const Pair z(z0, z1);
    size = Pair(fabsf(z0), fabsf(z1));
    float a, b;
    fma2(size, Pair(0.35f), Pair(1.f)).get(a, b);
    const Pair t(reciprocal_fast(a), reciprocal_fast(b));
    Pair q = fma2(t, Pair(0.0452263094f), Pair(-0.186698169f));
    q = fma2(q, t, Pair(0.214374468f));
    q = fma2(q, t, Pair(0.00660444144f));
    q = fma2(q, t, Pair(0.143951952f));
    q = fma2(q, t, Pair(0.136762664f));
    q = fma2(q, t, Pair(0.139778391f));
    tail = mul2(q, t);
    mul2(mul2(z, z), Pair(-0.5f * 1.44269504f)).get(a, b);
    bell = Pair(exp2_fast(a), exp2_fast(b));
}
// q bell below zero, 1 - q bell above: Phi(z) and the slope of z Phi(z) from what they are at -|z|.  Chosen, not computed
// from one another: 1 - (1 - m) would leave nothing of a small m.
__device__ __forceinline__ Pair either_side(float z0, float z1, Pair q, Pair bell) {
    float low0, low1, high0, high1;
    const Pair m = mul2(q, bell);
    m.get(low0, low1);
    fma2(m, Pair(-1.f), Pair(1.f)).get(high0, high1);
    return Pair(z0 >= 0.f ? high0 : low0, z1 >= 0.f ? high1 : low1);
}
__device__ __forceinline__ void gelu2(float &v0, float &v1) {
    Pair bell, size, tail;
    normal_parts(v0, v1, bell, size, tail);
    mul2(Pair(v0, v1), either_side(v0, v1, tail, bell)).get(v0, v1);
}
// v *= slope of GELU at z
__device__ __forceinline__ void times_gelu_slope2(float &v0, float &v1, float z0, float z1) {
    Pair bell, size, tail;
    normal_parts(z0, z1, bell, size, tail);
    const Pair q = fma2(size, Pair(-0.39894228f), tail);
    mul2(Pair(v0, v1), either_side(z0, z1, q, bell)).get(v0, v1);
}

// act(z) of n values; the switch is outside the loops, and taken by all threads alike.
template <int n>
__device__ __forceinline__ void activate(float (&v)[n], int act) {
    if (act == EP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v[i]));   // (a NaN stays one)
    } else if (act == EP_ACT_GELU) {
#pragma unroll
        for (int i = 0; i + 1 < n; i += 2) gelu2(v[i], v[i + 1]);
        if constexpr (n % 2 == 1) {
            float none = 0.f;
            gelu2(v[n - 1], none);
        }
    } else if (act == EP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] *= reciprocal_fast(1.f + exp_fast(-v[i]));   // (1 / infinity: far below zero the sigmoid is 0)
    }
}
// v *= act'(z)
template <int n>
__device__ __forceinline__ void times_slope(float (&v)[n], const float (&z)[n], int act) {
    if (act == EP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = z[i] > 0.f ? v[i] : 0.f;
    } else if (act == EP_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < n; i += 2) times_gelu_slope2(v[i], v[i + 1], z[i], z[i + 1]);
    } else if (act == EP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float s = reciprocal_fast(1.f + exp_fast(-z[i]));
            v[i] *= s * fmaf(z[i], 1.f - s, 1.f);
        }
    }
}

// What a thread needs of n columns, the same for every row that it finishes.
template <int n>
struct Columns {
    float bias[n], scale[n];
    __device__ __forceinline__ void load(const Epilogue &e, int col) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            bias[i] = 0.f;
            scale[i] = 1.f;
        }
        if (e.bias) {   // (vec is only set where the bias is aligned too)
            if (e.bias_type == EP_F32)
                load_chunk(static_cast<const float *>(e.bias), col, e.N, n > 1 && e.vec, 0.f, bias);
            else if (e.bias_type == EP_BF16)
                load_chunk(static_cast<const __nv_bfloat16 *>(e.bias), col, e.N, n > 1 && e.vec, 0.f, bias);
            else
                load_chunk(static_cast<const __half *>(e.bias), col, e.N, n > 1 && e.vec, 0.f, bias);
        }
        if (e.w_scale) load_chunk(e.w_scale, col, e.N, n > 1 && e.vec, 1.f, scale);
    }
};

// n finished sums of one row, from column col on: scale, bias, (store z), activation, residual, store.  `r` holds the
// residual, where there is one.
template <typename O, int n>
__device__ __forceinline__ void finish(const Epilogue &e, int64_t row, int col, const Columns<n> &c, float (&v)[n],
                                       const float (&r)[n]) {
    if constexpr (std::is_same_v<O, __half>) {
        if (e.factor) {
            const float f = *e.factor;
#pragma unroll
            for (int i = 0; i < n; ++i) v[i] *= f;
        }
    }
    if (e.x_scale) {
        const float xs = e.x_scale[row];
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] *= xs * c.scale[i];
    }
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] += c.bias[i];
    const bool vec = n > 1 && e.vec;
    if (e.preact) store_chunk(static_cast<O *>(e.preact) + row * e.N, col, e.N, vec, v);
    activate(v, e.act);
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] += r[i];
    }
    store_chunk(static_cast<O *>(e.out) + row * e.N, col, e.N, vec, v);
}
template <typename O, int n>
__device__ __forceinline__ void load_residual(const Epilogue &e, int64_t row, int col, float (&r)[n]) {
    if (e.residual)
        load_chunk(static_cast<const O *>(e.residual) + row * e.ldr, col, e.N, n > 1 && e.vec, 0.f, r);
    else {
#pragma unroll
        for (int i = 0; i < n; ++i) r[i] = 0.f;
    }
}

// ---------------------------------------------------------------------------------------------- a chunk of the output
// A warp's 32 rows of a few columns, one row per lane, are finished in registers and leave through shared memory by TMA,
// which writes whole lines and cuts off what lies outside the matrix.  (Finished from shared memory in a coalesced
// order instead, addresses, bounds and types made 18 instructions per element, and the epilogue took longer than the
// sums and the memory both: 169343 x 128 -> 512 in 137 us.)  Boxes have rows of 128 bytes where the tile allows: TMA
// takes them row by row, and rows of 64 bytes cost as much.
constexpr int SLOT_BYTES = 4096;   // a warp's room in shared memory: one such chunk
template <typename O, int COLS>
struct ChunkStore {
    static constexpr int G = 16 / (int)sizeof(O);                                   // columns of a 16-byte piece
    static constexpr int WIDTH = 128 / (int)sizeof(O) < COLS ? 128 / (int)sizeof(O) : COLS;
    static constexpr int ROW = WIDTH * (int)sizeof(O);                              // bytes of a row of the box: 64 or 128
    // Where piece c of row r lies: as the swizzle of a TMA box of 64- or 128-byte rows has it (no two lanes that
    // access a piece each together meet in a bank).
    static __device__ __forceinline__ int at(int r, int c) { return r * ROW + ((ROW == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7)) << 4); }
    // 32 of a lane's columns, from piece c0 on
    static __device__ __forceinline__ void write(char *slot, int lane, int c0, const float (&v)[32]) {
#pragma unroll
        for (int c = 0; c < 32 / G; ++c) {
            float w[G];
#pragma unroll
            for (int i = 0; i < G; ++i) w[i] = v[c * G + i];
            store_chunk(reinterpret_cast<O *>(slot + at(lane, c0 + c)), 0, 1 << 30, true, w);
        }
    }
    static __device__ __forceinline__ void add(const char *slot, int lane, int c0, float (&v)[32]) {
#pragma unroll
        for (int c = 0; c < 32 / G; ++c) {
            float w[G];
            load_chunk(reinterpret_cast<const O *>(slot + at(lane, c0 + c)), 0, 1 << 30, true, 0.f, w);
#pragma unroll
            for (int i = 0; i < G; ++i) v[c * G + i] += w[i];
        }
    }
};

// Called by the whole warp; the elected lane (always the same one) issues.
__device__ __forceinline__ void tma_store_3d_elected(const CUtensorMap *map, const void *src, int x, int y, int z) {
    asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                 "@pe cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];\n"
                 "@pe cp.async.bulk.commit_group;\n}" ::"l"(map),
                 "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
// Until at most PENDING of the warp's stores still read shared memory; all lanes may then write there.  (Only the elected
// lane has any to wait for.)
template <int PENDING>
__device__ __forceinline__ void stores_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
    __syncwarp();
}
// What the lanes have written becomes visible to the stores that are issued next.
__device__ __forceinline__ void before_stores() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

// Rows that TMA cannot write: a warp's 32 x 32 sums from shared memory (element j of row r at 32 r + (j + r) % 32, which
// keeps lanes in different banks both ways), a column to each lane so that neighbouring lanes write neighbouring elements.
// What counts here is the number of instructions: each takes a warp about five clocks (with addresses and bounds worked
// out for every row, 10000 x 65 fp32 took 5.5 us a chunk).
template <typename O>
struct LooseRows {
    O *out, *z;
    const O *residual;
    const float *x_scale;
    int64_t ldr;
    int ldo, rows, act;
    float bias, scale;
    const float *sums;
};
template <typename O>
__device__ __noinline__ void finish_rows(LooseRows<O> w) {
    const int lane = threadIdx.x & 31;
    const bool plain = !w.z && !w.residual && !w.x_scale && w.act == EP_ACT_NONE;
#pragma unroll 1
    for (int r0 = 0; r0 < w.rows; r0 += 8, w.sums += 8 * 32) {
        const bool whole = r0 + 8 <= w.rows;
        float v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = w.sums[r * 32 + ((lane + r0 + r) & 31)];
        if (plain) {
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] += w.bias;
        } else {
            float add[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) add[r] = 0.f;
            if (w.residual) {
#pragma unroll
                for (int r = 0; r < 8; ++r, w.residual += w.ldr)
                    if (whole || r0 + r < w.rows) add[r] = to_f32(*w.residual);
            }
            if (w.x_scale) {
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (whole || r0 + r < w.rows) v[r] *= w.x_scale[r0 + r] * w.scale;
            }
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] += w.bias;
            if (w.z) {
#pragma unroll
                for (int r = 0; r < 8; ++r, w.z += w.ldo)
                    if (whole || r0 + r < w.rows) *w.z = from_f32<O>(v[r]);
            }
            activate(v, w.act);
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] += add[r];
        }
        if (whole) {
#pragma unroll
            for (int r = 0; r < 8; ++r, w.out += w.ldo) *w.out = from_f32<O>(v[r]);
        } else {
#pragma unroll
            for (int r = 0; r < 8; ++r, w.out += w.ldo)
                if (r0 + r < w.rows) *w.out = from_f32<O>(v[r]);
        }
    }
}

// ---------------------------------------------------------------------------------------------- the tile kernel
//
// 128 x BN outputs per tile, one block per SM that goes from tile to tile: one warp brings k-blocks (128 bytes along k)
// by TMA into a ring, the last one issues the MMAs, the others finish a tile while the next one is being summed (two
// accumulators in TMEM).
//
// PARTS == 3: fp32 operands as three bf16 numbers each, x = x1 + x2 + x3 (|x2| < 2^-7 |x|, |x3| <= 2^-16 |x|).  Of the
// nine products the six down to 2^-16 are summed; the other three are below 2^-22 together.  x1 w1 has an accumulator of
// its own, the five small products share a second one.
//
// RUNS: the tensor core's fp32 sums are truncated, which costs up to an ulp of the running sum a step, always
// downwards (measured on sums of one sign: 1.0e-7 of the result a step, after 64 steps as after 4096).  Where the output is
// fp32, sums therefore run over 4 k-blocks only (16 steps), and the epilogue's threads add the runs to nearest in their
// registers.  Sums of 16-bit outputs run up to a ninth of the output's rounding unit (through_kb).  Longer ones are
// added up beside the accumulator, in the TMEM that otherwise is the second accumulator (GemmShape::keep): the MMAs then
// wait while a run is added, 1 to 2 % of the time (weights' gradient of 169343 x 2048 x 2048 fp16 1045 -> 1066 us, of
// 60000 x 4096 x 4096 1520 -> 1550).
//
// PAIR: two blocks of a cluster (one TPC's two SMs) work on one tile of 256 x BN.  Either keeps 128 rows of A and half of
// B in its shared memory and 128 rows of the sums in its TMEM; the first one's MMA warp issues for both.  A block then
// loads half as much of B for the same product: a 128 x 256 tile alone needs 96 bytes a clock from the L2 at full rate.
constexpr int BM = 128;               // rows of a block
constexpr int A_BYTES = BM * 128;
constexpr int RUN_KB = 4;
// The k-blocks (of four steps) that may run through where the output is of 16 bits: 512 steps cost 5e-5 and fp16's rounding
// 4.9e-4, 4096 steps 4.2e-4 and bf16's 3.9e-3.
constexpr int through_kb(int out_type) { return out_type == EP_F16 ? 128 : 1024; }
constexpr int MAX_STAGES = 8;
constexpr int TMEM_COLS = 512;

struct GemmShared {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], t_full[2], t_empty[2], drain;
    uint32_t tmem_base;
    int abort;
};

// The shared memory of a block: ring of operand stages, then per epilogue warp room for chunks on their way out.
// The epilogue's instructions follow one another closely (sum, bias, activation, store), so it takes warps to fill a
// scheduler: 16 where every one of them still has 32 columns (169343 x 128 -> 512 bf16: 41 us against 51 with 8, through
// GELU and with a residual 95 against 137; all of 16-bit outputs).  18 warps leave a thread 96 registers, which sums in
// runs exceed: the kernel of split fp32 in pairs spills 336 bytes, two others of fp32 outputs 12.
template <int BN, int PARTS, bool PAIR>
struct TileMemory {
    static constexpr int EPI_WARPS = BN >= 128 ? 16 : 8;
    static constexpr int THREADS = 32 * (EPI_WARPS + 2);
    static constexpr int B_ROWS = PAIR ? BN / 2 : BN;
    static constexpr int B_BYTES = B_ROWS * 128;
    static constexpr int STAGE_BYTES = PARTS * (A_BYTES + B_BYTES);
    static constexpr int STAGING_BYTES = EPI_WARPS * SLOT_BYTES;
    static constexpr int REST = 1024 + STAGING_BYTES + (int)sizeof(GemmShared);
    static constexpr int FIT = (227 * 1024 - REST) / STAGE_BYTES;
    static constexpr int STAGES = FIT < MAX_STAGES ? FIT : MAX_STAGES;
    static constexpr int RING_BYTES = STAGES * STAGE_BYTES;
    static constexpr size_t TOTAL = (size_t)REST + RING_BYTES;
    static_assert(STAGES >= 2 && TOTAL <= 227 * 1024, "shared memory of a block");
};

struct GemmShape {
    int64_t M;
    int N;
    int tiles_n, tiles_m;
    int step_m, step_n;   // one worker's way from tile to tile: tiles of M and of N
    int64_t tiles;        // tiles of the output
    int64_t items;        // tiles x splits
    int splits, kb;       // shares of the sum; k-blocks of all of it (share s takes k-blocks s, s + splits, ...)
    int run_kb;           // k-blocks of a run
    bool keep;            // 16-bit outputs: a share has several runs, added up in TMEM
    bool a_mn, b_mn;      // operand stored along its rows
    bool backwards;       // the last row of tiles first: where A has just been written, its end is still in the L2
    uint32_t idesc;       // without the number of columns
};

// The four K-steps of one k-block.
#define EP_UMMA_KBLOCK(GROUP, KIND)                                                                                        \
    asm volatile("{\n.reg .pred pe, pa, pt;\n"                                                                             \
                 "elect.sync _|pe, 0xffffffff;\n"                                                                          \
                 "setp.ne.b32 pa, %10, 0;\nsetp.eq.b32 pt, 0, 0;\n"                                                        \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %5, %9, pa;\n"                             \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %2, %6, %9, pt;\n"                             \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %3, %7, %9, pt;\n"                             \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %4, %8, %9, pt;\n}" ::"r"(d_tmem),             \
                 "l"(adesc), "l"(a1), "l"(a2), "l"(a3), "l"(bdesc), "l"(b1), "l"(b2), "l"(b3), "r"(idesc),                 \
                 "r"(accumulate_first)                                                                                     \
                 : "memory")
template <bool F8, bool PAIR>
__device__ __forceinline__ void umma_kblock_elected(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint64_t astep,
                                                    uint64_t bstep, uint32_t idesc, uint32_t accumulate_first) {
    const uint64_t a1 = adesc + astep, a2 = a1 + astep, a3 = a2 + astep;
    const uint64_t b1 = bdesc + bstep, b2 = b1 + bstep, b3 = b2 + bstep;
    if constexpr (F8 && PAIR)
        EP_UMMA_KBLOCK("2", "f8f6f4");
    else if constexpr (F8)
        EP_UMMA_KBLOCK("1", "f8f6f4");
    else if constexpr (PAIR)
        EP_UMMA_KBLOCK("2", "f16");
    else
        EP_UMMA_KBLOCK("1", "f16");
}
#undef EP_UMMA_KBLOCK

// Forms for a pair of blocks.  The barrier's address may be the other block's (shared::cluster).
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// (relaxed: nothing but the reading of TMEM goes before it, which tcgen05's own fence and wait order; with release an
// arrival at the other block took 1500 clocks)
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void load_tile_elected(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                     "@pe cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], "
                     "[%1, {%2, %3, %4}], [%5];\n}" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                     : "memory");
    else
        asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                     "@pe cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], "
                     "[%1, {%2, %3, %4}], [%5];\n}" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                     : "memory");
}
// One arrival at the barrier, of both blocks where there are two, when all MMAs issued so far are done.
template <bool PAIR>
__device__ __forceinline__ void commit_elected(uint64_t *bar) {
    if constexpr (PAIR)
        asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                     "@pe tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(
                         smem_u32(bar)),
                     "h"((uint16_t)3)
                     : "memory");
    else
        umma_commit_elected(bar);
}

// Shared-memory descriptor of an operand tile, 128-byte swizzle.  K-major: rows of 128 bytes along k, groups of 8 rows
// 1024 bytes apart; a K-step is 32 bytes further along the row.  MN-major: boxes of 64 columns x 64 k, 8192 bytes
// apart; inside a box rows of 128 bytes hold the 64 columns of one k, groups of 8 k are 1024 bytes apart, and a K-step
// of 16 k is two groups on.
__device__ __forceinline__ uint64_t operand_desc(uint32_t smem, bool mn) {
    const uint64_t lead = mn ? 8192 >> 4 : 1;
    return (uint64_t)((smem & 0x3FFFFu) >> 4) | (lead << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// One worker's tiles: first, first + workers, ...  Tiles of one row of tiles come one after another (they share A, and B
// stays in the L2); splits outermost.  Only the first is found by division.
template <int TILE_M, int TILE_N>
struct Items {
    const GemmShape &g;
    int tm, tn, split;
    __device__ __forceinline__ Items(const GemmShape &shape, int64_t first) : g(shape) {
        split = (int)(first / g.tiles);
        const int64_t tile = first - (int64_t)split * g.tiles;
        tm = (int)(tile / g.tiles_n);
        tn = (int)(tile - (int64_t)tm * g.tiles_n);
    }
    __device__ __forceinline__ bool more() const { return split < g.splits; }
    __device__ __forceinline__ void next() {
        tm += g.step_m;
        tn += g.step_n;
        if (tn >= g.tiles_n) {
            tn -= g.tiles_n;
            ++tm;
        }
        while (tm >= g.tiles_m) {
            tm -= g.tiles_m;
            ++split;
        }
    }
    __device__ __forceinline__ int m0() const { return (g.backwards ? g.tiles_m - 1 - tm : tm) * TILE_M; }
    __device__ __forceinline__ int n0() const { return tn * TILE_N; }
    // Columns that the MMAs compute: the last tile's are cut to what the matrix has, in steps of 16.
    __device__ __forceinline__ int columns() const { return min(TILE_N, (g.N - n0() + 15) & ~15); }
    __device__ __forceinline__ int kbn() const { return (g.kb - split + g.splits - 1) / g.splits; }
};

template <int BN, bool F8, int PARTS, bool RUNS, bool PAIR, typename O>
__global__ void __launch_bounds__(TileMemory<BN, PARTS, PAIR>::THREADS, 1) linear_tiles(const __grid_constant__ CUtensorMap map_a,
                                                                const __grid_constant__ CUtensorMap map_b,
                                                                const __grid_constant__ CUtensorMap map_out,
                                                                const __grid_constant__ CUtensorMap map_z,
                                                                const GemmShape g, const Epilogue e, int *status) {
    using Mem = TileMemory<BN, PARTS, PAIR>;
    constexpr int B_BYTES = Mem::B_BYTES, STAGE_BYTES = Mem::STAGE_BYTES, STAGES = Mem::STAGES;
    constexpr int EPI_WARPS = Mem::EPI_WARPS, TMA_WARP = EPI_WARPS;
    constexpr int ACC_COLS = BN * (PARTS == 3 ? 2 : 1);
    constexpr int KE = F8 ? 128 : 64;   // elements of k in a k-block
    constexpr int TILE_M = PAIR ? 2 * BM : BM;
    static_assert(2 * ACC_COLS <= TMEM_COLS, "accumulators");
    static_assert(PARTS == 1 || RUNS, "the split product is summed in runs");

    extern __shared__ char smem_raw[];
    char *ring = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    char *staging = ring + Mem::RING_BYTES;
    GemmShared *sh = reinterpret_cast<GemmShared *>(staging + Mem::STAGING_BYTES);
    const uint32_t rank = PAIR ? cluster_rank() : 0;     // rank 0 issues the MMAs
    const int64_t worker = PAIR ? blockIdx.x >> 1 : blockIdx.x;
    using Walk = Items<TILE_M, BN>;
    volatile int *abort_flag = &sh->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&sh->full[s], 1);
            mbar_init(&sh->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sh->t_full[b], 1);
            mbar_init(&sh->t_empty[b], PAIR ? 2 * EPI_WARPS : EPI_WARPS);   // (of both blocks, at the first one's)
        }
        mbar_init(&sh->drain, 1);
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                         "r"(TMEM_COLS)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                         "r"(TMEM_COLS)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_meet();   // the other block's barriers are ready
    tc_fence_after();
    ep_wait_for_launch_before();          // (everything up to here needs no memory of the launch before)
    ep_let_next_launch_start();
    const uint32_t tmem_base = sh->tmem_base;

    if (warp == TMA_WARP) {
        uint32_t it = 0, s = 0, ph = 0;
        bool ok = true;
        const uint32_t ring_base = smem_u32(ring);
        for (Walk t(g, worker); ok && t.more(); t.next()) {
            const int m = t.m0() + (int)rank * BM, n = t.n0() + (int)rank * (t.columns() / 2);   // this block's rows of A and of B
            const int kbn = t.kbn();
            for (int kb = 0; kb < kbn; ++kb, ++it) {
                if (!(ok = mbar_wait_warp(&sh->empty[s], ph ^ 1u, abort_flag))) break;
                if (rank == 0) mbar_expect_tx_elected(&sh->full[s], (PAIR ? 2 : 1) * STAGE_BYTES);
                const uint32_t bar = PAIR ? in_block(smem_u32(&sh->full[s]), 0) : smem_u32(&sh->full[s]);
                const int k = (t.split + kb * g.splits) * KE;
                uint32_t dst = ring_base + s * (uint32_t)STAGE_BYTES;
#pragma unroll
                for (int p = 0; p < PARTS; ++p, dst += A_BYTES) {
                    if (!g.a_mn)
                        load_tile_elected<PAIR>(dst, &map_a, k, m, p, bar);
                    else {
#pragma unroll
                        for (int b = 0; b < BM / 64; ++b)
                            load_tile_elected<PAIR>(dst + b * 8192, &map_a, m + 64 * b, k, p, bar);
                    }
                }
#pragma unroll
                for (int p = 0; p < PARTS; ++p, dst += B_BYTES) {
                    if (!g.b_mn)
                        load_tile_elected<PAIR>(dst, &map_b, k, n, p, bar);
                    else {
#pragma unroll
                        for (int b = 0; b < Mem::B_ROWS / 64; ++b)
                            load_tile_elected<PAIR>(dst + b * 8192, &map_b, n + 64 * b, k, p, bar);
                    }
                }
                if (++s == (uint32_t)STAGES) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
        // after an abort the loads already issued get time to land before the block leaves (those of a pair all count at
        // the first block's barriers, and neither leaves before the other)
        if (rank == 0 && lane == 0 && (!ok || *abort_flag))
#pragma unroll 1
            for (uint32_t j = it > (uint32_t)STAGES ? it - (uint32_t)STAGES : 0u; j < it; ++j)
                mbar_wait_quiet(&sh->full[j % (uint32_t)STAGES], (j / (uint32_t)STAGES) & 1u, DRAIN_LIMIT_CLOCKS);
    } else if (warp == TMA_WARP + 1) {
        uint32_t acc = 0, s = 0, ph = 0;
        bool ok = true;
        const uint32_t ring_base = smem_u32(ring);
        const uint64_t astep = g.a_mn ? 2048 >> 4 : 32 >> 4, bstep = g.b_mn ? 2048 >> 4 : 32 >> 4;
        for (Walk t(g, worker); rank == 0 && ok && t.more(); t.next()) {
            const int kbn = t.kbn();
            const uint32_t idesc = g.idesc | (uint32_t)(t.columns() >> 3) << 17;
            for (int kb = 0; ok && kb < kbn; ++acc) {
                const int run_end = RUNS || g.keep ? min(kb + g.run_kb, kbn) : kbn;
                const uint32_t buf = g.keep ? 0u : acc & 1u, use = g.keep ? acc & 1u : (acc >> 1) & 1u;
                if (!(ok = mbar_wait_warp(&sh->t_empty[buf], use ^ 1u, abort_flag))) break;
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + buf * ACC_COLS;
                for (uint32_t first = 0; kb < run_end; ++kb, first = 1) {
                    if (!(ok = mbar_wait_warp(&sh->full[s], ph, abort_flag))) break;
                    tc_fence_after();
                    const uint32_t a = ring_base + s * (uint32_t)STAGE_BYTES, b = a + PARTS * A_BYTES;
                    if constexpr (PARTS == 1) {
                        umma_kblock_elected<F8, PAIR>(d_tmem, operand_desc(a, g.a_mn), operand_desc(b, g.b_mn), astep, bstep, idesc,
                                                first);
                    } else {
                        constexpr int pa[6] = {0, 2, 0, 1, 1, 0}, pb[6] = {0, 0, 2, 1, 0, 1};
#pragma unroll
                        for (int q = 0; q < 6; ++q)
                            umma_kblock_elected<F8, PAIR>(d_tmem + (q == 0 ? 0 : BN), operand_desc(a + pa[q] * A_BYTES, g.a_mn),
                                                    operand_desc(b + pb[q] * B_BYTES, g.b_mn), astep, bstep, idesc,
                                                    q <= 1 ? first : 1u);
                    }
                    commit_elected<PAIR>(&sh->empty[s]);
                    if (++s == (uint32_t)STAGES) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                if (ok) commit_elected<PAIR>(&sh->t_full[buf]);
            }
        }
        if (rank == 0 && __any_sync(FULL, !ok || *abort_flag)) {
            commit_elected<PAIR>(&sh->drain);
            if (lane == 0) mbar_wait_quiet(&sh->drain, 0u, DRAIN_LIMIT_CLOCKS);
        }
    } else {
        const int quad = warp & 3, piece = warp >> 2;   // TMEM lanes 32 quad.. and a piece of the columns are this warp's
        constexpr int COLS = BN * 4 / EPI_WARPS;
        using C = ChunkStore<O, COLS>;
        constexpr int SUBS = COLS / 32;
        static_assert(C::WIDTH == COLS, "a warp's columns leave as one box");
        char *slot = staging + warp * SLOT_BYTES;
        const int m_off = (int)rank * BM + quad * 32;   // this warp's rows in the tile
        const uint32_t t_empty = PAIR ? in_block(smem_u32(&sh->t_empty[0]), 0) : smem_u32(&sh->t_empty[0]);
        auto give_back = [&](uint32_t buf) {   // the accumulator, once every column of it is in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR)
                    arrive_at(t_empty + buf * 8);
                else
                    mbar_arrive(&sh->t_empty[buf]);
            }
        };
        uint32_t acc = 0;
        bool ok = true;
        const bool by_tma = e.tma && !e.share, with_z = e.preact != nullptr;
        const bool scaled = std::is_same_v<O, __half> && e.factor && !e.share;   // (shares are joined first)
        const float factor = scaled ? *e.factor : 1.f;
        // The residual is copied into the slot that the result will leave from, and added in place.
        auto fetch_residual = [&](int64_t row0, int col) {
            constexpr int PER_ROW = C::WIDTH / C::G;
            const int c = lane % PER_ROW;
#pragma unroll
            for (int r = lane / PER_ROW; r < 32; r += 32 / PER_ROW) {
                const int64_t row = row0 + r;
                if (row < e.M && col + c * C::G < e.N)
                    copy_async<16>(slot + C::at(r, c), static_cast<const O *>(e.residual) + row * e.ldr + col + c * C::G);
            }
            copies_end_group();
        };
        for (Walk t(g, worker); ok && t.more(); t.next()) {
            const int col = t.n0() + piece * COLS;
            const int64_t row0 = (int64_t)t.m0() + m_off;   // (below 2^31 where there are rows)
            const bool mine = row0 < e.M && col < e.N;
            // while the sums are on their way: the residual, and bias and scale of this warp's columns, one to a lane
            if (by_tma && e.residual && !with_z && mine) {
                stores_read<0>();
                fetch_residual(row0, col);
            }
            float bias[SUBS], scale[SUBS];
#pragma unroll
            for (int q = 0; q < SUBS; ++q) {
                const int c = col + q * 32 + lane;
                bias[q] = by_tma && e.bias && c < e.N ? load_param(e.bias, e.bias_type, c) : 0.f;
                scale[q] = by_tma && e.w_scale && c < e.N ? e.w_scale[c] : 1.f;
            }
            // The sums, 32 columns at a time: in runs they are in registers, otherwise they are read from TMEM where they are
            // needed (twice where z is stored too: cheaper than keeping them).
            float run[RUNS ? 32 : 1];
            uint32_t buf = 0, taddr = 0;
            if constexpr (RUNS) {
                static_assert(SUBS == 1, "sums in runs are of fp32 outputs");
                const int kbn = t.kbn();
#pragma unroll
                for (int j = 0; j < 32; ++j) run[j] = 0.f;
                for (int kb = 0; kb < kbn; kb += g.run_kb, ++acc) {
                    buf = acc & 1u;
                    if (!(ok = mbar_wait_warp(&sh->t_full[buf], (acc >> 1) & 1u, abort_flag))) break;
                    tc_fence_after();
                    taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + buf * ACC_COLS + piece * COLS;
                    uint32_t a[32];
                    tmem_ld32_issue(taddr, a);
                    tmem_ld_wait(a);
                    if constexpr (PARTS == 3) {
                        uint32_t w[32];
                        tmem_ld32_issue(taddr + BN, w);
                        tmem_ld_wait(w);
#pragma unroll
                        for (int j = 0; j < 32; ++j) run[j] += __uint_as_float(a[j]) + __uint_as_float(w[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) run[j] += __uint_as_float(a[j]);
                    }
                    give_back(buf);
                }
                if (!ok) break;
            } else if (g.keep) {
                const uint32_t from = tmem_base + ((uint32_t)(quad * 32) << 16) + piece * COLS;
                const int kbn = t.kbn();
                taddr = from + ACC_COLS;
                for (int kb = 0; kb < kbn; kb += g.run_kb, ++acc) {
                    if (!(ok = mbar_wait_warp(&sh->t_full[0], acc & 1u, abort_flag))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int q = 0; q < COLS; q += 16) {
                        uint32_t a[16];
                        tmem_ld16(from + q, a);
                        if (kb > 0) {
                            uint32_t w[16];
                            tmem_ld16(taddr + q, w);
#pragma unroll
                            for (int j = 0; j < 16; ++j) a[j] = __float_as_uint(__uint_as_float(a[j]) + __uint_as_float(w[j]));
                        }
                        tmem_st16(taddr + q, a);
                    }
                    tmem_st_wait();
                    give_back(0);
                }
                if (!ok) break;
            } else {
                buf = acc & 1u;
                if (!(ok = mbar_wait_warp(&sh->t_full[buf], (acc >> 1) & 1u, abort_flag))) break;
                ++acc;
                tc_fence_after();
                taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + buf * ACC_COLS + piece * COLS;
            }
            auto sums = [&](int q, float(&v)[32]) {
                if constexpr (RUNS) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = run[j];
                } else {
                    uint32_t a[32];
                    tmem_ld32_issue(taddr + q * 32, a);
                    tmem_ld_wait(a);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(a[j]);
                }
            };
            auto all_read = [&] {
                if (!RUNS && !g.keep) give_back(buf);
            };
            if (!mine) {
                all_read();
                continue;
            }
            if (e.share) {
#pragma unroll 1
                for (int q = 0; q < SUBS && col + q * 32 < e.N; ++q) {
                    float v[32];
                    sums(q, v);
                    stores_read<0>();
                    ChunkStore<float, 32>::write(slot, lane, 0, v);
                    before_stores();
                    tma_store_3d_elected(&map_out, slot, col + q * 32, (int)row0, t.split);
                }
                all_read();
            } else if (by_tma) {
                const float xs = e.x_scale && row0 + lane < e.M ? e.x_scale[row0 + lane] : 0.f;
                auto biased = [&](int q, float(&v)[32]) {
                    sums(q, v);
                    if (scaled) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= factor;
                    }
                    const float s = SUBS > 1 && q == 1 ? scale[SUBS - 1] : scale[0], b = SUBS > 1 && q == 1 ? bias[SUBS - 1] : bias[0];
                    if (e.x_scale) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= xs * __shfl_sync(FULL, s, j);
                    }
                    if (e.bias) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(FULL, b, j);
                    }
                };
                if (with_z) {   // z leaves first, from the same slot
                    stores_read<0>();
#pragma unroll 1
                    for (int q = 0; q < SUBS; ++q) {
                        float v[32];
                        biased(q, v);
                        C::write(slot, lane, q * (32 / C::G), v);
                    }
                    before_stores();
                    tma_store_3d_elected(&map_z, slot, col, (int)row0, 0);
                    if (e.residual) {
                        stores_read<0>();
                        fetch_residual(row0, col);
                    }
                }
#pragma unroll 1
                for (int q = 0; q < SUBS; ++q) {
                    float v[32];
                    biased(q, v);
                    activate(v, e.act);
                    if (q == 0) {   // only now does the slot have to be free, or the residual there
                        if (e.residual) {
                            copies_wait<0>();
                            __syncwarp();
                        } else
                            stores_read<0>();
                    }
                    if (e.residual) C::add(slot, lane, q * (32 / C::G), v);
                    C::write(slot, lane, q * (32 / C::G), v);
                }
                all_read();
                before_stores();
                tma_store_3d_elected(&map_out, slot, col, (int)row0, 0);
            } else {
                float *loose = reinterpret_cast<float *>(slot);
#pragma unroll 1
                for (int q = 0; q < SUBS; ++q) {
                    const int at = col + q * 32;
                    float v[32];
                    sums(q, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) loose[lane * 32 + ((j + lane) & 31)] = scaled ? v[j] * factor : v[j];
                    __syncwarp();
                    if (at + lane < e.N) {
                        LooseRows<O> w{static_cast<O *>(e.out) + row0 * e.N + at + lane, nullptr, nullptr, nullptr, e.ldr, e.N,
                                       (int)min(e.M - row0, (int64_t)32), e.act, 0.f, 1.f, loose};
                        if (e.preact) w.z = static_cast<O *>(e.preact) + row0 * e.N + at + lane;
                        if (e.residual) w.residual = static_cast<const O *>(e.residual) + row0 * e.ldr + at + lane;
                        if (e.bias) w.bias = load_param(e.bias, e.bias_type, at + lane);
                        if (e.x_scale) {
                            w.x_scale = e.x_scale + row0;
                            w.scale = e.w_scale[at + lane];
                        }
                        finish_rows<O>(w);
                    }
                    __syncwarp();
                }
                all_read();
            }
        }
        copies_wait<0>();
        // what has been stored is written before the block ends: the launch that follows may already be waiting for it
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncthreads();
    if constexpr (PAIR) cluster_meet();   // neither block leaves while the other may still signal it
    if (sh->abort && threadIdx.x == 0) ep_raise(status, EP_ERR_TIMEOUT);
    if (warp == 0) {
        tc_fence_after();
        if constexpr (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// The shares of a split sum, then the epilogue: 32 chunks of 8 columns a block, 8 threads to each, which add the shares
// s, s + 8, ... in order; then the eight in order.
// Blocks past those fold the partial sums of dbias, where there are any: 8 columns a block, 32 threads to each (one launch
// less for a backward pass).
struct BiasFold {
    const float *parts;   // [slabs][n_out]; NULL: none
    int slabs, n_out;
    float *dbias;
};
__host__ __device__ constexpr int join_chunks() { return 32; }
template <typename O>
__global__ void __launch_bounds__(256) linear_join(const float *shares, int splits, const Epilogue e, int join_blocks,
                                                   const BiasFold bias) {
    __shared__ __align__(16) float part[8][join_chunks()][9];
    if ((int)blockIdx.x >= join_blocks) {
        const int c = ((int)blockIdx.x - join_blocks) * 8 + (threadIdx.x & 7), r0 = threadIdx.x >> 3;
        double *sums = reinterpret_cast<double *>(part);   // [32][8]
        ep_wait_for_launch_before();
        double t = 0.0;
        if (c < bias.n_out)
            for (int r = r0; r < bias.slabs; r += 32 * 16) {
                float v[16];
#pragma unroll
                for (int q = 0; q < 16; ++q) v[q] = r + 32 * q < bias.slabs ? bias.parts[(size_t)(r + 32 * q) * bias.n_out + c] : 0.f;
#pragma unroll
                for (int q = 0; q < 16; ++q) t += (double)v[q];
            }
        sums[threadIdx.x] = t;
        __syncthreads();
        if (threadIdx.x < 8 && c < bias.n_out) {
#pragma unroll
            for (int q = 1; q < 32; ++q) t += sums[q * 8 + threadIdx.x];
            bias.dbias[c] = (float)t;
        }
        return;
    }
    const int chunks = (e.N + 7) / 8;
    const int64_t total = e.M * chunks, i = (int64_t)blockIdx.x * join_chunks() + (threadIdx.x & 31);
    const int s0 = threadIdx.x >> 5;
    const int64_t row = i / chunks;
    const int col = (int)(i - row * chunks) * 8;
    ep_wait_for_launch_before();
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (i < total) {
        const float *from = shares + ((int64_t)s0 * e.M + row) * e.ld_share + col;
        const int64_t apart = 8 * e.M * e.ld_share;
        for (int s = s0; s < splits; s += 8 * 5, from += 5 * apart) {   // five shares at a time, none alone at the end
            float4 a[5], b[5];
#pragma unroll
            for (int q = 0; q < 5; ++q) {
                const bool there = s + 8 * q < splits;
                a[q] = there ? *reinterpret_cast<const float4 *>(from + q * apart) : make_float4(0.f, 0.f, 0.f, 0.f);
                b[q] = there ? *reinterpret_cast<const float4 *>(from + q * apart + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int q = 0; q < 5; ++q) {
                v[0] += a[q].x, v[1] += a[q].y, v[2] += a[q].z, v[3] += a[q].w;
                v[4] += b[q].x, v[5] += b[q].y, v[6] += b[q].z, v[7] += b[q].w;
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) part[s0][threadIdx.x & 31][q] = v[q];
    __syncthreads();
    if (s0 > 0 || i >= total) return;
#pragma unroll
    for (int s = 1; s < 8; ++s)
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] += part[s][threadIdx.x][q];
    Columns<8> c;
    c.load(e, col);
    float add[8];
    load_residual<O>(e, row, col, add);
    finish<O>(e, row, col, c, v, add);
}

// ---------------------------------------------------------------------------------------------- few rows
// The sum of lane r's row: NaN where it is infinite because a number of that row of x, or of w, is.  (Rare, and kept out of
// the way of what is not: written out in the kernel it made 8 rows of 1024 8 % slower.)
__device__ __noinline__ float nan_of_infinities(float sum, const float *x, int64_t ldx, const float *w, int n_in) {
    const int lane = threadIdx.x & 31;
    for (unsigned left = __ballot_sync(FULL, isinf(sum)); left; left &= left - 1) {
        const int r = __ffs(left) - 1;
        bool infinite = false;
        for (int c = lane; c < n_in; c += 32) infinite |= isinf(x[r * ldx + c]) || isinf(w[c]);
        if (__any_sync(FULL, infinite) && lane == r) sum = CUDART_NAN_F;
    }
    return sum;
}

// Dot products: `share` warps of a block (1, 2, 4 or 8 of its 8) to one column of ROWS rows.  Their lanes share out the row
// of W, in 16-byte chunks (VEC) or, where it is not aligned for that, element by element next to one another; W is read
// once, x comes from the L1.  Sums are fp32 multiply-adds to nearest, so all types are exact to fp32 here.
template <typename T, int ROWS, bool VEC>
__global__ void __launch_bounds__(256) linear_few_rows(const T *__restrict__ x, int64_t ldx, const T *__restrict__ w, int64_t ldw,
                                                       int n_in, const Epilogue e, int share) {
    constexpr int N = VEC ? 16 / (int)sizeof(T) : 1;
    __shared__ float part[8][ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = (int)blockIdx.x * (8 / share) + warp / share, mine = warp % share;
    float sum[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sum[r] = 0.f;
    if (col < e.N) {
        const T *wr = w + col * ldw;
#pragma unroll 4
        for (int c = (mine * 32 + lane) * N; c < n_in; c += share * 32 * N) {
            float a[N];
            load_chunk(wr, c, n_in, VEC, 0.f, a);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (r < e.M) {
                    float b[N];
                    load_chunk(x + r * ldx, c, n_in, VEC, 0.f, b);
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[r] = fmaf(a[i], b[i], sum[r]);
                }
            }
        }
    }
    float v[1] = {0.f};
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) sum[r] += __shfl_xor_sync(FULL, sum[r], o);
        if (lane == r) v[0] = sum[r];
    }
    if (share > 1) {
        if (lane < ROWS) part[warp][lane] = v[0];
        __syncthreads();
        if (mine == 0 && lane < ROWS)
            for (int s = 1; s < share; ++s) v[0] += part[warp + s][lane];
    }
    if constexpr (sizeof(T) == 4) {
        // The tiles split fp32 numbers, and an infinity splits into NaN: so it does here.  A sum is only infinite where an
        // operand is, or where it overflows, which stays an infinity.
        if (col < e.N && mine == 0 && __builtin_expect(__any_sync(FULL, isinf(v[0])), 0))
            v[0] = nan_of_infinities(v[0], x, ldx, w + col * ldw, n_in);
    }
    if (col < e.N && mine == 0 && lane < ROWS && lane < e.M) {
        Columns<1> c;
        c.load(e, col);
        float add[1];
        if (e.out_type == EP_BF16) {
            load_residual<__nv_bfloat16>(e, lane, col, add);
            finish<__nv_bfloat16>(e, lane, col, c, v, add);
        } else if (e.out_type == EP_F16) {
            load_residual<__half>(e, lane, col, add);
            finish<__half>(e, lane, col, c, v, add);
        } else {
            load_residual<float>(e, lane, col, add);
            finish<float>(e, lane, col, c, v, add);
        }
    }
}

// ---------------------------------------------------------------------------------------------- operands
// x = x1 + x2 + x3, each the bf16 nearest to what is left (x1 by truncation: it never overflows to infinity).
__device__ __forceinline__ void split3(float x, __nv_bfloat16 (&p)[3]) {
    const float a = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    p[0] = __float2bfloat16_rn(a);
    const float r = x - a;
    p[1] = __float2bfloat16_rn(r);
    p[2] = __float2bfloat16_rn(r - __bfloat162float(p[1]));
}

// Copies matrices (bound by memory: 84336 x 647 bf16 in 44 us, 5.0 TB/s): rows of `cols` elements `ld` apart to rows ld_to
// apart (a multiple of 16 bytes; the tail is zero).
// PARTS == 3: fp32 to three bf16 matrices, part_stride elements apart.  blockIdx.y chooses one of two matrices.
struct PackJob {
    const void *from;
    void *to;
    int64_t ld, rows, part_stride;
    int cols, ld_to;
};
template <typename T, typename O, int PARTS>
__global__ void __launch_bounds__(256) pack_rows(const PackJob first, const PackJob second) {
    const PackJob &j = blockIdx.y ? second : first;
    const T *from = static_cast<const T *>(j.from), *end = from + (j.rows - 1) * j.ld + j.cols;
    O *to = static_cast<O *>(j.to);
    ep_let_next_launch_start();
    constexpr int N = PARTS == 3 ? 8 : 16 / (int)sizeof(O);   // elements of a thread: 16 bytes of each output
    const int chunks = j.ld_to / N;
    const int64_t total = j.rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = i / chunks;
        const int col = (int)(i - row * chunks) * N;
        T e[N];
        load_elements_anywhere(from + row * j.ld + col, j.cols - col, from, end, e);
        if constexpr (PARTS == 3) {
            __nv_bfloat16 p[8][3];
#pragma unroll
            for (int q = 0; q < 8; ++q) split3(e[q], p[q]);
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                alignas(16) __nv_bfloat16 o[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) o[q] = p[q][k];
                *reinterpret_cast<uint4 *>(to + k * j.part_stride + row * j.ld_to + col) = *reinterpret_cast<const uint4 *>(o);
            }
        } else {
            alignas(16) O o[N];
#pragma unroll
            for (int q = 0; q < N; ++q) o[q] = e[q];
            *reinterpret_cast<uint4 *>(to + row * j.ld_to + col) = *reinterpret_cast<const uint4 *>(o);
        }
    }
}

// fp16 holds nothing below 2^-25 and nothing above 65504, where a mean loss over many rows, or a loss scale, puts whole
// gradients.  So dz that has to be rounded to fp16 is first multiplied by the power of two that brings the largest finite
// |dout| to [2^14, 2^15) (the slopes are below 1.13), and the products' sums by its inverse: elements down to 2^-28 of that
// largest keep fp16's 11 bits, what is lost of smaller ones is below 2^-39 of it.  dout is read once more for it (232965 x 256
// fp16: 24 us of 179).  Each block leaves its largest; the blocks of linear_dz take the largest of those.
constexpr int PEAK_BLOCKS_PER_SM = 4;
template <typename D>
__global__ void __launch_bounds__(256) linear_peaks(const D *__restrict__ dout, int64_t total, float *__restrict__ peaks) {
    __shared__ float tops[8];
    constexpr int N = 16 / (int)sizeof(D), Q = 4;   // Q 16-byte chunks in flight
    float top = 0.f;
    auto look = [&](D v) {
        const float size = fabsf(to_f32(v));
        top = fmaxf(top, size < INFINITY ? size : 0.f);
    };
    // the elements before the first 16-byte boundary and after the last whole chunk are the last block's
    const int64_t before = min((int64_t)((16 - (reinterpret_cast<uintptr_t>(dout) & 15)) & 15) / (int)sizeof(D), total);
    const int64_t chunks = (total - before) / N, step = (int64_t)gridDim.x * 256;
    const uint4 *from = reinterpret_cast<const uint4 *>(dout + before);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += Q * step) {
        alignas(16) D e[Q][N];
#pragma unroll
        for (int q = 0; q < Q; ++q) *reinterpret_cast<uint4 *>(e[q]) = i + q * step < chunks ? from[i + q * step] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int c = 0; c < N; ++c) look(e[q][c]);
    }
    if (blockIdx.x == gridDim.x - 1) {
        if (threadIdx.x < before) look(dout[threadIdx.x]);
        const int64_t rest = before + chunks * N + threadIdx.x;
        if (rest < total) look(dout[rest]);
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < 8; ++w) top = fmaxf(top, tops[w]);
        peaks[blockIdx.x] = top;
    }
}
struct Peaks {   // NULL: dz is written as it is
    float *each;
    int n;
    float *factor;   // out: the inverse of the power of two
};

// dz = dout act'(z), written for the products (16 bits as they are, fp32 as three bf16 parts; rows ld_to apart, zero
// beyond N), and the sums of its columns over this block's rows: part[blockIdx.y][N].  One rounding of dz to the operands'
// 16 bits, because the tensor core takes nothing wider beside them: it makes the products' error 1.4 times what rounding
// them alone leaves (0.0023 for 0.0017 of bf16), and two parts would move ten bytes for seven.  232965 x 256 bf16 through
// GELU: 62 us, 5.8 TB/s, with instruction issue close behind (25 an element).
constexpr int DZ_CHUNKS = 16, DZ_ROWS = 16;   // a block covers 128 columns, 16 rows at a time
constexpr int DZ_THREADS = DZ_CHUNKS * DZ_ROWS;
constexpr int DZ_STAGES = 4;                  // rows in flight per thread and one more (see the ring in rows.cuh)
template <typename T, typename D>
constexpr int dz_pieces() { return (8 * (int)(sizeof(T) + sizeof(D))) / 16; }   // 16-byte pieces of 8 elements of dout and z
template <typename T, typename D, int PARTS>
__global__ void __launch_bounds__(DZ_THREADS) linear_dz(const D *__restrict__ dout, const T *__restrict__ z, int act, int64_t rows,
                                                        int n_out, void *to_raw, int ld_to, int64_t part_stride,
                                                        float *__restrict__ part, bool vec, const Peaks peaks) {
    constexpr int D_PIECES = 8 * (int)sizeof(D) / 16, Z_PIECES = 8 * (int)sizeof(T) / 16;
    __shared__ float fold[DZ_ROWS][DZ_CHUNKS * 8];
    extern __shared__ uint4 ring[];   // [DZ_STAGES][D_PIECES + Z_PIECES][DZ_THREADS], where vec
    const int cx = threadIdx.x % DZ_CHUNKS, r0 = threadIdx.x / DZ_CHUNKS;
    const int col = (blockIdx.x * DZ_CHUNKS + cx) * 8;
    // all blocks go over the rows side by side, so that what is written last lies together (see GemmShape::backwards)
    const int64_t begin = (int64_t)blockIdx.y * DZ_ROWS, step = (int64_t)gridDim.y * DZ_ROWS;
    ep_let_next_launch_start();
    float scale = 1.f;
    if constexpr (std::is_same_v<T, __half>) {
        if (peaks.each) {
            float top = 0.f;
            for (int i = threadIdx.x; i < peaks.n; i += DZ_THREADS) top = fmaxf(top, peaks.each[i]);
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
            if ((threadIdx.x & 31) == 0) fold[0][threadIdx.x >> 5] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < DZ_THREADS / 32; ++w) top = fmaxf(top, fold[0][w]);
            __syncthreads();   // (fold is used again)
            const int up = top > 0.f ? min(14 - ilogbf(top), 126) : 0;
            scale = scalbnf(1.f, up);
            if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *peaks.factor = scalbnf(1.f, -up);
        }
    }
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    auto work = [&](int64_t row, float(&v)[8], const float(&zz)[8]) {
        if (act != EP_ACT_NONE) times_slope(v, zz, act);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];   // (zero past the row's end: dout reads as zero there)
        if (!to_raw) return;
        if constexpr (PARTS == 3) {
            __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(to_raw) + row * ld_to + col;
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
        } else {
            if constexpr (std::is_same_v<T, __half>) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= scale;
            }
            store_chunk(static_cast<T *>(to_raw) + row * ld_to, col, ld_to, true, v);
        }
    };
    if (vec) {
        auto slot = [&](int s) { return ring + (size_t)s * (D_PIECES + Z_PIECES) * DZ_THREADS + threadIdx.x; };
        auto fetch = [&](int64_t row, int s) {
            if (row < rows && col < n_out) {
                uint4 *to = slot(s);
#pragma unroll
                for (int p = 0; p < D_PIECES; ++p) copy_async<16>(to + p * DZ_THREADS, reinterpret_cast<const uint4 *>(dout + row * n_out + col) + p);
                if (act != EP_ACT_NONE)
#pragma unroll
                    for (int p = 0; p < Z_PIECES; ++p)
                        copy_async<16>(to + (D_PIECES + p) * DZ_THREADS, reinterpret_cast<const uint4 *>(z + row * n_out + col) + p);
            }
            copies_end_group();
        };
        int64_t ahead = begin + r0;
#pragma unroll
        for (int s = 0; s < DZ_STAGES - 1; ++s, ahead += step) fetch(ahead, s);
        int s = 0;
        for (int64_t row = begin + r0; row < rows; row += step, ahead += step) {
            fetch(ahead, s == 0 ? DZ_STAGES - 1 : s - 1);   // into the slots of the row before
            copies_wait<DZ_STAGES - 1>();
            if (col < n_out) {   // (whole chunks: rows of ld_to and of n_out elements end at the same one)
                float v[8], zz[8];
                const uint4 *from = slot(s);
                auto held = [&](auto type, int at, float(&to)[8]) {
                    using E = decltype(type);
                    alignas(16) E e[8];
#pragma unroll
                    for (int p = 0; p < 8 * (int)sizeof(E) / 16; ++p) reinterpret_cast<uint4 *>(e)[p] = from[(at + p) * DZ_THREADS];
#pragma unroll
                    for (int i = 0; i < 8; ++i) to[i] = to_f32(e[i]);
                };
                held(D{}, 0, v);
                if (act != EP_ACT_NONE) held(T{}, D_PIECES, zz);
                work(row, v, zz);
            }
            s = s + 1 == DZ_STAGES ? 0 : s + 1;
        }
        copies_wait<0>();
    } else if (col < ld_to) {
        for (int64_t row = begin + r0; row < rows; row += step) {
            float v[8], zz[8];
            D d[8];
            load_elements_anywhere(dout + row * n_out + col, n_out - col, dout, dout + rows * n_out, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_f32(d[i]);
            if (act != EP_ACT_NONE) {
                T q[8];
                load_elements_anywhere(z + row * n_out + col, n_out - col, z, z + rows * n_out, q);
#pragma unroll
                for (int i = 0; i < 8; ++i) zz[i] = to_f32(q[i]);
            }
            work(row, v, zz);
        }
    }
    if (!part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) fold[r0][cx * 8 + i] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < DZ_CHUNKS * 8; c += DZ_THREADS) {
        const int to = blockIdx.x * DZ_CHUNKS * 8 + c;
        if (to >= n_out) continue;
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < DZ_ROWS; ++q) t += fold[q][c];
        part[(size_t)blockIdx.y * n_out + to] = t;
    }
}

// ---------------------------------------------------------------------------------------------- host side
constexpr int MAX_WIDTH = 65536;
// Whether the dot products serve rows x n_in -> n_out, and not the tiles.  They go by the CUDA cores, about 4 products a
// picosecond: up to 2^24 products they are the faster ones (1024 x 1024 bf16: 8 rows in 4.8 us against 6.0; 4096 x 4096:
// 1 row 6.9 against 10.0, 2 rows 12.3 against 10.0).  fp32 operands would first have to be split (4096 x 4096: 8 rows
// 38 us against 76), so there they serve every call of up to 8 rows.
constexpr int FEW_ROWS = 8;
bool few_rows(int64_t rows, int n_in, int n_out, int type) {
    return rows <= FEW_ROWS && (type == EP_F32 || rows * n_in * n_out <= (1ll << 24));
}
constexpr int PACK_BLOCKS_PER_SM = 8;

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// An operand as the tile kernel reads it: `parts` matrices [rows][cols], rows ld elements apart.
struct Operand {
    const void *base;
    int type;             // EP_BF16, EP_F16 or EP_E4M3
    int64_t rows;
    int cols;
    int64_t ld;
    int parts;
    int64_t part_stride;
};

// A tile of the operand is 128 bytes of k (K-major) or 64 of its columns x 64 k (MN-major) by box_rows rows.
bool encode_operand(CUtensorMap *map, const Operand &o, bool mn, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t size = (cuuint64_t)ep::type_size(o.type);
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.parts};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * size, (cuuint64_t)(o.parts > 1 ? o.part_stride : o.ld * o.rows) * size};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / size), (cuuint32_t)(mn ? 64 : box_rows), 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUtensorMapDataType type = o.type == EP_BF16  ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                     : o.type == EP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_UINT8;
    return fn(map, type, 3, const_cast<void *>(o.base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// A matrix [depth][rows][cols] as a warp of the tile kernel writes it: boxes of 32 rows of 128 bytes
// (64 bytes where a warp has only 32 columns of 16 bits).
bool encode_result(CUtensorMap *map, void *base, int type, int64_t depth, int64_t rows, int cols, int64_t ld, int bn) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t size = (cuuint64_t)ep::type_size(type);
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * size, (cuuint64_t)(ld * rows) * size};
    const cuuint32_t width = (cuuint32_t)std::min<int64_t>(128 / (int64_t)size, bn == 256 ? 64 : 32);
    const cuuint32_t box[3] = {width, 32, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUtensorMapDataType t = type == EP_BF16  ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                  : type == EP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                   : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    return fn(map, t, 3, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              width * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct GemmPlan {
    int bn, splits, workers;
    bool runs, pair;
    int ld_share;
    GemmShape shape;
    size_t share_bytes(int64_t M) const { return splits > 1 ? sizeof(float) * (size_t)splits * (size_t)M * (size_t)ld_share : 0; }
};

// Tile and split of the sum, by the clocks that a launch would take.  A k-block costs the longer of its MMAs (128 x bn x
// 64 products at 4096 a clock and SM) and its operands' bytes (64 a clock and SM from the L2); a tile's end 20 clocks a
// column and 1000 more; the join of a split sum 5000 and its shares' bytes (3400 a clock).  The sum is only split while
// the tiles leave workers idle, into shares of at least 4 k-blocks.  (With the largest tile that fills one wave instead,
// the weights' gradient of 232965 x 256 x 256 went by tiles of 64 columns that read each operand up to four times.)
GemmPlan plan_gemm(const ep_ctx *ctx, int64_t M, int N, int64_t K, int type, int out_type) {
    const int ke = type == EP_E4M3 ? 128 : 64, parts = type == EP_F32 ? 3 : 1;
    const bool fp32_out = out_type == EP_F32;
    const int kb = (int)ep::ceil_div(K, ke);
    GemmPlan best{};
    double best_cost = 0.0;
    for (int pair = 0; pair <= 1; ++pair)
        for (int bn : {256, 128, 64}) {
            if (bn == (pair ? 64 : 256) || (fp32_out && bn != (parts == 3 && !pair ? 64 : 128))) continue;
            GemmPlan p{};
            p.runs = fp32_out;
            p.pair = pair;
            p.bn = bn;
            p.shape.M = M;
            p.shape.N = N;
            p.shape.kb = kb;
            p.shape.tiles_n = (int)ep::ceil_div(N, bn);
            p.shape.tiles_m = (int)ep::ceil_div(M, pair ? 2 * BM : BM);
            p.shape.tiles = (int64_t)p.shape.tiles_m * p.shape.tiles_n;
            const int workers = pair ? ctx->sm_count / 2 : ctx->sm_count;
            p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(workers / p.shape.tiles, kb / 4));
            const int per = (int)ep::ceil_div(kb, p.splits);
            p.shape.splits = p.splits;
            p.shape.run_kb = fp32_out ? RUN_KB : through_kb(out_type);
            p.shape.keep = !fp32_out && per > p.shape.run_kb;
            p.shape.items = p.shape.tiles * p.splits;
            p.workers = (int)std::min<int64_t>(p.shape.items, workers);
            p.shape.step_m = p.workers / p.shape.tiles_n;
            p.shape.step_n = p.workers % p.shape.tiles_n;
            p.ld_share = (int)round_up(N, 8);
            const double mma = (parts == 3 ? 6 : 1) * 2.0 * bn;
            const double load = parts * (16384.0 + 128.0 * (pair ? bn / 2 : bn)) / 64.0;
            const double item = per * std::max(mma, load) + 20.0 * bn + 1000.0;
            const double cost = ep::ceil_div(p.shape.items, p.workers) * item +
                                (p.splits > 1 ? 5000.0 + p.share_bytes(M) / 3400.0 : 0.0);
            if (!best.bn || cost < best_cost) {
                best_cost = cost;
                best = p;
            }
        }
    return best;
}

struct Maps {
    CUtensorMap a, b, out, z;   // out: of the shares, where the sum is split
};

template <int BN, bool F8, int PARTS, bool RUNS, bool PAIR, typename O>
int launch_tiles(ep_ctx *ctx, const GemmPlan &p, const Maps &m, const Epilogue &e, cudaStream_t stream) {
    auto kernel = linear_tiles<BN, F8, PARTS, RUNS, PAIR, O>;
    constexpr size_t smem = TileMemory<BN, PARTS, PAIR>::TOTAL;
    EP_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(PAIR ? 2 * p.workers : p.workers));
    cfg.blockDim = dim3(TileMemory<BN, PARTS, PAIR>::THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2] = {};
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = 2;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = PAIR ? 2 : 1;
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    EP_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, m.a, m.b, m.out, m.z, p.shape, e, ctx->d_status));
    return EP_OK;
}

// (the type of the output is fp32 exactly where sums are kept in runs)
template <bool F8, typename O>
int launch_width(ep_ctx *ctx, const GemmPlan &p, const Maps &m, const Epilogue &e, cudaStream_t stream) {
    if (p.pair)
        return p.bn == 256 ? launch_tiles<256, F8, 1, false, true, O>(ctx, p, m, e, stream)
                           : launch_tiles<128, F8, 1, false, true, O>(ctx, p, m, e, stream);
    return p.bn == 128 ? launch_tiles<128, F8, 1, false, false, O>(ctx, p, m, e, stream)
                       : launch_tiles<64, F8, 1, false, false, O>(ctx, p, m, e, stream);
}
template <bool F8>
int launch_type(ep_ctx *ctx, const GemmPlan &p, const Maps &m, const Epilogue &e, cudaStream_t stream) {
    if (p.runs)
        return p.pair ? launch_tiles<128, F8, 1, true, true, float>(ctx, p, m, e, stream)
                      : launch_tiles<128, F8, 1, true, false, float>(ctx, p, m, e, stream);
    return e.out_type == EP_BF16 ? launch_width<F8, __nv_bfloat16>(ctx, p, m, e, stream) : launch_width<F8, __half>(ctx, p, m, e, stream);
}

// D = A B^T by tiles, with the epilogue; `share` is room for the shares of a split sum.  Adds to *kernels.
// bias: sums to fold in the joining launch; without one (*folded stays false) that is left to the caller.
int run_gemm(ep_ctx *ctx, GemmPlan p, const Operand &a, bool a_mn, const Operand &b, bool b_mn, Epilogue e, float *share,
             cudaStream_t stream, int *kernels, const BiasFold &bias = BiasFold{}, bool *folded = nullptr) {
    const uint32_t fmt = a.type == EP_BF16 ? 1u : 0u;   // f16 and e4m3 are both format 0 of their kinds
    p.shape.a_mn = a_mn;
    p.shape.b_mn = b_mn;
    p.shape.idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
                    ((uint32_t)((p.pair ? 2 * BM : BM) >> 4) << 24);
    e.share = p.splits > 1 ? share : nullptr;
    e.ld_share = p.ld_share;
    Maps m{};
    bool ok = encode_operand(&m.a, a, a_mn, BM) && encode_operand(&m.b, b, b_mn, p.pair ? p.bn / 2 : p.bn);
    if (e.share)
        ok = ok && encode_result(&m.out, share, EP_F32, p.splits, e.M, p.ld_share, p.ld_share, p.bn);
    else if (e.tma)
        ok = ok && encode_result(&m.out, e.out, e.out_type, 1, e.M, e.N, e.N, p.bn) &&
             (!e.preact || encode_result(&m.z, e.preact, e.out_type, 1, e.M, e.N, e.N, p.bn));
    if (!ok) return ep::fail(ctx, EP_ERR_CUDA, "cuTensorMapEncodeTiled failed for a product of %lld x %d", (long long)e.M, e.N);
    int rc;
    if (a.parts == 3)
        rc = p.pair ? launch_tiles<128, false, 3, true, true, float>(ctx, p, m, e, stream)
                    : launch_tiles<64, false, 3, true, false, float>(ctx, p, m, e, stream);
    else
        rc = a.type == EP_E4M3 ? launch_type<true>(ctx, p, m, e, stream) : launch_type<false>(ctx, p, m, e, stream);
    if (rc != EP_OK) return rc;
    ++*kernels;
    if (p.splits > 1) {
        // (a split sum has at most as many tiles as there are SMs: the grid is far below its limit)
        const int blocks = (int)ep::ceil_div(e.M * ((e.N + 7) / 8), join_chunks());
        const unsigned grid = (unsigned)(blocks + (bias.parts ? ep::ceil_div(bias.n_out, 8) : 0));
        if (folded) *folded = bias.parts != nullptr;
        if (e.out_type == EP_BF16)
            EP_CUDA(ctx, ep::launch_early(linear_join<__nv_bfloat16>, dim3(grid), dim3(256), 0, stream, (const float *)share, p.splits, e, blocks, bias));
        else if (e.out_type == EP_F16)
            EP_CUDA(ctx, ep::launch_early(linear_join<__half>, dim3(grid), dim3(256), 0, stream, (const float *)share, p.splits, e, blocks, bias));
        else
            EP_CUDA(ctx, ep::launch_early(linear_join<float>, dim3(grid), dim3(256), 0, stream, (const float *)share, p.splits, e, blocks, bias));
        ++*kernels;
    }
    return EP_OK;
}

bool tma_ready(const void *p, int64_t ld, int type) { return ep::aligned(p, 16) && ld * ep::type_size(type) % 16 == 0; }

// The copy of an operand that TMA can read: fp32 always (three bf16 parts), others when unaligned.
struct Packed {
    int ld, parts, type;
    int64_t part_stride;
    size_t bytes;
};
Packed packed_form(int64_t rows, int cols, int type) {
    Packed p;
    p.parts = type == EP_F32 ? 3 : 1;
    p.type = type == EP_F32 ? EP_BF16 : type;
    p.ld = (int)round_up(cols, type == EP_E4M3 ? 16 : 8);
    p.part_stride = rows * p.ld;
    p.bytes = (size_t)p.parts * (size_t)p.part_stride * (size_t)ep::type_size(p.type);
    return p;
}

struct Matrix {
    const void *base;   // NULL: not wanted
    int64_t ld, rows;
    int cols;
    void *room;         // for its copy
};
// Two matrices as operands, copied first (in one launch) where they have to be.
int make_operands(ep_ctx *ctx, const Matrix &first, const Matrix &second, int type, bool needs_copy, cudaStream_t stream,
                  Operand *a, Operand *b, int *kernels) {
    auto operand = [&](const Matrix &m) {
        if (!needs_copy) return Operand{m.base, type, m.rows, m.cols, m.ld, 1, 0};
        const Packed p = packed_form(m.rows, m.cols, type);
        return Operand{m.room, p.type, m.rows, m.cols, p.ld, p.parts, p.part_stride};
    };
    *a = operand(first);
    *b = operand(second);
    if (!needs_copy) return EP_OK;
    auto job = [&](const Matrix &m) {
        const Packed p = packed_form(m.rows, m.cols, type);
        return PackJob{m.base, m.room, m.ld, m.base ? m.rows : 0, p.part_stride, m.cols, p.ld};
    };
    const PackJob x = job(first), w = job(second);
    const int64_t threads = std::max(x.rows * (x.ld_to / 8), w.rows * (w.ld_to / 8));
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>(ep::ceil_div(threads, 256), (int64_t)ctx->sm_count * PACK_BLOCKS_PER_SM)), 2);
    if (type == EP_F32)
        pack_rows<float, __nv_bfloat16, 3><<<grid, 256, 0, stream>>>(x, w);
    else if (type == EP_E4M3)
        pack_rows<uint8_t, uint8_t, 1><<<grid, 256, 0, stream>>>(x, w);
    else
        pack_rows<uint16_t, uint16_t, 1><<<grid, 256, 0, stream>>>(x, w);
    EP_CUDA(ctx, cudaGetLastError());
    ++*kernels;
    return EP_OK;
}

bool linear_shape_ok(int64_t rows, int n_in, int n_out) {
    return rows >= 0 && rows <= (1ll << 31) - 256 && n_in >= 1 && n_in <= MAX_WIDTH && n_out >= 1 && n_out <= MAX_WIDTH;
}
bool linear_types_ok(int in_type, int out_type) {
    if (in_type == EP_E4M3) return ep::float_type(out_type);
    return ep::float_type(in_type) && (out_type == in_type || out_type == EP_F32);
}

struct LinearWorkspace {
    void *x, *w;
    float *share;
    GemmPlan plan;
    size_t bytes;
};
LinearWorkspace linear_workspace(const ep_ctx *ctx, int64_t rows, int n_in, int n_out, int in_type, int out_type, bool aligned,
                                 void *base) {
    ep::Arena a(base);
    LinearWorkspace w{};
    if (!few_rows(rows, n_in, n_out, in_type)) {
        const bool copy = in_type == EP_F32 || !aligned;
        if (copy) {
            w.x = a.take<char>(packed_form(rows, n_in, in_type).bytes);
            w.w = a.take<char>(packed_form(n_out, n_in, in_type).bytes);
        }
        w.plan = plan_gemm(ctx, rows, n_out, n_in, in_type, out_type);
        w.share = a.take<float>(w.plan.share_bytes(rows) / sizeof(float));
    }
    w.bytes = std::max<size_t>(a.used, 256);
    return w;
}

struct BackwardWorkspace {
    void *dz, *x, *w;
    float *dbias_parts, *share;
    Peaks peaks;   // of fp16 alone
    GemmPlan dx, dw;
    Packed dz_form;
    int slabs;   // blocks that share out the rows in linear_dz
    size_t bytes;
};
BackwardWorkspace backward_workspace(const ep_ctx *ctx, int64_t rows, int n_in, int n_out, int in_type, bool aligned, void *base) {
    ep::Arena a(base);
    BackwardWorkspace w{};
    const bool copy = in_type == EP_F32 || !aligned;
    w.dz_form = packed_form(rows, n_out, in_type);
    w.dz = a.take<char>(w.dz_form.bytes);
    if (copy) {
        w.x = a.take<char>(packed_form(rows, n_in, in_type).bytes);
        w.w = a.take<char>(packed_form(n_out, n_in, in_type).bytes);
    }
    const int across = (int)ep::ceil_div(w.dz_form.ld, DZ_CHUNKS * 8);
    const int64_t want = std::max<int64_t>(1, (int64_t)ctx->sm_count * 4 / across);   // about what stays resident
    w.slabs = (int)std::max<int64_t>(1, std::min<int64_t>(want, ep::ceil_div(rows, 2 * DZ_ROWS)));
    w.dbias_parts = a.take<float>((size_t)w.slabs * n_out);
    if (in_type == EP_F16) {
        w.peaks.n = (int)std::max<int64_t>(1, std::min<int64_t>(ep::ceil_div(rows * n_out, 256 * 16), (int64_t)ctx->sm_count * PEAK_BLOCKS_PER_SM));
        w.peaks.each = a.take<float>(w.peaks.n + 1);
        w.peaks.factor = w.peaks.each ? w.peaks.each + w.peaks.n : nullptr;
    }
    w.dx = plan_gemm(ctx, std::max<int64_t>(rows, 1), n_in, n_out, in_type, in_type);
    w.dw = plan_gemm(ctx, n_out, n_in, std::max<int64_t>(rows, 1), in_type, in_type);
    w.share = a.take<float>(std::max(w.dx.share_bytes(rows), w.dw.share_bytes(n_out)) / sizeof(float));
    w.bytes = std::max<size_t>(a.used, 256);
    return w;
}

// As many warps to a column as the columns leave idle (about 2 blocks an SM), and no more than have a chunk each.
template <int ROWS, typename T>
int launch_few_rows_of(ep_ctx *ctx, const void *x, int64_t ldx, const void *w, int64_t ldw, int n_in, const Epilogue &e, bool vec,
                       cudaStream_t stream) {
    const int per_pass = 32 * (vec ? 16 / (int)sizeof(T) : 1);
    int share = 1;
    while (share < 8 && (int64_t)e.N * share * 2 <= (int64_t)ctx->sm_count * 16 && n_in > share * per_pass) share *= 2;
    const int grid = (int)ep::ceil_div(e.N, 8 / share);
    if (vec)
        linear_few_rows<T, ROWS, true><<<grid, 256, 0, stream>>>((const T *)x, ldx, (const T *)w, ldw, n_in, e, share);
    else
        linear_few_rows<T, ROWS, false><<<grid, 256, 0, stream>>>((const T *)x, ldx, (const T *)w, ldw, n_in, e, share);
    EP_CUDA(ctx, cudaGetLastError());
    return EP_OK;
}
template <int ROWS>
int launch_few_rows(ep_ctx *ctx, const void *x, int64_t ldx, const void *w, int64_t ldw, int in_type, int n_in, const Epilogue &e,
                    bool vec, cudaStream_t stream) {
    if (in_type == EP_F32) return launch_few_rows_of<ROWS, float>(ctx, x, ldx, w, ldw, n_in, e, vec, stream);
    if (in_type == EP_BF16) return launch_few_rows_of<ROWS, __nv_bfloat16>(ctx, x, ldx, w, ldw, n_in, e, vec, stream);
    if (in_type == EP_F16) return launch_few_rows_of<ROWS, __half>(ctx, x, ldx, w, ldw, n_in, e, vec, stream);
    return launch_few_rows_of<ROWS, e4m3>(ctx, x, ldx, w, ldw, n_in, e, vec, stream);
}

template <typename T, typename D, int PARTS>
void launch_dz(const BackwardWorkspace &w, const void *dout, const void *z, int act, int64_t rows, int n_out, bool write, bool sum,
               bool vec, bool scaled, cudaStream_t stream) {
    if (scaled) linear_peaks<D><<<w.peaks.n, 256, 0, stream>>>((const D *)dout, rows * n_out, w.peaks.each);
    const dim3 grid((unsigned)ep::ceil_div(w.dz_form.ld, DZ_CHUNKS * 8), (unsigned)w.slabs);
    const size_t smem = vec ? (size_t)DZ_STAGES * dz_pieces<T, D>() * DZ_THREADS * 16 : 0;
    cudaFuncSetAttribute(linear_dz<T, D, PARTS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         DZ_STAGES * dz_pieces<T, D>() * DZ_THREADS * 16);
    linear_dz<T, D, PARTS><<<grid, DZ_THREADS, smem, stream>>>((const D *)dout, (const T *)z, act, rows, n_out,
                                                                     write ? w.dz : nullptr, w.dz_form.ld, w.dz_form.part_stride,
                                                                     sum ? w.dbias_parts : nullptr, vec, scaled ? w.peaks : Peaks{});
}

int linear_run(ep_ctx *ctx, const LinearWorkspace &ws, const void *x, int64_t ldx, const void *w, int64_t ldw, int in_type,
               int64_t rows, int n_in, int n_out, bool aligned, const Epilogue &e, cudaStream_t stream, int *kernels) {
    if (few_rows(rows, n_in, n_out, in_type)) {
        const int n = 16 / ep::type_size(in_type);
        const bool vec = aligned && n_in % n == 0;
        ++*kernels;
        if (rows == 1) return launch_few_rows<1>(ctx, x, ldx, w, ldw, in_type, n_in, e, vec, stream);
        if (rows == 2) return launch_few_rows<2>(ctx, x, ldx, w, ldw, in_type, n_in, e, vec, stream);
        if (rows <= 4) return launch_few_rows<4>(ctx, x, ldx, w, ldw, in_type, n_in, e, vec, stream);
        return launch_few_rows<8>(ctx, x, ldx, w, ldw, in_type, n_in, e, vec, stream);
    }
    const bool copy = in_type == EP_F32 || !aligned;
    Operand a, b;
    int rc = make_operands(ctx, Matrix{x, ldx, rows, n_in, ws.x}, Matrix{w, ldw, n_out, n_in, ws.w}, in_type, copy, stream, &a, &b,
                           kernels);
    if (rc == EP_OK) rc = run_gemm(ctx, ws.plan, a, false, b, false, e, ws.share, stream, kernels);
    return rc;
}

int linear_backward_run(ep_ctx *ctx, const BackwardWorkspace &ws, const void *dout, int dout_type, const void *preact, int act,
                        const void *x, int64_t ldx, const void *w, int64_t ldw, int in_type, int64_t rows, int n_in, int n_out,
                        bool aligned, void *dx, void *dweight, float *dbias, cudaStream_t stream, int *kernels) {
    const bool copy = in_type == EP_F32 || !aligned;
    const bool direct = act == EP_ACT_NONE && dout_type == in_type && !copy && tma_ready(dout, n_out, in_type);
    const bool write = !direct && (dx || dweight);
    const bool scaled = write && in_type == EP_F16 && (act != EP_ACT_NONE || dout_type != EP_F16);   // (dz is rounded)
    if (write || dbias) {
        const bool vec = n_out % 8 == 0 && ep::aligned(dout, 16) && ep::aligned(preact, 16);
        if (in_type == EP_F32)
            launch_dz<float, float, 3>(ws, dout, preact, act, rows, n_out, write, dbias, vec, scaled, stream);
        else if (in_type == EP_BF16 && dout_type == EP_BF16)
            launch_dz<__nv_bfloat16, __nv_bfloat16, 1>(ws, dout, preact, act, rows, n_out, write, dbias, vec, scaled, stream);
        else if (in_type == EP_BF16)
            launch_dz<__nv_bfloat16, float, 1>(ws, dout, preact, act, rows, n_out, write, dbias, vec, scaled, stream);
        else if (dout_type == EP_F16)
            launch_dz<__half, __half, 1>(ws, dout, preact, act, rows, n_out, write, dbias, vec, scaled, stream);
        else
            launch_dz<__half, float, 1>(ws, dout, preact, act, rows, n_out, write, dbias, vec, scaled, stream);
        EP_CUDA(ctx, cudaGetLastError());
        *kernels += scaled ? 2 : 1;
    }
    Operand dz;
    if (direct)
        dz = Operand{dout, in_type, rows, n_out, n_out, 1, 0};
    else
        dz = Operand{ws.dz, ws.dz_form.type, rows, n_out, ws.dz_form.ld, ws.dz_form.parts, ws.dz_form.part_stride};
    Epilogue e{};
    e.out_type = in_type;
    e.bias_type = EP_F32;
    e.factor = scaled ? ws.peaks.factor : nullptr;
    Operand xs{}, wt{};
    int rc = EP_OK;
    bool folded = false;
    if (dx || dweight)
        rc = make_operands(ctx, Matrix{dweight ? x : nullptr, ldx, rows, n_in, ws.x}, Matrix{dx ? w : nullptr, ldw, n_out, n_in, ws.w},
                           in_type, copy, stream, &xs, &wt, kernels);
    if (rc != EP_OK) return rc;
    if (dx) {
        e.out = dx;
        e.M = rows;
        e.N = n_in;
        e.vec = n_in % 8 == 0 && ep::aligned(dx, 16);
        e.tma = tma_ready(dx, n_in, in_type);
        GemmPlan back = ws.dx;
        back.shape.backwards = true;
        rc = run_gemm(ctx, back, dz, false, wt, true, e, ws.share, stream, kernels);
        if (rc != EP_OK) return rc;
    }
    if (dweight) {
        e.out = dweight;
        e.M = n_out;
        e.N = n_in;
        e.vec = n_in % 8 == 0 && ep::aligned(dweight, 16);
        e.tma = tma_ready(dweight, n_in, in_type);
        rc = run_gemm(ctx, ws.dw, dz, true, xs, true, e, ws.share, stream, kernels,
                      dbias ? BiasFold{ws.dbias_parts, ws.slabs, n_out, dbias} : BiasFold{}, &folded);
        if (rc != EP_OK) return rc;
    }
    if (dbias && !folded) {
        rc = ep::sum_partials(ctx, ws.dbias_parts, ws.slabs, n_out, dbias, stream);
        if (rc != EP_OK) return rc;
        ++*kernels;
    }
    return EP_OK;
}

}  // namespace

using namespace ep;

namespace {
bool type_aligned(const void *p, int type) { return !p || aligned(p, (size_t)type_size(type)); }
}  // namespace

extern "C" {

size_t ep_linear_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t n_in, int32_t n_out, int32_t in_type,
                                 int32_t out_type, int32_t is_aligned) {
    if (!ctx || !linear_shape_ok(rows, n_in, n_out) || !linear_types_ok(in_type, out_type)) return 0;
    return linear_workspace(ctx, rows, n_in, n_out, in_type, out_type, is_aligned != 0, nullptr).bytes;
}

int ep_linear(ep_ctx *ctx, const void *x, int64_t ldx, const void *w, int64_t ldw, int32_t in_type, const float *x_scale,
              const float *w_scale, const void *bias, int32_t bias_type, int32_t act, const void *residual, int64_t ldr,
              void *out, int32_t out_type, void *preact, int64_t rows, int32_t n_in, int32_t n_out, void *workspace,
              size_t workspace_bytes, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (!linear_shape_ok(rows, n_in, n_out))
        return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld, n_in %d or n_out %d out of range", (long long)rows, n_in, n_out);
    if (!linear_types_ok(in_type, out_type) || (bias && !float_type(bias_type)))
        return fail(ctx, EP_ERR_INVALID_ARG, "no product of type %d with output of type %d", in_type, out_type);
    if (act < EP_ACT_NONE || act > EP_ACT_SILU) return fail(ctx, EP_ERR_INVALID_ARG, "unknown activation %d", act);
    if (ldx < n_in || ldw < n_in || (residual && ldr < n_out)) return fail(ctx, EP_ERR_INVALID_ARG, "a row stride is shorter than its row");
    if (rows == 0) return EP_OK;
    if ((in_type == EP_E4M3) != (x_scale != nullptr) || (in_type == EP_E4M3) != (w_scale != nullptr))
        return fail(ctx, EP_ERR_INVALID_ARG, "scales go with 8-bit inputs, and with no others");
    if (!x || !w || !out || !type_aligned(x, in_type) || !type_aligned(w, in_type) || !type_aligned(out, out_type) ||
        !type_aligned(preact, out_type) || !type_aligned(residual, out_type) || !type_aligned(bias, bias ? bias_type : EP_E4M3) ||
        !aligned(x_scale, 4) || !aligned(w_scale, 4))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    const bool ready = tma_ready(x, ldx, in_type) && tma_ready(w, ldw, in_type);
    const LinearWorkspace ws = linear_workspace(ctx, rows, n_in, n_out, in_type, out_type, ready, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < ws.bytes)
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    Epilogue e{};
    e.x_scale = x_scale;
    e.w_scale = w_scale;
    e.bias = bias;
    e.bias_type = bias_type;
    e.act = act;
    e.residual = residual;
    e.ldr = ldr;
    e.out = out;
    e.preact = preact;
    e.out_type = out_type;
    e.M = rows;
    e.N = n_out;
    e.vec = n_out % 8 == 0 && aligned(out, 16) && aligned(preact, 16) && aligned(residual, 16) && aligned(bias, 16) &&
            aligned(w_scale, 16) &&
            (!residual || ldr * type_size(out_type) % 16 == 0);
    e.tma = tma_ready(out, n_out, out_type) && tma_ready(preact, n_out, out_type) &&
            (!residual || tma_ready(residual, ldr, out_type));
    DeviceGuard guard(ctx->device);
    Timed tm(ctx, static_cast<cudaStream_t>(cuda_stream), EP_TIMER_LINEAR);
    int kernels = 0;
    const int rc = linear_run(ctx, ws, x, ldx, w, ldw, in_type, rows, n_in, n_out, ready, e, static_cast<cudaStream_t>(cuda_stream),
                              &kernels);
    tm.end(kernels);
    return rc;
}

size_t ep_linear_backward_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t n_in, int32_t n_out, int32_t in_type,
                                          int32_t is_aligned) {
    if (!ctx || !linear_shape_ok(rows, n_in, n_out) || !float_type(in_type)) return 0;
    return backward_workspace(ctx, rows, n_in, n_out, in_type, is_aligned != 0, nullptr).bytes;
}

int ep_linear_backward(ep_ctx *ctx, const void *dout, int32_t dout_type, const void *preact, int32_t act, const void *x,
                       int64_t ldx, const void *w, int64_t ldw, int32_t in_type, int64_t rows, int32_t n_in, int32_t n_out,
                       void *dx, void *dweight, float *dbias, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (!linear_shape_ok(rows, n_in, n_out))
        return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld, n_in %d or n_out %d out of range", (long long)rows, n_in, n_out);
    if (!float_type(in_type) || !(dout_type == in_type || dout_type == EP_F32))
        return fail(ctx, EP_ERR_INVALID_ARG, "no gradient of type %d for a product of type %d", dout_type, in_type);
    if (act < EP_ACT_NONE || act > EP_ACT_SILU) return fail(ctx, EP_ERR_INVALID_ARG, "unknown activation %d", act);
    if (ldx < n_in || ldw < n_in) return fail(ctx, EP_ERR_INVALID_ARG, "a row stride is shorter than its row");
    if (!type_aligned(dweight, in_type) || !aligned(dbias, 4)) return fail(ctx, EP_ERR_INVALID_ARG, "misaligned pointer");
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    DeviceGuard guard(ctx->device);
    if (rows == 0) {
        if (dweight) EP_CUDA(ctx, cudaMemsetAsync(dweight, 0, (size_t)n_out * n_in * type_size(in_type), stream));
        if (dbias) EP_CUDA(ctx, cudaMemsetAsync(dbias, 0, sizeof(float) * (size_t)n_out, stream));
        return EP_OK;
    }
    if (!dout || (dweight && !x) || (dx && !w) || (act != EP_ACT_NONE && !preact) || !type_aligned(dout, dout_type) ||
        !type_aligned(preact, in_type) || !type_aligned(x, in_type) || !type_aligned(w, in_type) || !type_aligned(dx, in_type))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    const bool ready = tma_ready(x, ldx, in_type) && tma_ready(w, ldw, in_type);
    const BackwardWorkspace ws = backward_workspace(ctx, rows, n_in, n_out, in_type, ready, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < ws.bytes)
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    Timed tm(ctx, stream, EP_TIMER_LINEAR);
    int kernels = 0;
    const int rc = linear_backward_run(ctx, ws, dout, dout_type, preact, act, x, ldx, w, ldw, in_type, rows, n_in, n_out, ready, dx,
                                       dweight, dbias, stream, &kernels);
    tm.end(kernels);
    return rc;
}

}  // extern "C"
