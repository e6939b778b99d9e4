// A layer of experts for a few rows: router, the k best parts of each row, both products of every chosen part, their sum.
//
//     p = softmax(x Wr^T + br);  ids, w as ep_route;   out = sum_i w_i (W2[e_i] act(W1[e_i] x + b1[e_i]) + b2[e_i]) + residual
//
// What it costs is reading the chosen experts' weights, once each: slots (a row's choice of a part) are sorted by part, up to 8
// rows of one part make a group, and a warp that fetches a row of weights multiplies it with all rows of the group.  Sums
// are fp32 multiply-adds and the hidden values stay in fp32, or, with enough slots, matrix instructions and two bf16 numbers to a
// hidden value (see there).
//
// Measured, on the device: one row, 2 of 64 experts of 1024 -> 4096 -> 1024 bf16 (33.6 MB of weights, 5.2 us at 6551 GB/s) 16.4 us, in three
// launches that wait for one another: router 5 us of latency, then 6 us each for 17 MB (the second's come to the L2 meanwhile).
// 16 rows, weights in 8 bits, 173 MB: 87 us, 2.0 TB/s: bound by instructions (0.47 a clock and scheduler: integers made floats) and by
// what 16 warps an SM keep in flight (three steps of 64 bytes a lane).  7 rows of 333 -> 1029 -> 77 fp32, not aligned: 27.6 us.
#include "activation.cuh"
#include "ep_common.cuh"
#include "rows.cuh"

#include <algorithm>
#include <type_traits>

using namespace eprow;

namespace {

constexpr int MAX_ROWS = 64, MAX_K = 32, MAX_EXPERTS = 4096, MAX_WIDTH = 65536;
constexpr int GROUP = 8;      // rows of a group
constexpr int THREADS = 512, WARPS = THREADS / 32;

struct Group {
    int expert, first, count;   // slots first .. first + count - 1 of the sorted list
};
// What the router leaves for the products.
struct Plan {
    int *n_groups;
    Group *groups;
    int *sorted;      // slot (row * k + i) at each place of the sorted list
    int *place;       // place of each slot; -1: none
};

// ---------------------------------------------------------------------------------------------- dot products
// N elements of a row: VEC, 16 bytes from column c + lane * N on; otherwise columns c + lane, c + lane + 32, ...; zero past n.
template <typename T, int N, bool VEC>
struct Chunk {
    alignas(16) T e[N];
    __device__ __forceinline__ void load(const T *row, int c, int lane, int n) {
        if constexpr (VEC) {
            constexpr int PIECES = N * (int)sizeof(T) / 16;
            const int col = c + lane * N;
#pragma unroll
            for (int p = 0; p < PIECES; ++p)
                reinterpret_cast<uint4 *>(e)[p] = col < n ? reinterpret_cast<const uint4 *>(row + col)[p] : make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = c + i * 32 + lane < n ? row[c + i * 32 + lane] : T{};
        }
    }
    // Elements 2 i and 2 i + 1.  (Integers without the conversion instruction, which runs at a quarter of this rate: the byte less
    // its sign's offset into the low bits of 2^23, and the offset off again.)
    __device__ __forceinline__ Pair pair(int i) const {
        if constexpr (std::is_same_v<T, i8> && VEC) {
            const uint32_t w = reinterpret_cast<const uint32_t *>(e)[i / 2] ^ 0x80808080u;
            return add2(Pair(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7640 + (i & 1) * 2)),
                             __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7641 + (i & 1) * 2))),
                        Pair(-8388736.f));
        } else
            return Pair(to_f32(e[2 * i]), to_f32(e[2 * i + 1]));
    }
};

// Sums over the lanes: half of them stay with either half of the lanes, until there is one to each.  The sum of pair j R + r
// goes to the lanes from (j R + r) 32 / (J R) on.
template <int J, int R>
__device__ __forceinline__ float over_lanes(const Pair (&t)[J][R], int lane) {
    constexpr int M = J * R;
    float v[M];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float lo, hi;
            t[j][r].get(lo, hi);
            v[j * R + r] = lo + hi;
        }
    int o = 16;
#pragma unroll
    for (int m = M / 2; m >= 1; m /= 2, o /= 2) {
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < m; ++i) {
            const float mine = upper ? v[i + m] : v[i], theirs = upper ? v[i] : v[i + m];
            v[i] = mine + __shfl_xor_sync(FULL, theirs, o);
        }
    }
#pragma unroll
    for (; o >= 1; o /= 2) v[0] += __shfl_xor_sync(FULL, v[0], o);
    return v[0];
}

// What a lane takes of a row at a time: 16 bytes, or, where rows are not aligned for that, 4 elements.
template <typename W, bool VEC>
constexpr int step_elements() { return VEC ? 16 / (int)sizeof(W) : 4; }
// w_j . x_r over a share of the columns, for J rows of weights and R rows of x, read straight into registers.
template <typename W, typename X, bool VEC, int J, int R>
__device__ __forceinline__ float dots(const W *const (&w)[J], const X *const (&x)[R], int from, int to, int n, int lane) {
    constexpr int N = step_elements<W, VEC>(), AHEAD = 2;
    Pair t[J][R];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) t[j][r] = Pair(0.f);
    for (int c0 = from; c0 < to; c0 += AHEAD * 32 * N) {
        Chunk<W, N, VEC> a[AHEAD][J];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
#pragma unroll
            for (int j = 0; j < J; ++j) a[q][j].load(w[j], c0 + q * 32 * N, lane, n);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            if (q > 0 && c0 + q * 32 * N >= to) break;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                Chunk<X, N, VEC> b;
                b.load(x[r], c0 + q * 32 * N, lane, n);
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    const Pair v = b.pair(i);
#pragma unroll
                    for (int j = 0; j < J; ++j) t[j][r] = fma2(a[q][j].pair(i), v, t[j][r]);
                }
            }
        }
    }
    return over_lanes(t, lane);
}
__device__ __forceinline__ float over_lanes(float v) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

template <typename W>
struct Rows {
    const W *first;
    int64_t ld;
    int count, from, to;   // rows, columns
};
// Products of (up to) four rows of weights that are not aligned for 16-byte accesses.
template <typename W, typename X, int R>
__device__ __forceinline__ float straight(const Rows<W> &rows, const X *const (&x)[R], int lane) {
    const W *w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = rows.first + min(j, rows.count - 1) * rows.ld;
    return dots<W, X, false, 4, R>(w, x, rows.from, rows.to, rows.to, lane);
}
// item(n) with the n of 1, 2, 4 and 8 that `count` rows need.
template <typename Item>
__device__ __forceinline__ void by_rows(int count, Item &item) {
    if (count == 1)
        item(std::integral_constant<int, 1>{});
    else if (count == 2)
        item(std::integral_constant<int, 2>{});
    else if (count <= 4)
        item(std::integral_constant<int, 4>{});
    else
        item(std::integral_constant<int, 8>{});
}
// Rows of weights on their way to shared memory, STREAM_STAGES - 1 steps ahead of their use and past the end of an item (four
// rows, and the columns that are wanted of them): what is in flight is what a warp gets out of the memory (weights read by the
// item into registers, used, and only then the next: 1.8 TB/s).  Each lane reads back what it copied itself.
constexpr int STREAM_ROWS = 4, STREAM_STAGES = 4;
constexpr size_t STREAM_BYTES = (size_t)STREAM_STAGES * STREAM_ROWS * THREADS * 16;
template <typename W, typename Find>
struct Stream {
    static constexpr int N = 16 / (int)sizeof(W), ROW = THREADS * 16, STAGE = STREAM_ROWS * ROW;   // bytes between rows, between stages
    const Find &find;      // the rows of an item
    const int64_t items, step;
    const char *const mine;
    int64_t item;
    const char *from;      // this lane's next chunk of the first row
    int64_t ld;            // bytes from row to row
    int count, left;       // rows; columns that are still to come, of all lanes
    int to_at, at;         // stages, in bytes
    __device__ __forceinline__ Stream(void *room, const Find &f, int64_t first, int64_t all, int64_t by)
        : find(f), items(all), step(by), mine(static_cast<const char *>(room) + threadIdx.x * 16), item(first), from(nullptr), ld(0), count(0),
          left(0), to_at(0), at(0) {
        open();
        for (int s = 0; s < STREAM_STAGES - 1; ++s) fetch();
    }
    __device__ __forceinline__ void open() {
        if (item < items) {
            const Rows<W> r = find(item);
            from = reinterpret_cast<const char *>(r.first + r.from) + (threadIdx.x & 31) * 16;
            ld = r.ld * (int64_t)sizeof(W);
            count = r.count;
            left = r.to - r.from;
        }
    }
    __device__ __forceinline__ void fetch() {
        if (left > 0) {
            if ((int)(threadIdx.x & 31) * N < left) {
                char *to = const_cast<char *>(mine) + to_at;
#pragma unroll
                for (int j = 0; j < STREAM_ROWS; ++j)
                    if (j < count) copy_async<16>(to + j * ROW, from + j * ld);
            }
            from += 512;
            left -= 32 * N;
            if (left <= 0) {
                item += step;
                open();
            }
        }
        copies_end_group();
        to_at = to_at + STAGE == STREAM_STAGES * STAGE ? 0 : to_at + STAGE;
    }
    // w_j . x_r of the item whose turn it is (its columns are from..to).
    template <typename X, int R>
    __device__ __forceinline__ void add(const X *const (&x)[R], int from, int to, Pair (&t)[STREAM_ROWS][R]) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int j = 0; j < STREAM_ROWS; ++j)
#pragma unroll
            for (int r = 0; r < R; ++r) t[j][r] = Pair(0.f);
#pragma unroll 1
        for (int c0 = from; c0 < to; c0 += 32 * N) {
            fetch();
            copies_wait<STREAM_STAGES - 1>();
            const int col = c0 + lane * N;
            const bool there = col < to;
            Chunk<W, N, true> a[STREAM_ROWS];
#pragma unroll
            for (int j = 0; j < STREAM_ROWS; ++j) {
                // (rows past the last are whatever was there before: their sums go nowhere)
                const uint4 v = *reinterpret_cast<const uint4 *>(mine + at + j * ROW);
                *reinterpret_cast<uint4 *>(a[j].e) = there ? v : make_uint4(0, 0, 0, 0);
            }
            // a few columns at a time: what is converted has to fit the registers beside the sums
            constexpr int SOME = R >= 8 || sizeof(X) == 4 || N < 8 ? 4 : 8;
#pragma unroll
            for (int q = 0; q < N; q += SOME) {
                Pair w[STREAM_ROWS][SOME / 2];
#pragma unroll
                for (int j = 0; j < STREAM_ROWS; ++j)
#pragma unroll
                    for (int i = 0; i < SOME / 2; ++i) w[j][i] = a[j].pair(q / 2 + i);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    using Bytes = typename Raw<SOME * (int)sizeof(X)>::type;
                    alignas(16) X b[SOME];
                    *reinterpret_cast<Bytes *>(b) = there ? *reinterpret_cast<const Bytes *>(x[r] + col + q) : Bytes{};
#pragma unroll
                    for (int i = 0; i < SOME / 2; ++i) {
                        const Pair v(to_f32(b[2 * i]), to_f32(b[2 * i + 1]));
#pragma unroll
                        for (int j = 0; j < STREAM_ROWS; ++j) t[j][r] = fma2(w[j][i], v, t[j][r]);
                    }
                }
            }
            at = at + STAGE == STREAM_STAGES * STAGE ? 0 : at + STAGE;
        }
    }
    template <typename X, int R>
    __device__ __forceinline__ float dots(const X *const (&x)[R], int from, int to) {
        Pair t[STREAM_ROWS][R];
        add<X, R>(x, from, to, t);
        return over_lanes(t, threadIdx.x & 31);
    }
};

// ---------------------------------------------------------------------------------------------- router
// logits[row][e] = x Wr^T + br: a warp to a part and R rows.
template <typename T, bool VEC, int R>
__global__ void __launch_bounds__(128) experts_logits(const T *x, int64_t ldx, const T *router, const void *bias, int bias_type, int rows,
                                                      int n_in, int experts, float *logits) {
    const int lane = threadIdx.x & 31, e = blockIdx.x * 4 + (threadIdx.x >> 5), row0 = blockIdx.y * R;
    ep_let_next_launch_start();
    if (e >= experts) return;
    const T *w[1] = {router + (int64_t)e * n_in};
    const T *xs[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xs[r] = x + min(row0 + r, rows - 1) * ldx;
    const float add = bias ? load_param(bias, bias_type, e) : 0.f;
    const float v = dots<T, T, VEC, 1, R>(w, xs, 0, n_in, n_in, lane);
    const int r = lane / (32 / R);
    if (lane % (32 / R) == 0 && row0 + r < rows) logits[(row0 + r) * experts + e] = v + add;
}

// A row's k best parts and their weights (as ep_route), by one warp.  (The first 128 logits are kept in registers.)
__device__ void choose(const float *logits, int experts, int k, bool part, bool renormalize, int lane, int32_t *ids, float *weights) {
    constexpr int KEPT = 4;
    float kept[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) kept[i] = part && 32 * i + lane < experts ? logits[32 * i + lane] : -INFINITY;
    auto each = [&](auto f) {
        if (!part) return;
#pragma unroll
        for (int i = 0; i < KEPT; ++i)
            if (32 * i < experts) f(kept[i], 32 * i + lane);
        for (int e = 32 * KEPT + lane; e < experts; e += 32) f(logits[e], e);
    };
    float top = -INFINITY;
    each([&](float v, int) { top = fmaxf(top, v); });
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
    part = part && top > -INFINITY;
    float s = 0.f;
    each([&](float v, int) { s += exp_fast(v - top); });
    s = over_lanes(s);
    float last = INFINITY, chosen = 0.f, mine = 0.f;
    int last_e = -1, mine_e = -1;
    for (int i = 0; i < k; ++i) {   // the best that comes after the one before: lower, or as high with a higher number
        float v = -INFINITY;
        int at = MAX_EXPERTS;
        each([&](float u, int e) {
            if (u > v && (u < last || (u == last && e > last_e))) {
                v = u;
                at = e;
            }
        });
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) {
            const float ov = __shfl_xor_sync(FULL, v, o);
            const int oe = __shfl_xor_sync(FULL, at, o);
            if (ov > v || (ov == v && oe < at)) {
                v = ov;
                at = oe;
            }
        }
        const bool got = v > -INFINITY;
        const float ex = got ? exp_fast(v - top) : 0.f;
        chosen += ex;
        if (lane == i) {
            mine = ex;
            mine_e = got ? at : -1;
        }
        last = v;
        last_e = at;
    }
    if (lane < k) {
        const float nan_too = s != s ? s : 0.f;
        ids[lane] = mine_e;
        weights[lane] = !part ? 0.f : renormalize ? mine / chosen + nan_too : mine / s;
    }
}

// ids and weights of all rows, and their slots sorted by part: one block.
__global__ void __launch_bounds__(1024) experts_choose(const float *logits, const uint8_t *valid, int rows, int experts, int k,
                                                       bool renormalize, int32_t *ids, float *weights, Plan plan) {
    __shared__ int count[MAX_EXPERTS + 1];   // slots of each part; then where they start
    __shared__ int groups_before[32], slots_before[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int e = threadIdx.x; e < experts; e += 1024) count[e] = 0;
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    for (int r = warp; r < rows; r += 32)
        choose(logits + r * experts, experts, k, !valid || valid[r], renormalize, lane, ids + r * k, weights + r * k);
    __syncthreads();
    const int slots = rows * k;
    for (int s = threadIdx.x; s < slots; s += 1024)
        if (ids[s] >= 0) atomicAdd(&count[ids[s]], 1);
    __syncthreads();
    // thread t has parts 4 t .. 4 t + 3 (MAX_EXPERTS of them in all)
    int c[4], g = 0, n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = threadIdx.x * 4 + i;
        c[i] = e < experts ? count[e] : 0;
        g += (c[i] + GROUP - 1) / GROUP;
        n += c[i];
    }
    int g_at = g, n_at = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int a = __shfl_up_sync(FULL, g_at, o), b = __shfl_up_sync(FULL, n_at, o);
        if (lane >= o) {
            g_at += a;
            n_at += b;
        }
    }
    if (lane == 31) {
        groups_before[warp] = g_at;
        slots_before[warp] = n_at;
    }
    __syncthreads();
    g_at -= g;
    n_at -= n;
    for (int w = 0; w < warp; ++w) {
        g_at += groups_before[w];
        n_at += slots_before[w];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = threadIdx.x * 4 + i;
        if (e < experts) count[e] = n_at;
        for (int f = 0; f < c[i]; f += GROUP) plan.groups[g_at++] = Group{e, n_at + f, min(c[i] - f, GROUP)};
        n_at += c[i];
    }
    if (threadIdx.x == 1023) *plan.n_groups = g_at;
    __syncthreads();
    for (int s = threadIdx.x; s < slots; s += 1024) {
        int at = -1;
        if (ids[s] >= 0) {
            at = atomicAdd(&count[ids[s]], 1);   // (in any order: a slot's sums do not depend on its place)
            plan.sorted[at] = s;
        }
        plan.place[s] = at;
    }
}

// The same for up to 64 slots, each compared with the others.
constexpr int FEW_SLOTS = 64;
struct alignas(16) FewSlots {
    int32_t ids[FEW_SLOTS];
    int starts[FEW_SLOTS];   // where a group starts that a slot is the first of
};
__device__ void plan_few(FewSlots &few, int slots, const Plan &plan) {
    const int s = threadIdx.x, e = s < FEW_SLOTS ? few.ids[s] : -1;   // (slots past the last hold -1)
    int before = 0, of_part = 0, earlier = 0, at = -1;                // slots of lower parts; slots of this part, and those of them before this one
    if (s < FEW_SLOTS) {
#pragma unroll 4
        for (int q = 0; q < FEW_SLOTS; q += 4) {
            if (q >= slots) break;
            const int4 o = *reinterpret_cast<const int4 *>(few.ids + q);
            before += (o.x >= 0 && o.x < e) + (o.y >= 0 && o.y < e) + (o.z >= 0 && o.z < e) + (o.w >= 0 && o.w < e);
            of_part += (o.x == e) + (o.y == e) + (o.z == e) + (o.w == e);
            earlier += (o.x == e && q < s) + (o.y == e && q + 1 < s) + (o.z == e && q + 2 < s) + (o.w == e && q + 3 < s);
        }
        at = e < 0 ? -1 : before + earlier;
        // a group starts at every eighth slot of a part; its number is that of the groups that start before it in the sorted list
        few.starts[s] = e >= 0 && earlier % GROUP == 0 ? at : 1 << 30;
        if (e >= 0) plan.sorted[at] = s;
        if (s < slots) plan.place[s] = at;
    }
    __syncthreads();
    if (s < FEW_SLOTS) {
        const int mine = few.starts[s];
        int number = 0, all = 0;
#pragma unroll 4
        for (int q = 0; q < FEW_SLOTS; q += 4) {
            const int4 o = *reinterpret_cast<const int4 *>(few.starts + q);
            number += (o.x < mine) + (o.y < mine) + (o.z < mine) + (o.w < mine);
            all += (o.x < 1 << 30) + (o.y < 1 << 30) + (o.z < 1 << 30) + (o.w < 1 << 30);
        }
        if (mine < 1 << 30) plan.groups[number] = Group{e, at, min(of_part - earlier, GROUP)};
        if (s == 0) *plan.n_groups = all;
    }
}

// All of the router in one launch, for a few rows: the blocks of a cluster share out the dot products, then the first one chooses
// and plans.
constexpr int ROUTER_BLOCKS = 8, ROUTER_JOBS = 4 * ROUTER_BLOCKS * WARPS;   // (a warp's dot products, four one after another at most)
template <typename T, bool VEC, int R>
__global__ void __launch_bounds__(THREADS) experts_router(const T *x, int64_t ldx, const T *router, const void *bias, int bias_type, int rows,
                                                          int n_in, int experts, float *logits, const uint8_t *valid, int k, bool renormalize,
                                                          int32_t *ids, float *weights, Plan plan) {
    __shared__ FewSlots few;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, across = (rows + R - 1) / R;
    ep_let_next_launch_start();
    for (int job = warp * ROUTER_BLOCKS + blockIdx.x; job < experts * across; job += ROUTER_BLOCKS * WARPS) {
        const int e = job / across, row0 = (job - e * across) * R;
        const T *w[1] = {router + (int64_t)e * n_in};
        const T *xs[R];
#pragma unroll
        for (int r = 0; r < R; ++r) xs[r] = x + min(row0 + r, rows - 1) * ldx;
        const float v = dots<T, T, VEC, 1, R>(w, xs, 0, n_in, n_in, lane);
        const int r = lane / (32 / R);
        if (lane % (32 / R) == 0 && row0 + r < rows) logits[(row0 + r) * experts + e] = v + (bias ? load_param(bias, bias_type, e) : 0.f);
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (blockIdx.x != 0) return;
    const int slots = rows * k;
    if (threadIdx.x < FEW_SLOTS) few.ids[threadIdx.x] = -1;
    __syncthreads();
    for (int r = warp; r < rows; r += WARPS) {
        choose(logits + r * experts, experts, k, !valid || valid[r], renormalize, lane, ids + r * k, weights + r * k);
        if (lane < k) few.ids[r * k + lane] = ids[r * k + lane];   // (written by this lane)
    }
    __syncthreads();
    plan_few(few, slots, plan);
}

// ---------------------------------------------------------------------------------------------- products
struct Weights {
    const void *w;
    const float *scale;   // of 8-bit integers
    const void *bias;
    int bias_type;
};

// hidden[place][j] = act(W1[e][j] . x + b1[e][j]): a warp to 4 rows of a part's weights; dots: their products with R rows of x.
template <typename T, int R, typename Dots>
__device__ __forceinline__ void hidden_of(const T *x, int64_t ldx, const Weights &w1, int n_hidden, int act, int k, const int *sorted,
                                          const Group &g, int j0, float *hidden, int lane, Dots dots) {
    const T *xs[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xs[r] = x + (sorted[g.first + min(r, g.count - 1)] / k) * ldx;
    constexpr int LANES = 32 / (STREAM_ROWS * R);
    const int j = j0 + lane / LANES / R, r = lane / LANES % R;
    const bool mine = lane % LANES == 0 && j < n_hidden && r < g.count;
    const int64_t at = (int64_t)g.expert * n_hidden + j;
    const float scale = mine && w1.scale ? w1.scale[at] : 1.f, bias = mine && w1.bias ? load_param(w1.bias, w1.bias_type, at) : 0.f;
    float v[1] = {dots(xs)};
    if (mine) {
        v[0] = fmaf(v[0], scale, bias);
        activate(v, act);
        hidden[(int64_t)(g.first + r) * n_hidden + j] = v[0];
    }
}
// Asks for bytes [from, to) of [0, all) of the L2 (in whole 16 bytes).
__device__ __forceinline__ void ask_l2(const char *base, int64_t all, int part, int parts) {
    const int64_t from = all * part / parts & ~int64_t(15), to = all * (part + 1) / parts & ~int64_t(15);
    if (to > from) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(base + from), "r"((uint32_t)(to - from)) : "memory");
}
template <typename T, typename W, bool VEC>
__global__ void __launch_bounds__(THREADS) experts_hidden(const T *x, int64_t ldx, Weights w1, int n_in, int n_hidden, int act, int k, Plan p,
                                                          const void *w2, int64_t w2_bytes, float *hidden) {
    const int lane = threadIdx.x & 31;
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    const int *sorted = p.sorted;
    const Group *groups = p.groups;
    const int n_groups = *p.n_groups;
    // While this product waits for its own weights, those of the next one come to the L2, where they fit it.
    if (w2_bytes && threadIdx.x < n_groups)
        ask_l2(static_cast<const char *>(w2) + groups[threadIdx.x].expert * w2_bytes, w2_bytes, blockIdx.x, gridDim.x);
    const int across = (n_hidden + STREAM_ROWS - 1) / STREAM_ROWS;
    const int64_t items = (int64_t)n_groups * across, step = (int64_t)gridDim.x * WARPS, first = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x;
    auto rows_of = [&](int64_t i) {
        const int q = (int)(i / across), j0 = (int)(i - (int64_t)q * across) * STREAM_ROWS;
        return Rows<W>{static_cast<const W *>(w1.w) + ((int64_t)groups[q].expert * n_hidden + j0) * n_in, n_in, min(STREAM_ROWS, n_hidden - j0), 0,
                       n_in};
    };
    // each item's products by the rows that its group has
    auto all = [&](auto products) {
        for (int64_t i = first; i < items; i += step) {
            const int q = (int)(i / across), j0 = (int)(i - (int64_t)q * across) * STREAM_ROWS;
            const Group g = groups[q];
            auto item = [&](auto rows) {
                hidden_of<T, decltype(rows)::value>(x, ldx, w1, n_hidden, act, k, sorted, g, j0, hidden, lane,
                                                    [&](const T *const (&xs)[decltype(rows)::value]) { return products(i, xs); });
            };
            by_rows(g.count, item);
        }
    };
    if constexpr (VEC) {
        extern __shared__ uint4 ring[];
        Stream<W, decltype(rows_of)> stream(ring, rows_of, first, items, step);
        all([&](int64_t, const auto &xs) { return stream.dots(xs, 0, n_in); });
        copies_wait<0>();
    } else
        all([&](int64_t i, const auto &xs) { return straight<W>(rows_of(i), xs, lane); });
}

// y[share][place][column of the block] = W2[e][column] . hidden over one share of the hidden values.
template <int R, typename Dots>
__device__ __forceinline__ void output_of(const float *hidden, int n_hidden, const Group &g, float *y, int cols, int at, int lane, Dots dots) {
    const float *xs[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xs[r] = hidden + (int64_t)(g.first + min(r, g.count - 1)) * n_hidden;
    const float v = dots(xs);
    constexpr int LANES = 32 / (STREAM_ROWS * R);
    const int j = lane / LANES / R, r = lane / LANES % R;
    if (lane % LANES == 0 && at + j < cols && r < g.count) y[(g.first + r) * cols + at + j] = v;
}
// A block has `cols` columns of the output, of all rows; its warps share out groups, 4 columns at a time, and shares of the hidden values.
template <typename T, typename W, bool VEC>
__global__ void __launch_bounds__(THREADS) experts_output(const float *hidden, Weights w2, int n_hidden, int n_out, int rows, int k, Plan p,
                                                          const int32_t *ids, const float *weights, const T *residual, int64_t ldr, T *out,
                                                          int cols, int shares, int per_share) {
    extern __shared__ uint4 ring[];   // of the weights, where VEC; then y[shares][rows * k][cols]
    float *y = reinterpret_cast<float *>(reinterpret_cast<char *>(ring) + (VEC ? STREAM_BYTES : 0));
    const int lane = threadIdx.x & 31, slots = rows * k;
    const int col0 = blockIdx.x * cols, mine = min(cols, n_out - col0);
    ep_wait_for_launch_before();
    const int across = (mine + STREAM_ROWS - 1) / STREAM_ROWS;
    const int items = *p.n_groups * across * shares, first = threadIdx.x >> 5;
    auto rows_of = [&](int64_t i) {
        const int share = (int)i % shares, q = (int)i / shares, at = q % across * STREAM_ROWS, from = share * per_share;
        return Rows<W>{static_cast<const W *>(w2.w) + ((int64_t)p.groups[q / across].expert * n_out + col0 + at) * n_hidden, n_hidden,
                       min(STREAM_ROWS, mine - at), from, min(from + per_share, n_hidden)};
    };
    auto all = [&](auto products) {
        for (int i = first; i < items; i += WARPS) {
            const int share = i % shares, q = i / shares, at = q % across * STREAM_ROWS;
            const Group g = p.groups[q / across];
            auto item = [&](auto rows) {
                output_of<decltype(rows)::value>(hidden, n_hidden, g, y + share * slots * cols, cols, at, lane,
                                                 [&](const float *const (&xs)[decltype(rows)::value]) { return products(i, xs, share); });
            };
            by_rows(g.count, item);
        }
    };
    if constexpr (VEC) {
        Stream<W, decltype(rows_of)> stream(ring, rows_of, first, items, WARPS);
        all([&](int, const auto &xs, int share) { return stream.dots(xs, share * per_share, min(share * per_share + per_share, n_hidden)); });
        copies_wait<0>();
    } else
        all([&](int i, const auto &xs, int) { return straight<W>(rows_of(i), xs, lane); });
    __syncthreads();
    for (int i = threadIdx.x; i < rows * mine; i += THREADS) {
        const int row = i / mine, c = i - row * mine;
        float sum = 0.f;
        for (int s = 0; s < k; ++s) {
            const int slot = row * k + s, at = p.place[slot];
            if (at < 0) continue;
            float v = 0.f;
            for (int h = 0; h < shares; ++h) v += y[(h * slots + at) * cols + c];
            const int64_t param = (int64_t)ids[slot] * n_out + col0 + c;
            if (w2.scale) v *= w2.scale[param];
            if (w2.bias) v += load_param(w2.bias, w2.bias_type, param);
            sum = fmaf(weights[slot], v, sum);
        }
        if (residual) sum += to_f32(residual[row * ldr + col0 + c]);
        out[(int64_t)row * n_out + col0 + c] = from_f32<T>(sum);
    }
}

// ---------------------------------------------------------------------------------------------- products by matrix instructions
//
// Where there are enough slots (enough_for_tensor), a warp multiplies 16 rows of weights with the (up to 8)
// rows of a group by matrix instructions, 16 x 8 x 16 at a time: a number of weights then costs a third of the instructions, most
// of them for making 8-bit integers 16-bit floats (which hold them exactly).  The order of the columns within a step is the lanes'
// own: each takes 16 bytes of its rows of weights, and the same columns of its row of x.  Hidden values go to the second
// product as the sum of two bf16 numbers (16 bits, beside outputs of 8 or 11 bits).
template <typename M>
__device__ __forceinline__ void multiply(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same_v<M, __half>)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes of weights as pairs of M.
template <typename M, typename W>
__device__ __forceinline__ void as_pairs(const uint4 &v, uint32_t (&p)[4 * sizeof(M) / sizeof(W)]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (!std::is_same_v<W, i8>)
            p[q] = w[q];
        else if constexpr (std::is_same_v<M, __half>) {
            const uint32_t u = w[q] ^ 0x80808080u;   // 1024 and the byte, less 1024 + 128
            const __half2 off = __half2half2(__ushort_as_half(0x6480));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t h = __byte_perm(u, 0x64646464u, i ? 0x4342 : 0x4140);
                const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&h), off);
                p[2 * q + i] = *reinterpret_cast<const uint32_t *>(&r);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {            // 128 and the low seven bits, less 128 or, of a negative number, 256
                const uint32_t b = __byte_perm(w[q], 0u, i ? 0x4342 : 0x4140);
                const uint32_t low = (b & 0x007f007fu) | 0x43004300u, off = (b & 0x00800080u) | 0x43004300u;
                const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&low), *reinterpret_cast<const __nv_bfloat162 *>(&off));
                p[2 * q + i] = *reinterpret_cast<const uint32_t *>(&r);
            }
        }
    }
}

struct TensorWork {
    const void *x;               // rows of x, or hidden values: high parts, and `low` further on low parts
    int64_t ldx, low;
    const void *w;               // [experts][rows][cols]
    int rows, cols, k;
    const float *scale;
    const void *bias;
    int bias_type, act;
    int shares, per_share;       // of the columns
    __nv_bfloat16 *hidden;       // out of the first product
    float *y;                    // out of the second: [share][slots][rows]
    int slots;
};
// The items of one product: group, 16 rows of weights, share of the columns.
template <typename W>
struct TensorItems {
    const TensorWork &e;
    const Group *groups;
    int across;
    struct Item {
        Group g;
        int row0, share, from, to;
    };
    __device__ __forceinline__ Item operator()(int64_t i) const {
        const int share = (int)(i % e.shares), q = (int)(i / e.shares), from = share * e.per_share;
        return Item{groups[q / across], q % across * 16, share, from, min(from + e.per_share, e.cols)};
    }
};
constexpr int TENSOR_STAGES = 4;   // (two blocks to an SM with three stages each: 90 us where this takes 80)
constexpr size_t TENSOR_BYTES = (size_t)TENSOR_STAGES * 4 * THREADS * 16;

// SECOND: from hidden values (two bf16 parts) to y; otherwise from x to hidden values.  M: what the matrix instructions take.
template <bool SECOND, typename M, typename W>
__global__ void __launch_bounds__(THREADS) experts_tensor(const TensorWork e, Plan p, const void *next, int64_t next_bytes) {
    constexpr int N = 16 / (int)sizeof(W), PAIRS = N / 2;
    extern __shared__ uint4 ring[];   // [TENSOR_STAGES][4][THREADS]
    const int lane = threadIdx.x & 31;
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    const int *sorted = p.sorted;
    const Group *groups = p.groups;
    const int n_groups = *p.n_groups;
    if (!SECOND && next_bytes && threadIdx.x < n_groups)
        ask_l2(static_cast<const char *>(next) + groups[threadIdx.x].expert * next_bytes, next_bytes, blockIdx.x, gridDim.x);
    const TensorItems<W> item_of{e, groups, (e.rows + 15) / 16};
    const int64_t items = (int64_t)n_groups * item_of.across * e.shares, step = (int64_t)gridDim.x * WARPS;
    const int64_t first = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x;
    // rows of weights on their way, as in Stream: of rows lane / 4 and that + 8, two steps of 4 lanes x 16 bytes
    constexpr int PIECE = THREADS * 16, STAGE = 4 * PIECE;
    char *const mine = reinterpret_cast<char *>(ring) + threadIdx.x * 16;
    int64_t ahead = first;
    const char *from[2] = {};   // this lane's next chunk of either row
    int left = 0, left_here[2] = {};   // columns still to come: of all lanes, and of either row from this lane's chunk on
    int to_at = 0, at = 0;      // stages, in bytes
    auto open = [&] {
        if (ahead < items) {
            const auto f = item_of(ahead);
            left = f.to - f.from;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = f.row0 + (lane >> 2) + 8 * r;
                from[r] = reinterpret_cast<const char *>(static_cast<const W *>(e.w) + ((int64_t)f.g.expert * e.rows + row) * e.cols + f.from) +
                          (lane & 3) * 16;
                left_here[r] = row < e.rows ? left - (lane & 3) * N : 0;
            }
        }
    };
    auto fetch = [&] {
        if (left > 0) {
            char *to = mine + to_at;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (left_here[q & 1] > (q >> 1) * 4 * N) copy_async<16>(to + q * PIECE, from[q & 1] + (q >> 1) * 64);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                from[r] += 128;
                left_here[r] -= 8 * N;
            }
            left -= 8 * N;
            if (left <= 0) {
                ahead += step;
                open();
            }
        }
        copies_end_group();
        to_at = to_at + STAGE == TENSOR_STAGES * STAGE ? 0 : to_at + STAGE;
    };
    open();
    for (int s = 0; s < TENSOR_STAGES - 1; ++s) fetch();
    for (int64_t i = first; i < items; i += step) {
        const auto it = item_of(i);
        const int n = lane >> 2;                     // this lane's row of x
        const bool there = n < it.g.count;
        const int place = it.g.first + (there ? n : 0);
        const M *x = static_cast<const M *>(e.x) + (SECOND ? (int64_t)place * e.cols : (sorted[place] / e.k) * e.ldx);
        float d[2][4] = {};
#pragma unroll 1
        for (int c0 = it.from; c0 < it.to; c0 += 8 * N) {
            fetch();
            copies_wait<TENSOR_STAGES - 1>();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col = c0 + (lane & 3) * N + h * 4 * N;
                const bool in = col < it.to;
                uint4 v[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    v[r] = *reinterpret_cast<const uint4 *>(mine + at + (2 * h + r) * PIECE);
                    // (a row past the last: whatever was there before, and its sums go nowhere)
                    if (!in) v[r] = make_uint4(0, 0, 0, 0);
                }
                uint32_t a[2][PAIRS];
                as_pairs<M, W>(v[0], a[0]);
                as_pairs<M, W>(v[1], a[1]);
#pragma unroll
                for (int part = 0; part < (SECOND ? 2 : 1); ++part) {
                    uint32_t b[PAIRS];
#pragma unroll
                    for (int q = 0; q < PAIRS / 4; ++q) {
                        const uint4 u = there && in ? reinterpret_cast<const uint4 *>(x + part * e.low + col)[q] : make_uint4(0, 0, 0, 0);
                        b[4 * q] = u.x, b[4 * q + 1] = u.y, b[4 * q + 2] = u.z, b[4 * q + 3] = u.w;
                    }
#pragma unroll
                    for (int q = 0; q < PAIRS; q += 2) multiply<M>(d[q / 2 & 1], a[0][q], a[1][q], a[0][q + 1], a[1][q + 1], b[q], b[q + 1]);
                }
            }
            at = at + STAGE == TENSOR_STAGES * STAGE ? 0 : at + STAGE;
        }
        // this lane's sums: rows of weights lane / 4 and that + 8, rows of x 2 (lane % 4) and the next
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int row = it.row0 + (lane >> 2) + 8 * (q >> 1), r = 2 * (lane & 3) + (q & 1);
            if (row >= e.rows || r >= it.g.count) continue;
            float v[1] = {d[0][q] + d[1][q]};
            if constexpr (SECOND)
                e.y[((int64_t)it.share * e.slots + it.g.first + r) * e.rows + row] = v[0];
            else {
                const int64_t at = (int64_t)it.g.expert * e.rows + row;
                v[0] = fmaf(v[0], e.scale ? e.scale[at] : 1.f, e.bias ? load_param(e.bias, e.bias_type, at) : 0.f);
                activate(v, e.act);
                const __nv_bfloat16 high = __float2bfloat16_rn(v[0]);
                __nv_bfloat16 *to = e.hidden + (int64_t)(it.g.first + r) * e.rows + row;
                to[0] = high;
                // (an infinity or a NaN has no rest)
                to[e.low] = __float2bfloat16_rn(fabsf(v[0]) < 3e38f ? v[0] - __bfloat162float(high) : 0.f);
            }
        }
    }
    copies_wait<0>();
}

// out = sum of the slots' outputs by their weights + residual.
template <typename T>
__global__ void __launch_bounds__(256) experts_sum(const float *y, int shares, int rows, int n_out, int k, Plan p, const int32_t *ids,
                                                   const float *weights, const float *scale, const void *bias, int bias_type,
                                                   const T *residual, int64_t ldr, T *out) {
    ep_wait_for_launch_before();
    const int i = blockIdx.x * 256 + threadIdx.x, row = i / n_out, c = i - row * n_out, slots = rows * k;
    if (row >= rows) return;
    float sum = 0.f;
    for (int s = 0; s < k; ++s) {
        const int slot = row * k + s, at = p.place[slot];
        if (at < 0) continue;
        float v = 0.f;
        for (int h = 0; h < shares; ++h) v += y[((int64_t)h * slots + at) * n_out + c];
        const int64_t param = (int64_t)ids[slot] * n_out + c;
        if (scale) v *= scale[param];
        if (bias) v += load_param(bias, bias_type, param);
        sum = fmaf(weights[slot], v, sum);
    }
    if (residual) sum += to_f32(residual[row * ldr + c]);
    out[(int64_t)row * n_out + c] = from_f32<T>(sum);
}

// ---------------------------------------------------------------------------------------------- host side
struct Layer {
    const void *x;
    int64_t ldx;
    int type;
    const void *router, *router_bias;
    int router_bias_type;
    const uint8_t *valid;
    int k;
    bool renormalize;
    Weights w1, w2;
    int w_type, act;
    const void *residual;
    int64_t ldr;
    void *out;
    int32_t *ids;
    float *weights;
    int64_t rows;
    int n_in, n_hidden, n_out, experts;
    cudaStream_t stream;
};
struct Space {
    float *logits, *hidden, *y;
    Plan plan;
    size_t bytes;
};
constexpr int MAX_SHARES = 4;   // of the hidden values, between warps of the second product by matrix instructions
Space space(int64_t rows, int n_hidden, int n_out, int experts, int k, void *base) {
    ep::Arena a(base);
    Space s{};
    const size_t slots = rows * k;
    s.logits = a.take<float>(rows * experts);
    s.hidden = a.take<float>(slots * n_hidden);
    s.y = a.take<float>(slots * n_out * MAX_SHARES);
    s.plan.n_groups = a.take<int>(1);
    s.plan.groups = a.take<Group>(slots);
    s.plan.sorted = a.take<int>(slots);
    s.plan.place = a.take<int>(slots);
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
}

constexpr int64_t L2_SHARE = 48ll << 20;   // what the next product's weights may take of the L2

template <typename T, typename W, bool VEC>
int run_products(ep_ctx *ctx, const Layer &l, const Space &s) {
    const int slots = (int)l.rows * l.k;
    const int64_t w2_bytes = (int64_t)l.n_out * l.n_hidden * sizeof(W);
    // (at most one group to a slot; what is asked for starts on 16 bytes)
    const bool ask = ep::aligned(l.w2.w, 16) && w2_bytes % 16 == 0 && w2_bytes * std::min(slots, l.experts) <= L2_SHARE;
    const size_t ring = VEC ? STREAM_BYTES : 0;
    auto first = experts_hidden<T, W, VEC>;
    if (VEC) EP_CUDA(ctx, cudaFuncSetAttribute(first, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ring));
    EP_CUDA(ctx, ep::launch_early(first, dim3(ctx->sm_count), dim3(THREADS), ring, l.stream, (const T *)l.x, l.ldx, l.w1, l.n_in, l.n_hidden,
                                  l.act, l.k, s.plan, l.w2.w, ask ? w2_bytes : (int64_t)0, s.hidden));
    constexpr int STEP = 32 * step_elements<W, VEC>();   // columns that a warp takes at a time
    constexpr size_t ROOM = 80 * 1024;                   // of y
    const int cols = std::max(1, std::min({(int)ep::ceil_div(l.n_out, ctx->sm_count), (int)(ROOM / (sizeof(float) * slots)), 64}));
    // shares of the hidden values, so that every warp has something to do
    const int items = l.k * (int)ep::ceil_div(cols, STREAM_ROWS);
    int shares = std::max(1, std::min({WARPS / items, (int)ep::ceil_div(l.n_hidden, 2 * STEP), (int)(ROOM / (sizeof(float) * slots * cols))}));
    const int per_share = (int)ep::ceil_div(ep::ceil_div(l.n_hidden, shares), STEP) * STEP;
    shares = (int)ep::ceil_div(l.n_hidden, per_share);
    auto second = experts_output<T, W, VEC>;
    EP_CUDA(ctx, cudaFuncSetAttribute(second, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(ring + ROOM)));
    EP_CUDA(ctx, ep::launch_early(second, dim3((unsigned)ep::ceil_div(l.n_out, cols)), dim3(THREADS), ring + sizeof(float) * shares * slots * cols,
                                  l.stream, s.hidden, l.w2, l.n_hidden, l.n_out, (int)l.rows, l.k, s.plan, l.ids, l.weights,
                                  (const T *)l.residual, l.ldr, (T *)l.out, cols, shares, per_share));
    return EP_OK;
}

// Both products by matrix instructions; M of the first as x, of the second bf16.
template <typename T, typename W>
int run_tensor(ep_ctx *ctx, const Layer &l, const Space &s) {
    const int slots = (int)l.rows * l.k;
    const int64_t w2_bytes = (int64_t)l.n_out * l.n_hidden * sizeof(W);
    const bool ask = w2_bytes % 16 == 0 && w2_bytes * std::min(slots, l.experts) <= L2_SHARE;
    TensorWork a{};
    a.x = l.x;
    a.ldx = l.ldx;
    a.low = (int64_t)slots * l.n_hidden;
    a.w = l.w1.w;
    a.rows = l.n_hidden;
    a.cols = l.n_in;
    a.k = l.k;
    a.scale = l.w1.scale;
    a.bias = l.w1.bias;
    a.bias_type = l.w1.bias_type;
    a.act = l.act;
    a.shares = 1;
    a.per_share = l.n_in;
    a.hidden = reinterpret_cast<__nv_bfloat16 *>(s.hidden);
    a.slots = slots;
    auto first = experts_tensor<false, T, W>;
    EP_CUDA(ctx, cudaFuncSetAttribute(first, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TENSOR_BYTES));
    EP_CUDA(ctx, ep::launch_early(first, dim3(ctx->sm_count), dim3(THREADS), TENSOR_BYTES, l.stream, a, s.plan, l.w2.w,
                                  ask ? w2_bytes : (int64_t)0));
    TensorWork b{};
    b.x = s.hidden;
    b.low = a.low;
    b.w = l.w2.w;
    b.rows = l.n_out;
    b.cols = l.n_hidden;
    b.k = l.k;
    constexpr int STEP = 8 * 16 / (int)sizeof(W);
    b.shares = (int)std::max<int64_t>(1, std::min<int64_t>(MAX_SHARES, ep::ceil_div(l.n_hidden, 4 * STEP)));
    b.per_share = (int)ep::ceil_div(ep::ceil_div(l.n_hidden, b.shares), STEP) * STEP;
    b.shares = (int)ep::ceil_div(l.n_hidden, b.per_share);
    b.y = s.y;
    b.slots = slots;
    auto second = experts_tensor<true, __nv_bfloat16, W>;
    EP_CUDA(ctx, cudaFuncSetAttribute(second, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TENSOR_BYTES));
    EP_CUDA(ctx, ep::launch_early(second, dim3(ctx->sm_count), dim3(THREADS), TENSOR_BYTES, l.stream, b, s.plan, (const void *)nullptr,
                                  (int64_t)0));
    EP_CUDA(ctx, ep::launch_early(experts_sum<T>, dim3((unsigned)ep::ceil_div(l.rows * l.n_out, 256)), dim3(256), 0, l.stream, s.y, b.shares,
                                  (int)l.rows, l.n_out, l.k, s.plan, l.ids, l.weights, l.w2.scale, l.w2.bias, l.w2.bias_type,
                                  (const T *)l.residual, l.ldr, (T *)l.out));
    return EP_OK;
}
// Multiply-adds grow with the slots, matrix instructions hardly do (16 rows of weights take 8 slots at once): from 16 slots on with integers,
// which the multiply-adds have to convert, from 40 with bf16.  Measured, multiply-adds -> matrix instructions, us, k = 2, 1024 -> 4096 -> 1024:
// integers, 4 rows of 64 parts 38 -> 38, 8 of 32 56 -> 55, 16 of 32 91 -> 88, 64 of 32 293 -> 118, 64 of 8 219 -> 78, 8 of 2 38 -> 30;
// bf16, 8 of 32 66 -> 82, 16 of 32 100 -> 119, 32 of 32 169 -> 157, 64 of 32 267 -> 172, 64 of 8 225 -> 106; and 64 rows of 2 parts of
// 256 -> 64 -> 64, integers 23 -> 18, bf16 21 -> 18.
bool enough_for_tensor(const Layer &l) { return l.rows * l.k >= (l.w_type == EP_I8 ? 16 : 40); }

bool sixteen(const void *p, int64_t ld, int size) { return ep::aligned(p, 16) && ld * size % 16 == 0; }

template <typename T, bool VEC>
int launch_logits(ep_ctx *ctx, const Layer &l, float *logits) {
    const int r = l.rows == 1 ? 1 : l.rows == 2 ? 2 : 4;
    auto kernel = r == 1 ? experts_logits<T, VEC, 1> : r == 2 ? experts_logits<T, VEC, 2> : experts_logits<T, VEC, 4>;
    kernel<<<dim3((unsigned)ep::ceil_div(l.experts, 4), (unsigned)ep::ceil_div(l.rows, r)), 128, 0, l.stream>>>(
        (const T *)l.x, l.ldx, (const T *)l.router, l.router_bias, l.router_bias_type, (int)l.rows, l.n_in, l.experts, logits);
    EP_CUDA(ctx, cudaGetLastError());
    return EP_OK;
}
template <typename T, bool VEC>
int launch_router(ep_ctx *ctx, const Layer &l, const Space &s, int r) {
    auto kernel = r == 1 ? experts_router<T, VEC, 1> : r == 2 ? experts_router<T, VEC, 2> : experts_router<T, VEC, 4>;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ROUTER_BLOCKS);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = l.stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = ROUTER_BLOCKS;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    EP_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, (const T *)l.x, l.ldx, (const T *)l.router, l.router_bias, l.router_bias_type, (int)l.rows,
                                    l.n_in, l.experts, s.logits, l.valid, l.k, l.renormalize, l.ids, l.weights, s.plan));
    return EP_OK;
}
template <typename T>
int run_layer(ep_ctx *ctx, const Layer &l, const Space &s, int *kernels) {
    const int size = sizeof(T), w_size = ep::type_size(l.w_type);
    const bool x_ready = sixteen(l.x, l.ldx, size);
    const bool router_ready = x_ready && sixteen(l.router, l.n_in, size);
    const int r = l.rows == 1 ? 1 : l.rows == 2 ? 2 : 4;
    if (l.rows * l.k <= FEW_SLOTS && ep::ceil_div(l.rows, r) * l.experts <= ROUTER_JOBS) {
        const int rc = router_ready ? launch_router<T, true>(ctx, l, s, r) : launch_router<T, false>(ctx, l, s, r);
        if (rc != EP_OK) return rc;
        *kernels = 3;
    } else {
        const int rc = router_ready ? launch_logits<T, true>(ctx, l, s.logits) : launch_logits<T, false>(ctx, l, s.logits);
        if (rc != EP_OK) return rc;
        EP_CUDA(ctx, ep::launch_early(experts_choose, dim3(1), dim3(1024), 0, l.stream, s.logits, l.valid, (int)l.rows, l.experts, l.k,
                                      l.renormalize, l.ids, l.weights, s.plan));
        *kernels = 4;
    }
    const bool vec = x_ready && sixteen(l.w1.w, l.n_in, w_size) && sixteen(l.w2.w, l.n_hidden, w_size);
    if constexpr (!std::is_same_v<T, float>) {
        if (vec && l.n_hidden % 8 == 0 && enough_for_tensor(l)) {
            if (l.w_type == EP_I8) {
                ++*kernels;
                return run_tensor<T, i8>(ctx, l, s);
            }
            if constexpr (std::is_same_v<T, __nv_bfloat16>) {
                ++*kernels;
                return run_tensor<T, T>(ctx, l, s);
            }
        }
    }
    if (l.w_type == EP_I8) return vec ? run_products<T, i8, true>(ctx, l, s) : run_products<T, i8, false>(ctx, l, s);
    return vec ? run_products<T, T, true>(ctx, l, s) : run_products<T, T, false>(ctx, l, s);
}

bool experts_shape_ok(int64_t rows, int n_in, int n_hidden, int n_out, int experts, int k) {
    auto width = [](int n) { return n >= 1 && n <= MAX_WIDTH; };
    return rows >= 0 && rows <= MAX_ROWS && width(n_in) && width(n_hidden) && width(n_out) && experts >= 1 && experts <= MAX_EXPERTS &&
           k >= 1 && k <= std::min(experts, MAX_K);
}

}  // namespace

using namespace ep;

namespace {
bool element_aligned(const void *p, int type) { return !p || aligned(p, (size_t)type_size(type)); }
}  // namespace

extern "C" {

size_t ep_experts_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t n_in, int32_t n_hidden, int32_t n_out, int32_t experts,
                                  int32_t k) {
    if (!ctx || !experts_shape_ok(rows, n_in, n_hidden, n_out, experts, k)) return 0;
    return space(rows, n_hidden, n_out, experts, k, nullptr).bytes;
}

int ep_experts(ep_ctx *ctx, const void *x, int64_t ldx, int32_t type, const void *router, const void *router_bias,
               int32_t router_bias_type, const uint8_t *valid, int32_t k, int32_t renormalize, const void *w1, const float *w1_scale,
               const void *b1, const void *w2, const float *w2_scale, const void *b2, int32_t w_type, int32_t bias_type, int32_t act,
               const void *residual, int64_t ldr, void *out, int32_t *ids, float *weights, int64_t rows, int32_t n_in,
               int32_t n_hidden, int32_t n_out, int32_t experts, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (rows > MAX_ROWS) return fail(ctx, EP_ERR_UNSUPPORTED, "%lld rows: a layer of experts takes up to %d", (long long)rows, MAX_ROWS);
    if (!experts_shape_ok(rows, n_in, n_hidden, n_out, experts, k))
        return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld, n_in %d, n_hidden %d, n_out %d, experts %d or k %d out of range", (long long)rows,
                    n_in, n_hidden, n_out, experts, k);
    if (!float_type(type) || (w_type != type && w_type != EP_I8) || (router_bias && !float_type(router_bias_type)) ||
        ((b1 || b2) && !float_type(bias_type)))
        return fail(ctx, EP_ERR_INVALID_ARG, "no experts of type %d for rows of type %d", w_type, type);
    if (act < EP_ACT_NONE || act > EP_ACT_SILU) return fail(ctx, EP_ERR_INVALID_ARG, "unknown activation %d", act);
    if (ldx < n_in || (residual && ldr < n_out)) return fail(ctx, EP_ERR_INVALID_ARG, "a row stride is shorter than its row");
    if (rows == 0) return EP_OK;
    if ((w_type == EP_I8) != (w1_scale != nullptr) || (w_type == EP_I8) != (w2_scale != nullptr))
        return fail(ctx, EP_ERR_INVALID_ARG, "scales go with 8-bit weights, and with no others");
    if (!x || !router || !w1 || !w2 || !out || !ids || !weights || !element_aligned(x, type) || !element_aligned(router, type) ||
        !element_aligned(w1, w_type) || !element_aligned(w2, w_type) || !element_aligned(out, type) || !element_aligned(residual, type) ||
        !element_aligned(router_bias, router_bias ? router_bias_type : EP_I8) || !element_aligned(b1, b1 ? bias_type : EP_I8) ||
        !element_aligned(b2, b2 ? bias_type : EP_I8) || !aligned(w1_scale, 4) || !aligned(w2_scale, 4) || !aligned(ids, 4) ||
        !aligned(weights, 4))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    const Space s = space(rows, n_hidden, n_out, experts, k, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes)
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    const Layer l{x,   ldx, type, router, router_bias, router_bias_type, valid, k, renormalize != 0, Weights{w1, w1_scale, b1, bias_type},
                  Weights{w2, w2_scale, b2, bias_type}, w_type, act, residual, ldr, out, ids, weights, rows, n_in, n_hidden, n_out,
                  experts, static_cast<cudaStream_t>(cuda_stream)};
    DeviceGuard guard(ctx->device);
    Timed tm(ctx, l.stream, EP_TIMER_EXPERTS);
    int kernels = 0;
    const int rc = type == EP_F32    ? run_layer<float>(ctx, l, s, &kernels)
                   : type == EP_BF16 ? run_layer<__nv_bfloat16>(ctx, l, s, &kernels)
                                     : run_layer<__half>(ctx, l, s, &kernels);
    tm.end(rc == EP_OK ? kernels : 0);
    return rc;
}

}  // extern "C"
