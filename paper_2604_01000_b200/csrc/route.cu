// Routing of rows to parts: softmax, the k largest, counts per part and the balance loss in one pass over the logits;
// and its gradient, again in one pass.
//
// A row stays in the registers of the L threads that share it.  A thread holds the same columns of every row that it
// meets, so the sums over rows (of the probabilities) stay in its registers too until the block ends; counts are
// integers in shared memory.  Blocks leave their sums in the workspace and a second, small kernel adds them in a fixed
// order.  One block (few rows) needs neither: it writes the results itself.
//
// Measured: 2449029 rows of 32 fp32 logits, k = 1: 75 us, 4.4 TB/s (68 us the pass, 8 the fold), bound by instruction issue
// (19 instructions a logit, 0.7 issued a clock and scheduler); backward of 169343 x 257 bf16, k = 8, renormalised: 85 us, 2.2 TB/s
// (78 not renormalised: the divisions and one sum more make a row's only weight a constant exactly), bound alike: rows of 514 bytes start anywhere, so that logits are picked and stored one by one; one row of 64: 4 us.
#include "ep_common.cuh"
#include "rows.cuh"

#include <algorithm>

using namespace eprow;

namespace {

constexpr int MAX_PARTS = 4096;
constexpr int MAX_K = 32;
constexpr int THREADS = 256;
// Blocks that stay resident (2449029 rows of 32: 75 us; with 4 to an SM, and 64 registers a thread, 80).
constexpr int BLOCKS_PER_SM = 3;

// The better of two (logit, column) pairs: the larger logit, of equal ones the lower column.
__device__ __forceinline__ void keep_better(float &v, int &c, float ov, int oc) {
    const bool take = ov > v || (ov == v && oc < c);
    v = take ? ov : v;
    c = take ? oc : c;
}
// Order-preserving map of a float to an unsigned (not for NaN); -0 and +0 map alike.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// The best pair over L neighbouring lanes.
template <int L>
__device__ __forceinline__ void best_of_lanes(float &v, int &c) {
    if constexpr (L == 32) {
        const uint32_t key = ordered(v), top = __reduce_max_sync(FULL, key);
        c = (int)__reduce_min_sync(FULL, key == top ? (uint32_t)c : 0x7fffffffu);
        const uint32_t b = top ^ (top & 0x80000000u ? 0x80000000u : 0xffffffffu);
        v = __uint_as_float(b);
    } else {
#pragma unroll
        for (int o = L / 2; o >= 1; o >>= 1) {
            const float ov = __shfl_xor_sync(FULL, v, o);
            const int oc = __shfl_xor_sync(FULL, c, o);
            keep_better(v, c, ov, oc);
        }
    }
}

// e = exp(l - shift) of a thread's columns, and their sum.
template <int V, int N>
__device__ __forceinline__ float exponentials(const float (&l)[V][N], float shift, float (&e)[V][N]) {
    Pair sum(0.f);
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float a, b;
            mul2(add2(Pair(l[j][i], l[j][i + 1]), Pair(-shift)), Pair(1.44269504f)).get(a, b);
            e[j][i] = exp2_fast(a);
            e[j][i + 1] = exp2_fast(b);
            sum = add2(sum, Pair(e[j][i], e[j][i + 1]));
        }
    float lo, hi;
    sum.get(lo, hi);
    return lo + hi;
}

struct Finish {   // what the last step needs to turn sums into results
    int parts, k;
    int64_t *counts, *routed;
    float *prob, *loss;
};

// prob, loss and routed from the sums over all rows: one block.  counts[] and prob[] (as sums) are already there.
__device__ void finish_block(const Finish &f, int64_t rows_routed, double *red) {
    const double rows = rows_routed > 0 ? (double)rows_routed : 1.0;
    double t = 0.0;
    for (int e = threadIdx.x; e < f.parts; e += blockDim.x) {
        const float p = (float)((double)f.prob[e] / rows);
        f.prob[e] = p;
        t += (double)f.counts[e] * (double)p;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) t += __shfl_xor_sync(FULL, t, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        t = red[0];
        for (int w = 1; w < (int)(blockDim.x >> 5); ++w) t += red[w];
        *f.loss = (float)(t * (double)f.parts / ((double)f.k * rows));
        *f.routed = rows_routed;
    }
}

template <typename T, typename Lay>
__global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) route_rows(const T *__restrict__ logits, int64_t rows, int parts, int k,
                                                      const uint8_t *__restrict__ valid, bool renormalize,
                                                      int32_t *__restrict__ ids, float *weights,
                                                      float *__restrict__ part_prob, int *__restrict__ part_count,
                                                      unsigned *ticket, Finish fin, int hist_at, bool spans) {
    constexpr int L = Lay::L, V = Lay::V, N = Lay::N, WIDE = Lay::WIDE;
    constexpr int GROUPS = THREADS / L;
    __shared__ float slots[L > 32 ? 64 : 1];
    constexpr int WARPS = THREADS / 32;
    __shared__ float warp_v[L > 32 ? 2 * WARPS : 1];   // rows that a whole block shares: each warp's best, two slots in turn
    __shared__ int warp_c[L > 32 ? 2 * WARPS : 1];
    __shared__ double red[8];
    extern __shared__ uint4 ring[];   // rows on their way, later the fold of the sums; then counts
    int *hist = reinterpret_cast<int *>(reinterpret_cast<char *>(ring) + hist_at);   // of [parts + 1] (the last: rows that take part)
    int turn = 0;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    ep_let_next_launch_start();
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;   // of route_fold, which goes on after this kernel
    for (int e = threadIdx.x; e <= parts; e += THREADS) hist[e] = 0;
    __syncthreads();
    float sum_p[V][N];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) sum_p[j][i] = 0.f;
    int took_part = 0;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    RowStream<T, Lay, THREADS> stream(reinterpret_cast<char *>(ring), logits, rows, parts, lane, group, spans);
    stream.begin((int64_t)blockIdx.x * GROUPS, step);

    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < rows; first += step) {
        const int64_t row = first + group;
        const bool mine = row < rows;
        float l[V][N];
        stream.next(first, step, mine && (!valid || valid[row]), -INFINITY, l);
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, l[j][i]);
        top = reduce_row<L, OpMaxNumber>(top, slots, turn);
        const bool part = top > -INFINITY;   // false for a row of NaN and -infinity alone, too
        const float shift = part ? top : 0.f;   // (-infinity - 0: the exponentials of a row left out are zero)
        took_part += part && lane == 0;

        // the k largest, one after the other, while the logits are still there: each thread offers the best of its columns
        // that is not taken (the first is the lowest column that holds the maximum just found)
        uint32_t taken = 0;
        auto best_left = [&](float &v, int &c) {
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (l[j][i] > v && !(taken >> (j * N + i) & 1)) {
                        v = l[j][i];
                        c = Lay::col(lane, j, i);
                    }
        };
        float chosen = 0.f, mine_exp = 0.f;   // the sum of the slots' exponentials, and that of this thread's first slot
        // a wide row's threads keep the best that each of them has left: only the warp whose own was taken looks again
        float best_v = -INFINITY;
        int best_c = MAX_PARTS;
        if constexpr (L > 32) best_left(best_v, best_c);
        for (int r = 0; r < k; ++r) {
            float v = r == 0 ? top : -INFINITY;
            int c = MAX_PARTS;
            if constexpr (L > 32) {
                v = best_v;
                c = best_c;
                best_of_lanes<32>(v, c);
                float *sv = warp_v + (r & 1) * WARPS;
                int *sc = warp_c + (r & 1) * WARPS;
                if ((threadIdx.x & 31) == 0) {
                    sv[threadIdx.x >> 5] = v;
                    sc[threadIdx.x >> 5] = c;
                }
                __syncthreads();
                v = sv[0];
                c = sc[0];
#pragma unroll
                for (int w = 1; w < WARPS; ++w) keep_better(v, c, sv[w], sc[w]);
            } else if (r == 0) {
#pragma unroll
                for (int j = V - 1; j >= 0; --j)
#pragma unroll
                    for (int i = N - 1; i >= 0; --i)
                        if (l[j][i] == top) c = Lay::col(lane, j, i);
                if (c == MAX_PARTS) v = -INFINITY;
                best_of_lanes<L>(v, c);
            } else {
                best_left(v, c);
                best_of_lanes<L>(v, c);
            }
            const bool got = v > -INFINITY;
            const float ex = got ? exp_fast(v - top) : 0.f;
            chosen += ex;
            if (lane == r % L) {
                if (mine) {
                    ids[row * k + r] = got ? c : -1;
                    if (r >= L) weights[row * k + r] = ex;   // finished below, by this thread
                }
                if (r < L) mine_exp = ex;
                if (got) atomicAdd(&hist[c], 1);
            }
            if (got && r + 1 < k && Lay::owner(c) == lane) {
                taken |= 1u << Lay::index(c);
                if constexpr (L > 32) {
                    best_v = -INFINITY;
                    best_c = MAX_PARTS;
                    best_left(best_v, best_c);
                }
            }
        }
        static_assert(V * N <= 32, "a bit of `taken` for every column of a thread");

        const float s = reduce_row<L, OpSum>(exponentials(l, shift, l), slots, turn);
        const float inverse = part ? reciprocal_fast(s) : 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; i += 2)
                fma2(Pair(l[j][i], l[j][i + 1]), Pair(inverse), Pair(sum_p[j][i], sum_p[j][i + 1])).get(sum_p[j][i], sum_p[j][i + 1]);
        if (mine) {
            // over all columns or, renormalised, over the chosen ones (divided, not multiplied by a reciprocal: the weight
            // of a row's only slot is exactly 1).  A NaN or +infinity in the row makes both sums' quotients NaN.
            const float nan_too = s != s ? s : 0.f;
            auto weight = [&](float ex) { return renormalize ? (part ? ex / chosen + nan_too : 0.f) : ex * inverse; };
            if (lane < k) weights[row * k + lane] = weight(mine_exp);
            for (int r = lane + L; r < k; r += L) weights[row * k + r] = weight(weights[row * k + r]);
        }
    }

    // the block's sums: over its groups in order, then to the workspace or, alone, to the results
    stream.end();
    if (took_part) atomicAdd(&hist[parts], took_part);
    __syncthreads();
    float *fold = reinterpret_cast<float *>(ring);   // (every thread is past its last copy)
    const bool alone = gridDim.x == 1;
    float *prob_to = alone ? fin.prob : part_prob + (size_t)blockIdx.x * parts;
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) fold[group * WIDE + Lay::col(lane, j, i)] = sum_p[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < parts; c += THREADS) {
            float t = 0.f;
#pragma unroll 4
            for (int q = 0; q < GROUPS; ++q) t += fold[q * WIDE + c];
            prob_to[c] = t;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (Lay::col(lane, j, i) < parts) prob_to[Lay::col(lane, j, i)] = sum_p[j][i];
    }
    if (alone) {
        for (int c = threadIdx.x; c < parts; c += THREADS) fin.counts[c] = hist[c];
        __syncthreads();
        finish_block(fin, hist[parts], red);
    } else {
        int *count_to = part_count + (size_t)blockIdx.x * (parts + 1);
        for (int c = threadIdx.x; c <= parts; c += THREADS) count_to[c] = hist[c];
    }
}

// counts[c] and prob[c] over the blocks' shares; column `parts` is the number of rows that took part.  The block that
// finishes last (the ticket tells) turns the sums into the results.
__global__ void __launch_bounds__(1024) route_fold(const float *part_prob, const int *part_count, int n,
                                                  unsigned *ticket, Finish f) {
    __shared__ double sp[32][33];
    __shared__ long long sc[32][33];
    __shared__ bool last;
    const int lane = threadIdx.x & 31, r0 = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    ep_wait_for_launch_before();
    double p = 0.0;
    long long m = 0;
    if (c <= f.parts)
        for (int r = r0; r < n; r += 32 * 8) {   // 8 loads of each at a time, none of them alone at the end
            float v[8];
            int u[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const bool there = r + 32 * q < n;
                v[q] = there && c < f.parts ? part_prob[(size_t)(r + 32 * q) * f.parts + c] : 0.f;
                u[q] = there ? part_count[(size_t)(r + 32 * q) * (f.parts + 1) + c] : 0;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                p += (double)v[q];
                m += u[q];
            }
        }
    sp[r0][lane] = p;
    sc[r0][lane] = m;
    __syncthreads();
    p = sp[lane][r0];   // a warp per column now
    m = sc[lane][r0];
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        p += __shfl_xor_sync(FULL, p, o);
        m += __shfl_xor_sync(FULL, m, o);
    }
    const int mine = blockIdx.x * 32 + r0;
    __syncthreads();
    if (lane == 0) {   // sums of the block's columns to the first row
        sp[0][r0] = p;
        sc[0][r0] = m;
    }
    if (gridDim.x == 1) {   // (up to 31 parts: no other block to wait for)
        __syncthreads();
        if (r0 > 0) return;
        const double rows = (double)max(sc[0][f.parts], 1ll);
        double t = 0.0;
        if (lane < f.parts) {
            const float mean = (float)(sp[0][lane] / rows);
            f.prob[lane] = mean;
            f.counts[lane] = sc[0][lane];
            t = (double)sc[0][lane] * (double)mean;
        }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) t += __shfl_xor_sync(FULL, t, o);
        if (lane == 0) {
            *f.loss = (float)(t * (double)f.parts / ((double)f.k * rows));
            *f.routed = sc[0][f.parts];
        }
        return;
    }
    if (lane == 0) {
        if (mine < f.parts) {
            f.prob[mine] = (float)p;
            f.counts[mine] = m;
        } else if (mine == f.parts)
            *f.routed = m;
        __threadfence();
    }
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    finish_block(f, *(volatile int64_t *)f.routed, &sp[0][0]);
}

template <typename T, typename Lay>
__global__ void __launch_bounds__(THREADS, BLOCKS_PER_SM) route_rows_backward(const T *__restrict__ logits, int64_t rows, int parts, int k,
                                                               const uint8_t *__restrict__ valid, bool renormalize,
                                                               const int32_t *__restrict__ ids,
                                                               const int64_t *__restrict__ counts,
                                                               const int64_t *__restrict__ routed,
                                                               const float *__restrict__ dweights,
                                                               const float *__restrict__ dloss, T *__restrict__ dlogits,
                                                               int *status, bool spans) {
    constexpr int L = Lay::L, V = Lay::V, N = Lay::N;
    constexpr int GROUPS = THREADS / L;
    __shared__ float slots[L > 32 ? 64 : 1];
    int turn = 0;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    float slope[V][N];   // d loss / d p of this thread's columns, the same for every row
    float unit = 0.f;
    if (dloss) {
        const double r = (double)max((long long)*routed, 1ll);
        unit = (float)((double)*dloss * (double)parts / ((double)k * r * r));
    }
    const bool endless = !(fabsf(unit) < 1e28f);   // slopes may not be finite: a row that takes no part is not zero times them
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = Lay::col(lane, j, i);
            slope[j][i] = dloss && c < parts ? unit * (float)counts[c] : 0.f;
        }
    extern __shared__ uint4 ring[];
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    RowStream<T, Lay, THREADS> stream(reinterpret_cast<char *>(ring), logits, rows, parts, lane, group, spans);
    stream.begin((int64_t)blockIdx.x * GROUPS, step);
    // what the next row needs besides its logits, a step ahead: whether it takes part, and this thread's first slot
    struct Ahead {
        bool read;
        int id;
        float dw;
    };
    auto look = [&](int64_t row) {
        Ahead a{row < rows && (!valid || valid[row]), -1, 0.f};
        if (dweights && row < rows && lane < k) {
            a.id = ids[row * k + lane];
            a.dw = dweights[row * k + lane];
        }
        return a;
    };
    Ahead ahead = look((int64_t)blockIdx.x * GROUPS + group);
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < rows; first += step) {
        const int64_t row = first + group;
        const bool mine = row < rows;
        const Ahead now = ahead;
        ahead = look(row + step);
        float p[V][N];
        stream.next(first, step, now.read, -INFINITY, p);
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, p[j][i]);
        top = reduce_row<L, OpMaxNumber>(top, slots, turn);
        const bool part = top > -INFINITY;
        const float shift = part ? top : 0.f;
        float s = exponentials(p, shift, p), dot;
        {
            Pair both(0.f);
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < N; i += 2) both = fma2(Pair(p[j][i], p[j][i + 1]), Pair(slope[j][i], slope[j][i + 1]), both);
            float odd;
            both.get(dot, odd);
            dot += odd;
        }
        s = reduce_row<L, OpSum>(s, slots, turn);
        dot = reduce_row<L, OpSum>(dot, slots, turn);
        const float inverse = part ? reciprocal_fast(s) : 0.f;
        dot *= inverse;
        // The slots, shared out over the row's threads; a thread keeps its first.  Renormalised: the sum of their p, then
        // the mean of dweights by p / sum (in this order: where a row's weights are constants, what reaches them cancels
        // exactly); otherwise the sum of dweights p.
        float chosen = 0.f, pulled = 0.f, first_w = 0.f;
        int first_id = -1;
        if (dweights) {
            if constexpr (L <= 32) __syncwarp();   // (wider rows have met at a sum)
            auto slot = [&](int id) {
                if (id < 0 || id >= parts) {
                    if (id != -1) ep_raise(status, EP_ERR_BAD_INDEX);
                    return 0.f;
                }
                return exp_fast(stream.element(first, id) - top) * inverse;
            };
            auto slots_after_first = [&](auto f) {
                for (int q = lane + L; q < k; q += L) f(slot(ids[row * k + q]), dweights[row * k + q]);
            };
            auto times = [](float w, float dw) { return w > 0.f ? dw * w : w; };   // (an empty slot's dw may be anything)
            if (part) {
                first_w = slot(now.id);
                first_id = now.id < parts ? now.id : -1;
                if (renormalize) {
                    chosen = first_w;
                    slots_after_first([&](float w, float) { chosen += w; });
                } else {
                    pulled = times(first_w, now.dw);
                    slots_after_first([&](float w, float dw) { pulled += times(w, dw); });
                }
            }
            if (renormalize) {
                chosen = reduce_row<L, OpSum>(chosen, slots, turn);
                if (part && chosen > 0.f) {
                    pulled = times(first_w / chosen, now.dw);
                    slots_after_first([&](float w, float dw) { pulled += times(w / chosen, dw); });
                }
            }
            pulled = reduce_row<L, OpSum>(pulled, slots, turn);
        }
        // with renormalised weights the slots' own terms of sum_e p_e dp_e cancel
        const float back = renormalize ? dot : dot + pulled;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; i += 2)
                mul2(mul2(Pair(p[j][i], p[j][i + 1]), Pair(inverse)), add2(Pair(slope[j][i], slope[j][i + 1]), Pair(-back)))
                    .get(p[j][i], p[j][i + 1]);
        if (endless && !part) Lay::set(0.f, p);
        T *to = dlogits + row * parts;
        if (mine) Lay::store(to, lane, parts, p);
        if (!dweights) continue;
        // the chosen columns once more, with their slots' terms: over what the row's threads have just stored
        if constexpr (L > 32)
            __syncthreads();
        else
            __syncwarp();
        if (part) {
            const float mean = renormalize ? pulled : 0.f, per = renormalize ? 1.f / chosen : 1.f;
            auto again = [&](int id, float w, float dw) {
                const float own = dloss ? unit * (float)counts[id] : 0.f;
                to[id] = from_f32<T>(w * (own + (dw - mean) * per - back));
            };
            if (first_id >= 0) again(first_id, first_w, now.dw);
            for (int q = lane + L; q < k; q += L) {
                const int id = ids[row * k + q];
                if (id >= 0 && id < parts) again(id, exp_fast(stream.element(first, id) - top) * inverse, dweights[row * k + q]);
            }
        }
        if constexpr (L > 32)   // the row's logits are no longer read
            __syncthreads();
        else
            __syncwarp();
    }
    stream.end();
}

template <typename Lay>
int grid_for(const ep_ctx *ctx, int64_t rows) {
    return (int)std::max<int64_t>(1, std::min<int64_t>(ep::ceil_div(rows, THREADS / Lay::L), (int64_t)ctx->sm_count * BLOCKS_PER_SM));
}

struct RouteArgs {
    ep_ctx *ctx;
    const void *logits;
    int64_t rows;
    int parts, k;
    const uint8_t *valid;
    bool renormalize;
    int32_t *ids;
    float *weights;
    float *part_prob;
    int *part_count;
    unsigned *ticket;
    Finish fin;
    cudaStream_t stream;
    int kernels;
};

template <typename T>
struct RouteLaunch {
    static constexpr int MAX_WIDTH = MAX_PARTS;
    RouteArgs &a;
    template <typename Lay>
    int run() const {
        constexpr int groups = THREADS / Lay::L;
        const size_t hist_at = std::max((size_t)RowStream<T, Lay, THREADS>::ring_bytes(a.parts),
                                        groups > 1 ? sizeof(float) * groups * Lay::WIDE : 0);
        const size_t smem = hist_at + sizeof(int) * (size_t)(a.parts + 1);
        // (two rounds of one block are quicker than two blocks and the fold after them: 128 x 64 fp32 in 5.0 us against 7.3)
        const int grid = a.rows <= 2 * groups ? 1 : grid_for<Lay>(a.ctx, a.rows);
        if (smem > 40 * 1024)   // (static shared memory counts too)
            EP_CUDA(a.ctx, cudaFuncSetAttribute(route_rows<T, Lay>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        route_rows<T, Lay><<<grid, THREADS, smem, a.stream>>>((const T *)a.logits, a.rows, a.parts, a.k, a.valid,
                                                                       a.renormalize, a.ids, a.weights, a.part_prob, a.part_count,
                                                                       a.ticket, a.fin, (int)hist_at, ep::aligned(a.logits, 16));
        EP_CUDA(a.ctx, cudaGetLastError());
        a.kernels = 1;
        if (grid > 1) {
            EP_CUDA(a.ctx, ep::launch_early(route_fold, dim3(a.parts / 32 + 1), dim3(1024), 0, a.stream, (const float *)a.part_prob,
                                            (const int *)a.part_count, grid, a.ticket, a.fin));
            a.kernels = 2;
        }
        return EP_OK;
    }
};

struct RouteBackArgs {
    ep_ctx *ctx;
    const void *logits;
    int64_t rows;
    int parts, k;
    const uint8_t *valid;
    bool renormalize;
    const int32_t *ids;
    const int64_t *counts, *routed;
    const float *dweights, *dloss;
    void *dlogits;
    cudaStream_t stream;
};

template <typename T>
struct RouteBackLaunch {
    static constexpr int MAX_WIDTH = MAX_PARTS;
    const RouteBackArgs &a;
    template <typename Lay>
    int run() const {
        const int smem = RowStream<T, Lay, THREADS>::ring_bytes(a.parts);
        if (smem > 40 * 1024)   // (static shared memory counts too)
            EP_CUDA(a.ctx, cudaFuncSetAttribute(route_rows_backward<T, Lay>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        route_rows_backward<T, Lay><<<grid_for<Lay>(a.ctx, a.rows), THREADS, smem, a.stream>>>(
            (const T *)a.logits, a.rows, a.parts, a.k, a.valid, a.renormalize, a.ids, a.counts, a.routed, a.dweights, a.dloss,
            (T *)a.dlogits, a.ctx->d_status, ep::aligned(a.logits, 16));
        EP_CUDA(a.ctx, cudaGetLastError());
        return EP_OK;
    }
};

bool route_shape_ok(int64_t rows, int parts) { return rows >= 0 && rows < (1ll << 31) && parts >= 1 && parts <= MAX_PARTS; }

struct RouteWorkspace {
    float *prob;
    int *count;
    unsigned *ticket;
    size_t bytes;
};

RouteWorkspace route_workspace(const ep_ctx *ctx, int parts, void *p) {
    ep::Arena a(p);
    RouteWorkspace w{};
    const size_t blocks = (size_t)ctx->sm_count * BLOCKS_PER_SM;
    w.prob = a.take<float>(blocks * parts);
    w.count = a.take<int>(blocks * (parts + 1));
    w.ticket = a.take<unsigned>(1);
    w.bytes = a.used;
    return w;
}

}  // namespace

using namespace ep;

extern "C" {

size_t ep_route_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t parts) {
    if (!ctx || !route_shape_ok(rows, parts)) return 0;
    return route_workspace(ctx, parts, nullptr).bytes;
}

int ep_route(ep_ctx *ctx, const void *logits, int32_t type, int64_t rows, int32_t parts, int32_t k, const uint8_t *valid,
             int32_t renormalize, int32_t *ids, float *weights, int64_t *counts, float *prob, float *loss, int64_t *routed,
             void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (!route_shape_ok(rows, parts))
        return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld or parts %d out of range", (long long)rows, parts);
    if (k < 1 || k > std::min(parts, MAX_K)) return fail(ctx, EP_ERR_INVALID_ARG, "k %d out of range for %d parts", k, parts);
    if (!float_type(type)) return fail(ctx, EP_ERR_INVALID_ARG, "logits of type %d are not supported", type);
    if (!counts || !prob || !loss || !routed || !aligned(counts, 8) || !aligned(prob, 4) || !aligned(loss, 4) || !aligned(routed, 8))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    DeviceGuard guard(ctx->device);
    if (rows == 0) {
        EP_CUDA(ctx, cudaMemsetAsync(counts, 0, sizeof(int64_t) * (size_t)parts, stream));
        EP_CUDA(ctx, cudaMemsetAsync(prob, 0, sizeof(float) * (size_t)parts, stream));
        EP_CUDA(ctx, cudaMemsetAsync(loss, 0, sizeof(float), stream));
        EP_CUDA(ctx, cudaMemsetAsync(routed, 0, sizeof(int64_t), stream));
        return EP_OK;
    }
    if (!logits || !ids || !weights || !aligned(logits, type_size(type)) || !aligned(ids, 4) || !aligned(weights, 4))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    const RouteWorkspace w = route_workspace(ctx, parts, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < w.bytes)
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    RouteArgs a{ctx, logits, rows, parts, k, valid, renormalize != 0, ids, weights, w.prob, w.count,
                w.ticket, Finish{parts, k, counts, routed, prob, loss}, stream, 0};
    const bool vec = parts % (16 / type_size(type)) == 0 && aligned(logits, 16);
    Timed tm(ctx, stream, EP_TIMER_ROUTE);
    const int rc = type == EP_F32    ? with_layout<float>(parts, vec, RouteLaunch<float>{a})
                   : type == EP_BF16 ? with_layout<__nv_bfloat16>(parts, vec, RouteLaunch<__nv_bfloat16>{a})
                                     : with_layout<__half>(parts, vec, RouteLaunch<__half>{a});
    tm.end(a.kernels);
    return rc;
}

int ep_route_backward(ep_ctx *ctx, const void *logits, int32_t type, int64_t rows, int32_t parts, int32_t k,
                      const uint8_t *valid, int32_t renormalize, const int32_t *ids, const int64_t *counts,
                      const int64_t *routed, const float *dweights, const float *dloss, void *dlogits, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (!route_shape_ok(rows, parts))
        return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld or parts %d out of range", (long long)rows, parts);
    if (k < 1 || k > std::min(parts, MAX_K)) return fail(ctx, EP_ERR_INVALID_ARG, "k %d out of range for %d parts", k, parts);
    if (!float_type(type)) return fail(ctx, EP_ERR_INVALID_ARG, "logits of type %d are not supported", type);
    if (rows == 0) return EP_OK;
    if (!logits || !ids || !counts || !routed || !dlogits || !aligned(logits, type_size(type)) || !aligned(ids, 4) ||
        !aligned(counts, 8) || !aligned(routed, 8) || !aligned(dweights, 4) || !aligned(dloss, 4) ||
        !aligned(dlogits, type_size(type)))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    RouteBackArgs a{ctx, logits, rows, parts, k, valid, renormalize != 0, ids, counts, routed, dweights, dloss, dlogits,
                    static_cast<cudaStream_t>(cuda_stream)};
    const bool vec = parts % (16 / type_size(type)) == 0 && aligned(logits, 16) && aligned(dlogits, 16);
    DeviceGuard guard(ctx->device);
    Timed tm(ctx, a.stream, EP_TIMER_ROUTE);
    const int rc = type == EP_F32    ? with_layout<float>(parts, vec, RouteBackLaunch<float>{a})
                   : type == EP_BF16 ? with_layout<__nv_bfloat16>(parts, vec, RouteBackLaunch<__nv_bfloat16>{a})
                                     : with_layout<__half>(parts, vec, RouteBackLaunch<__half>{a});
    tm.end(rc == EP_OK ? 1 : 0);
    return rc;
}

}  // extern "C"
