// A layer of experts for a few rows: router, the k best parts of each row, both products of every chosen part, their sum.
//
//     p = softmax(x Wr^T + br);  ids, w as ep_route;   out = sum_i w_i (W2[e_i] act(W1[e_i] x + b1[e_i]) + b2[e_i]) + residual
//
// What it costs is reading the chosen experts' weights, once each: slots (a row's choice of a part) are sorted by part, up to 8
// rows of one part make a group, and a warp that fetches a row of weights multiplies it with all rows of the group.  Sums
// are fp32 multiply-adds; the hidden values stay in fp32.
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
    __device__ __forceinline__ Pair pair(int i) const { return Pair(to_f32(e[2 * i]), to_f32(e[2 * i + 1])); }
};

// sum[j][r] = w_j . x_r over this lane's columns.
template <typename W, typename X, bool VEC, int J, int R>
__device__ __forceinline__ void dots(const W *const (&w)[J], const X *const (&x)[R], int from, int to, int n, int lane, float (&sum)[J][R]) {
    constexpr int N = 16 / (int)sizeof(W);
    Pair t[J][R];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) t[j][r] = Pair(0.f);
#pragma unroll 2
    for (int c = from; c < to; c += 32 * N) {
        Chunk<W, N, VEC> a[J];
#pragma unroll
        for (int j = 0; j < J; ++j) a[j].load(w[j], c, lane, n);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Chunk<X, N, VEC> b;
            b.load(x[r], c, lane, n);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const Pair v = b.pair(i);
#pragma unroll
                for (int j = 0; j < J; ++j) t[j][r] = fma2(a[j].pair(i), v, t[j][r]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float lo, hi;
            t[j][r].get(lo, hi);
            sum[j][r] = lo + hi;
        }
}
__device__ __forceinline__ float over_lanes(float v) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

// ---------------------------------------------------------------------------------------------- router
// logits[row][e] = x Wr^T + br: a warp to a part and up to 8 rows.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) experts_logits(const T *x, int64_t ldx, const T *router, const void *bias, int bias_type, int rows,
                                                      int n_in, int experts, float *logits) {
    const int lane = threadIdx.x & 31, e = blockIdx.x * 8 + (threadIdx.x >> 5), row0 = blockIdx.y * GROUP;
    ep_let_next_launch_start();
    if (e >= experts) return;
    const T *w[1] = {router + (int64_t)e * n_in};
    const T *xs[GROUP];
#pragma unroll
    for (int r = 0; r < GROUP; ++r) xs[r] = x + min(row0 + r, rows - 1) * ldx;
    const float add = bias ? load_param(bias, bias_type, e) : 0.f;
    if (rows - row0 == 1) {
        const T *one[1] = {xs[0]};
        float sum[1][1];
        dots<T, T, VEC, 1, 1>(w, one, 0, n_in, n_in, lane, sum);
        const float v = over_lanes(sum[0][0]);
        if (lane == 0) logits[row0 * experts + e] = v + add;
    } else {
        float sum[1][GROUP];
        dots<T, T, VEC, 1, GROUP>(w, xs, 0, n_in, n_in, lane, sum);
#pragma unroll
        for (int r = 0; r < GROUP; ++r) {
            const float v = over_lanes(sum[0][r]);
            if (lane == 0 && row0 + r < rows) logits[(row0 + r) * experts + e] = v + add;
        }
    }
}

// A row's k best parts and their weights (as ep_route), by one warp.
__device__ void choose(const float *l, int experts, int k, bool part, bool renormalize, int lane, int32_t *ids, float *weights) {
    float top = -INFINITY;
    if (part)
        for (int e = lane; e < experts; e += 32) top = fmaxf(top, l[e]);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
    part = part && top > -INFINITY;
    float s = 0.f;
    if (part)
        for (int e = lane; e < experts; e += 32) s += exp_fast(l[e] - top);
    s = over_lanes(s);
    float last = INFINITY, chosen = 0.f, mine = 0.f;
    int last_e = -1, mine_e = -1;
    for (int i = 0; i < k; ++i) {   // the best that comes after the one before: lower, or as high with a higher number
        float v = -INFINITY;
        int at = MAX_EXPERTS;
        if (part)
            for (int e = lane; e < experts; e += 32) {
                const float u = l[e];
                if (u > v && (u < last || (u == last && e > last_e))) {
                    v = u;
                    at = e;
                }
            }
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

// ---------------------------------------------------------------------------------------------- products
struct Weights {
    const void *w;
    const float *scale;   // of 8-bit integers
    const void *bias;
    int bias_type;
};

// hidden[place][j] = act(W1[e][j] . x + b1[e][j]): a warp to J rows of a part's weights.
template <typename T, typename W, bool VEC, int J, int R>
__device__ __forceinline__ void hidden_of(const T *x, int64_t ldx, const Weights &w1, int n_in, int n_hidden, int act, int k, const Plan &p,
                                          const Group &g, int j0, float *hidden, int lane) {
    const W *w[J];
    const T *xs[R];
#pragma unroll
    for (int j = 0; j < J; ++j) w[j] = static_cast<const W *>(w1.w) + ((int64_t)g.expert * n_hidden + min(j0 + j, n_hidden - 1)) * n_in;
#pragma unroll
    for (int r = 0; r < R; ++r) xs[r] = x + (p.sorted[g.first + min(r, g.count - 1)] / k) * ldx;
    float sum[J][R];
    dots<W, T, VEC, J, R>(w, xs, 0, n_in, n_in, lane, sum);
    // sum q of the J x R goes to lane q
    float v[1] = {0.f};
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float t = over_lanes(sum[j][r]);
            if (lane == j * R + r) v[0] = t;
        }
    const int j = j0 + lane / R, r = lane % R;
    if (lane < J * R && j < n_hidden && r < g.count) {
        const int64_t at = (int64_t)g.expert * n_hidden + j;
        if (w1.scale) v[0] *= w1.scale[at];
        if (w1.bias) v[0] += load_param(w1.bias, w1.bias_type, at);
        activate(v, act);
        hidden[(int64_t)(g.first + r) * n_hidden + j] = v[0];
    }
}
template <typename T, typename W, bool VEC>
__global__ void __launch_bounds__(THREADS) experts_hidden(const T *x, int64_t ldx, Weights w1, int n_in, int n_hidden, int act, int k, Plan p,
                                                          float *hidden) {
    constexpr int J = 4;
    const int lane = threadIdx.x & 31;
    ep_wait_for_launch_before();
    ep_let_next_launch_start();
    const int across = (n_hidden + J - 1) / J;
    const int64_t items = (int64_t)*p.n_groups * across, step = (int64_t)gridDim.x * WARPS;
    for (int64_t i = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5); i < items; i += step) {
        const Group g = p.groups[i / across];
        const int j0 = (int)(i % across) * J;
        if (g.count == 1)
            hidden_of<T, W, VEC, J, 1>(x, ldx, w1, n_in, n_hidden, act, k, p, g, j0, hidden, lane);
        else if (g.count == 2)
            hidden_of<T, W, VEC, J, 2>(x, ldx, w1, n_in, n_hidden, act, k, p, g, j0, hidden, lane);
        else if (g.count <= 4)
            hidden_of<T, W, VEC, J, 4>(x, ldx, w1, n_in, n_hidden, act, k, p, g, j0, hidden, lane);
        else
            hidden_of<T, W, VEC, J, 8>(x, ldx, w1, n_in, n_hidden, act, k, p, g, j0, hidden, lane);
    }
}

// y[share][place][column of the block] = W2[e][column] . hidden over one share of the hidden values.
template <typename W, bool VEC, int J, int R>
__device__ __forceinline__ void output_of(const Weights &w2, int n_hidden, int n_out, const Group &g, int col0, int from, int to, const float *hidden,
                                          float *y, int cols, int at, int lane) {
    const W *w[J];
    const float *xs[R];
#pragma unroll
    for (int j = 0; j < J; ++j) w[j] = static_cast<const W *>(w2.w) + ((int64_t)g.expert * n_out + min(col0 + j, n_out - 1)) * n_hidden;
#pragma unroll
    for (int r = 0; r < R; ++r) xs[r] = hidden + (int64_t)(g.first + min(r, g.count - 1)) * n_hidden;
    float sum[J][R];
    dots<W, float, VEC, J, R>(w, xs, from, to, to, lane, sum);
    float v = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float t = over_lanes(sum[j][r]);
            if (lane == j * R + r) v = t;
        }
    const int j = lane / R, r = lane % R;
    if (lane < J * R && at + j < cols && r < g.count) y[(g.first + r) * cols + at + j] = v;
}
// A block has `cols` columns of the output, of all rows; its warps share out groups, columns and shares of the hidden values.
template <typename T, typename W, bool VEC>
__global__ void __launch_bounds__(THREADS) experts_output(const float *hidden, Weights w2, int n_hidden, int n_out, int rows, int k, Plan p,
                                                          const int32_t *ids, const float *weights, const T *residual, int64_t ldr, T *out,
                                                          int cols, int shares, int per_share) {
    constexpr int J = 4;
    extern __shared__ float y[];   // [shares][rows * k][cols]
    const int lane = threadIdx.x & 31, slots = rows * k;
    const int col0 = blockIdx.x * cols, mine = min(cols, n_out - col0);
    ep_wait_for_launch_before();
    const int across = (mine + J - 1) / J;
    const int items = *p.n_groups * across * shares;
    for (int i = threadIdx.x >> 5; i < items; i += WARPS) {
        const int share = i % shares, q = i / shares;
        const Group g = p.groups[q / across];
        const int at = q % across * J;
        const int from = share * per_share, to = min(from + per_share, n_hidden);
        float *ys = y + share * slots * cols;
        if (g.count == 1)
            output_of<W, VEC, J, 1>(w2, n_hidden, n_out, g, col0 + at, from, to, hidden, ys, cols, at, lane);
        else if (g.count == 2)
            output_of<W, VEC, J, 2>(w2, n_hidden, n_out, g, col0 + at, from, to, hidden, ys, cols, at, lane);
        else if (g.count <= 4)
            output_of<W, VEC, J, 4>(w2, n_hidden, n_out, g, col0 + at, from, to, hidden, ys, cols, at, lane);
        else
            output_of<W, VEC, J, 8>(w2, n_hidden, n_out, g, col0 + at, from, to, hidden, ys, cols, at, lane);
    }
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
    float *logits, *hidden;
    Plan plan;
    size_t bytes;
};
Space space(int64_t rows, int n_hidden, int experts, int k, void *base) {
    ep::Arena a(base);
    Space s{};
    const size_t slots = rows * k;
    s.logits = a.take<float>(rows * experts);
    s.hidden = a.take<float>(slots * n_hidden);
    s.plan.n_groups = a.take<int>(1);
    s.plan.groups = a.take<Group>(slots);
    s.plan.sorted = a.take<int>(slots);
    s.plan.place = a.take<int>(slots);
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
}

template <typename T, typename W, bool VEC>
int run_products(ep_ctx *ctx, const Layer &l, const Space &s) {
    constexpr int STEP = 32 * 16 / (int)sizeof(W);   // columns that a warp takes at a time
    const int slots = (int)l.rows * l.k;
    EP_CUDA(ctx, ep::launch_early(experts_hidden<T, W, VEC>, dim3(ctx->sm_count), dim3(THREADS), 0, l.stream, (const T *)l.x, l.ldx, l.w1,
                                  l.n_in, l.n_hidden, l.act, l.k, s.plan, s.hidden));
    const int cols = std::max(1, std::min({(int)ep::ceil_div(l.n_out, ctx->sm_count), (int)(160 * 1024 / (sizeof(float) * slots)), 64}));
    // shares of the hidden values, so that every warp has something to do
    const int items = l.k * (int)ep::ceil_div(cols, 4);
    int shares = std::max(1, std::min({WARPS / items, (int)ep::ceil_div(l.n_hidden, 2 * STEP), (int)(160 * 1024 / (sizeof(float) * slots * cols))}));
    const int per_share = (int)ep::ceil_div(ep::ceil_div(l.n_hidden, shares), STEP) * STEP;
    shares = (int)ep::ceil_div(l.n_hidden, per_share);
    const size_t smem = sizeof(float) * shares * slots * cols;
    auto kernel = experts_output<T, W, VEC>;
    if (smem > 48 * 1024) EP_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    EP_CUDA(ctx, ep::launch_early(kernel, dim3((unsigned)ep::ceil_div(l.n_out, cols)), dim3(THREADS), smem, l.stream, s.hidden, l.w2, l.n_hidden,
                                  l.n_out, (int)l.rows, l.k, s.plan, l.ids, l.weights, (const T *)l.residual, l.ldr, (T *)l.out, cols,
                                  shares, per_share));
    return EP_OK;
}

bool sixteen(const void *p, int64_t ld, int size) { return ep::aligned(p, 16) && ld * size % 16 == 0; }

template <typename T>
int run_layer(ep_ctx *ctx, const Layer &l, const Space &s) {
    const int size = sizeof(T), w_size = ep::type_size(l.w_type);
    const bool x_ready = sixteen(l.x, l.ldx, size);
    const dim3 grid((unsigned)ep::ceil_div(l.experts, 8), (unsigned)ep::ceil_div(l.rows, GROUP));
    auto logits = x_ready && sixteen(l.router, l.n_in, size) ? experts_logits<T, true> : experts_logits<T, false>;
    logits<<<grid, 256, 0, l.stream>>>((const T *)l.x, l.ldx, (const T *)l.router, l.router_bias, l.router_bias_type, (int)l.rows, l.n_in,
                                       l.experts, s.logits);
    EP_CUDA(ctx, cudaGetLastError());
    EP_CUDA(ctx, ep::launch_early(experts_choose, dim3(1), dim3(1024), 0, l.stream, s.logits, l.valid, (int)l.rows, l.experts, l.k,
                                  l.renormalize, l.ids, l.weights, s.plan));
    const bool vec = x_ready && sixteen(l.w1.w, l.n_in, w_size) && sixteen(l.w2.w, l.n_hidden, w_size);
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
    return space(rows, n_hidden, experts, k, nullptr).bytes;
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
    const Space s = space(rows, n_hidden, experts, k, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes)
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    const Layer l{x,   ldx, type, router, router_bias, router_bias_type, valid, k, renormalize != 0, Weights{w1, w1_scale, b1, bias_type},
                  Weights{w2, w2_scale, b2, bias_type}, w_type, act, residual, ldr, out, ids, weights, rows, n_in, n_hidden, n_out,
                  experts, static_cast<cudaStream_t>(cuda_stream)};
    DeviceGuard guard(ctx->device);
    Timed tm(ctx, l.stream, EP_TIMER_EXPERTS);
    const int rc = type == EP_F32    ? run_layer<float>(ctx, l, s)
                   : type == EP_BF16 ? run_layer<__nv_bfloat16>(ctx, l, s)
                                     : run_layer<__half>(ctx, l, s);
    tm.end(rc == EP_OK ? 4 : 0);
    return rc;
}

}  // extern "C"
