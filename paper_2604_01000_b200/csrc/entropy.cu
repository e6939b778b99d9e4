// Softmax cross entropy of x W^T + b over many classes, and its gradient; the logits only ever exist a piece at a time.
//
//     l = x W^T + b;   lse = log sum_c exp l_c;   row_loss = lse - l_target;   loss = mean of row_loss over the rows that count
//     G = (exp(l - lse) - [c = target]) g,  g = dloss / rows + drow;   dx = G W;   dW = G^T x;   db = column sums of G
//
// A piece (some rows by some classes) of logits is made by the products' tile kernel and stays in the L2; the row
// kernels here go over it: the forward's keep a running maximum and sum for each row, the backward's make G of it, in the
// operands' type, for two more products.
#include "ep_common.cuh"
#include "rows.cuh"

#include <algorithm>

using namespace eprow;
using ep::Matrix;
using ep::Operand;
using ep::Packed;

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

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

// ---------------------------------------------------------------------------------------------- forward
// The statistics of rows over one piece of classes, added to those of the pieces before (first: there are none).
// WARPS warps to a row.
template <int WARPS>
__global__ void __launch_bounds__(256) entropy_rows(const float *__restrict__ logits, int ld, int64_t rows, int classes, int class0,
                                                    const void *__restrict__ bias, int bias_type, const int32_t *__restrict__ targets,
                                                    bool first, float2 *running, float *at_target) {
    __shared__ Running part[8];
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

// lse and loss of each row from its statistics, and each block's sum of losses and count of rows that take part.
constexpr int FINISH_ROWS = 1024;   // a block's
__global__ void __launch_bounds__(256) entropy_finish(const float2 *__restrict__ running, const float *__restrict__ at_target,
                                                      const int32_t *__restrict__ targets, int64_t rows, int classes, float *lse,
                                                      float *row_loss, double *sums, long long *counts, int *status) {
    __shared__ double sum[8];
    __shared__ int count[8];
    double total = 0.0;
    int live = 0;
    for (int i = threadIdx.x; i < FINISH_ROWS; i += 256) {
        const int64_t row = (int64_t)blockIdx.x * FINISH_ROWS + i;
        if (row >= rows) break;
        float z = 0.f, loss = 0.f;
        if (target_of(targets, row, classes, status) >= 0) {
            const float2 r = running[row];
            z = r.x + logf(r.y);
            if (r.x == -INFINITY && r.y == 0.f)   // every class is closed: the row takes no part
                z = -INFINITY;
            else {
                loss = z - at_target[row];
                ++live;
            }
        }
        lse[row] = z;
        row_loss[row] = loss;
        total += (double)loss;
    }
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
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) {
            total += sum[w];
            live += count[w];
        }
        sums[blockIdx.x] = total;
        counts[blockIdx.x] = live;
    }
}
__global__ void __launch_bounds__(256) entropy_mean(const double *__restrict__ sums, const long long *__restrict__ counts, int blocks,
                                                    float *loss, long long *counted) {
    __shared__ double sum[8];
    __shared__ long long count[8];
    double total = 0.0;
    long long live = 0;
    for (int i = threadIdx.x; i < blocks; i += 256) {
        total += sums[i];
        live += counts[i];
    }
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
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) {
            total += sum[w];
            live += count[w];
        }
        *loss = (float)(total / (double)(live > 0 ? live : 1));
        *counted = live;
    }
}

// ---------------------------------------------------------------------------------------------- backward
// The rows' weights g (0 for rows that take no part), and each block's largest finite |g|.  A row that takes no part counts for
// nothing, whatever x holds there; but 0 times an infinity or a NaN is NaN, so such rows of x are looked through: a block's
// unclean is 1 where one holds any, and dW is then made of a copy of x with zeros there.
template <typename T>
__global__ void __launch_bounds__(256) entropy_weights(const float *__restrict__ lse, const int32_t *__restrict__ targets, int64_t rows,
                                                       int classes, const long long *__restrict__ counted,
                                                       const float *__restrict__ dloss, const float *__restrict__ drow,
                                                       const T *__restrict__ x, int64_t ldx, int n_in, float *weights, float *peaks,
                                                       int *unclean, int *status) {
    __shared__ int bad_rows;
    __shared__ float tops[8];
    const double mean = dloss ? (double)*dloss / (double)(*counted > 0 ? *counted : 1) : 0.0;   // (the two terms may cancel)
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) bad_rows = 0;
    __syncthreads();
    float top = 0.f;
    for (int64_t row0 = (int64_t)blockIdx.x * 256; row0 < rows; row0 += (int64_t)gridDim.x * 256) {
        const int64_t row = row0 + threadIdx.x;
        bool dead = false;
        if (row < rows) {
            dead = target_of(targets, row, classes, status) < 0 || lse[row] == -INFINITY;
            const float g = dead ? 0.f : (float)(mean + (drow ? (double)drow[row] : 0.0));
            weights[row] = g;
            if (fabsf(g) < INFINITY) top = fmaxf(top, fabsf(g));
        }
        if (!x) continue;
        for (unsigned left = __ballot_sync(FULL, dead); left; left &= left - 1) {
            const T *from = x + (row0 + (threadIdx.x & ~31) + __ffs(left) - 1) * ldx;
            bool bad = false;
            for (int c = lane; c < n_in; c += 32) bad |= !(fabsf(to_f32(from[c])) < INFINITY);
            if (bad) bad_rows = 1;
        }
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
    if (lane == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) top = fmaxf(top, tops[w]);
        peaks[blockIdx.x] = top;
        unclean[blockIdx.x] = bad_rows;
    }
}

// What the blocks of entropy_weights have found, together.  fp16 holds nothing below 2^-25, where a mean over many rows puts
// whole gradients: G is multiplied by the power of two that brings the largest |g| to [2^14, 2^15) (|p - 1| is at most 1), and
// the products' sums by its inverse.
struct Scale {
    float up, down;
    int unclean;
};
__global__ void __launch_bounds__(256) entropy_scale(const float *__restrict__ peaks, const int *__restrict__ unclean, int n, bool scaled,
                                                     Scale *out) {
    __shared__ float tops[8];
    float top = 0.f;
    bool bad = false;
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
        const int up = scaled && top > 0.f ? min(14 - ilogbf(top), 126) : 0;
        *out = Scale{scalbnf(1.f, up), scalbnf(1.f, -up), any};
    }
}

// x with zeros in the rows that take no part (see entropy_weights).  from: x, copied only if a row needs it; NULL: `to` is a
// copy of x already, of `parts` matrices.
template <typename E>
__global__ void __launch_bounds__(256) entropy_clean(const E *__restrict__ from, int64_t ld, int64_t rows, int cols,
                                                     const int32_t *__restrict__ targets, const float *__restrict__ lse, int classes,
                                                     const Scale *scale, E *to, int ld_to, int parts, int64_t part_stride) {
    if (!scale->unclean) return;
    const int lane = threadIdx.x & 31;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows; row += (int64_t)gridDim.x * 8) {
        const int t = targets[row];
        const bool dead = t < 0 || t >= classes || lse[row] == -INFINITY;
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
                                                      const void *__restrict__ bias, int bias_type, const int32_t *__restrict__ targets,
                                                      const float *__restrict__ lse, const float *__restrict__ weights,
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
            const float g = weights[row], z = lse[row];
            const int mine = g != 0.f ? targets[row] - class0 : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = exp_fast(v[i] + b[i] - z) - (col + i == mine ? 1.f : 0.f);
                v[i] = g != 0.f && col + i < classes ? p * g : 0.f;
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

// ---------------------------------------------------------------------------------------------- host side
constexpr int MAX_WIDTH = 65536, MAX_CLASSES = 1 << 24;
constexpr int64_t PIECE = 1 << 24;   // elements of a piece

// Rows x classes in pieces; of the shorter side as much as goes, so that little of what is summed over pieces is large.
struct Pieces {
    int64_t rows;
    int classes;
    int64_t across;   // pieces along the rows
    int down;         // and along the classes
};
Pieces make_pieces(int64_t rows, int classes) {
    Pieces p;
    auto up = [](int64_t v) { return std::max<int64_t>(1, (v + 255) / 256) * 256; };
    if (rows >= classes) {
        p.classes = std::min(classes, 16384);
        p.rows = std::min(rows, std::max<int64_t>(256, PIECE / up(p.classes) / 256 * 256));
    } else {
        p.rows = std::min<int64_t>(rows, 16384);
        p.classes = (int)std::min<int64_t>(classes, std::max<int64_t>(256, PIECE / up(p.rows) / 256 * 256));
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

struct ForwardSpace {
    void *x, *w;
    float *logits, *share, *at_target;
    float2 *running;
    double *sums;
    long long *counts;
    Pieces pieces;
    size_t bytes;
};
ForwardSpace forward_space(const ep_ctx *ctx, int64_t rows, int n_in, int classes, int type, bool aligned, void *base) {
    ep::Arena a(base);
    ForwardSpace s{};
    s.pieces = make_pieces(rows, classes);
    if (type == EP_F32 || !aligned) {
        s.x = a.take<char>(ep::packed_form(rows, n_in, type).bytes);
        s.w = a.take<char>(ep::packed_form(classes, n_in, type).bytes);
    }
    if (rows) {
        s.logits = a.take<float>(s.pieces.rows * padded(s.pieces.classes));
        s.share = a.take<float>(most_of(s.pieces, rows, classes, [&](int64_t r, int c) { return ep::product_bytes(ctx, r, padded(c), n_in, type, EP_F32); }) / 4);
    }
    s.at_target = a.take<float>(rows);
    s.running = a.take<float2>(rows);
    s.sums = a.take<double>(ep::ceil_div(rows, FINISH_ROWS));
    s.counts = a.take<long long>(ep::ceil_div(rows, FINISH_ROWS));
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
}

struct Backward {
    void *x, *w;          // copies
    void *g;
    float *logits, *share, *dx, *dweight, *part, *weights, *peaks;
    int *unclean;
    Scale *scale;
    Pieces pieces;
    int blocks;           // of entropy_weights
    int slabs;            // of a piece's rows, for the columns' sums
    size_t bytes;
};
Backward backward_space(const ep_ctx *ctx, int64_t rows, int n_in, int classes, int type, bool aligned, void *base) {
    ep::Arena a(base);
    Backward s{};
    s.pieces = make_pieces(rows, classes);
    const Pieces &p = s.pieces;
    const Packed x = ep::packed_form(rows, n_in, type);
    s.x = a.take<char>(x.bytes);   // (of aligned 16-bit x too: see entropy_clean)
    if (type == EP_F32 || !aligned) s.w = a.take<char>(ep::packed_form(classes, n_in, type).bytes);
    if (rows) {
        s.g = a.take<char>(ep::packed_form(p.rows, p.classes, type).bytes);
        s.logits = a.take<float>(p.rows * padded(p.classes));
        s.share = a.take<float>(most_of(p, rows, classes, [&](int64_t r, int c) {
                                    size_t most = ep::product_bytes(ctx, r, padded(c), n_in, type, EP_F32);
                                    for (int out : {type, (int)EP_F32}) {
                                        most = std::max(most, ep::product_bytes(ctx, r, n_in, c, type, out));
                                        most = std::max(most, ep::product_bytes(ctx, c, n_in, r, type, out));
                                    }
                                    return most;
                                }) / 4);
        if (type != EP_F32 && p.down > 1) s.dx = a.take<float>(p.rows * n_in);
        if (type != EP_F32 && p.across > 1) s.dweight = a.take<float>((int64_t)classes * n_in);
        const int want = std::max(1, ctx->sm_count * 4 / (int)ep::ceil_div(p.classes, G_CHUNKS * 8));
        s.slabs = (int)std::max<int64_t>(1, std::min<int64_t>(want, ep::ceil_div(p.rows, 2 * G_ROWS)));
        s.part = a.take<float>((size_t)p.across * s.slabs * classes);
    }
    s.weights = a.take<float>(rows);
    s.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(ep::ceil_div(rows, 256), ctx->sm_count * 2));
    s.peaks = a.take<float>(s.blocks);
    s.unclean = a.take<int>(s.blocks);
    s.scale = a.take<Scale>(1);
    s.bytes = std::max<size_t>(a.used, 256);
    return s;
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

// `rows` of an operand from row `first` on.
Operand rows_of(Operand o, int64_t first, int64_t rows) {
    o.base = static_cast<const char *>(o.base) + first * o.ld * ep::type_size(o.type);
    o.rows = rows;
    return o;
}

int operands(ep_ctx *ctx, Inputs &in, void *x_room, void *w_room, Operand *x, Operand *w) {
    *x = Operand{in.x, in.type, in.rows, in.n_in, in.ldx, 1, 0};
    *w = Operand{in.w, in.type, in.classes, in.n_in, in.ldw, 1, 0};
    if (in.type != EP_F32 && in.aligned) return EP_OK;
    return ep::make_operands(ctx, Matrix{in.x, in.ldx, in.rows, in.n_in, x_room}, Matrix{in.w, in.ldw, in.classes, in.n_in, w_room},
                             in.type, in.stream, x, w, &in.kernels);
}

int logits_of(ep_ctx *ctx, Inputs &in, const Operand &x, const Operand &w, int64_t row0, int64_t rows, int class0, int classes,
              float *logits, float *share) {
    return ep::product(ctx, rows_of(x, row0, rows), false, rows_of(w, class0, classes), false, rows, padded(classes), in.n_in, logits,
                       EP_F32, false, nullptr, share, in.stream, &in.kernels);
}

int forward_run(ep_ctx *ctx, Inputs &in, const ForwardSpace &s, float *loss, float *row_loss, float *lse, long long *counted) {
    Operand x, w;
    int rc = operands(ctx, in, s.x, s.w, &x, &w);
    const Pieces &p = s.pieces;
    for (int64_t row0 = 0; rc == EP_OK && row0 < in.rows; row0 += p.rows)
        for (int class0 = 0; class0 < in.classes; class0 += p.classes) {
            const int64_t rows = std::min(p.rows, in.rows - row0);
            const int classes = std::min(p.classes, in.classes - class0);
            rc = logits_of(ctx, in, x, w, row0, rows, class0, classes, s.logits, s.share);
            if (rc != EP_OK) return rc;
            const bool wide = classes > 2048 || rows < 8 * ctx->sm_count;
            auto kernel = wide ? entropy_rows<8> : entropy_rows<1>;
            kernel<<<(unsigned)ep::ceil_div(rows, wide ? 1 : 8), 256, 0, in.stream>>>(
                s.logits, padded(classes), rows, classes, class0, in.bias, in.bias_type, in.targets + row0, class0 == 0,
                s.running + row0, s.at_target + row0);
            EP_CUDA(ctx, cudaGetLastError());
            ++in.kernels;
        }
    if (rc != EP_OK) return rc;
    const int blocks = (int)ep::ceil_div(in.rows, FINISH_ROWS);
    entropy_finish<<<blocks, 256, 0, in.stream>>>(s.running, s.at_target, in.targets, in.rows, in.classes, lse, row_loss, s.sums,
                                                  s.counts, ctx->d_status);
    entropy_mean<<<1, 256, 0, in.stream>>>(s.sums, s.counts, blocks, loss, counted);
    EP_CUDA(ctx, cudaGetLastError());
    in.kernels += 2;
    return EP_OK;
}

struct Given {
    const float *lse, *dloss, *drow;
    const long long *counted;
};
struct Wanted {
    void *dx, *dweight;
    float *dbias;
};

template <typename T>
void launch_weights(ep_ctx *ctx, const Inputs &in, const Backward &s, const Given &g, bool look) {
    entropy_weights<T><<<s.blocks, 256, 0, in.stream>>>(g.lse, in.targets, in.rows, in.classes, g.counted, g.dloss, g.drow,
                                                        look ? (const T *)in.x : nullptr, in.ldx, in.n_in, s.weights, s.peaks, s.unclean,
                                                        ctx->d_status);
    entropy_scale<<<1, 256, 0, in.stream>>>(s.peaks, s.unclean, s.blocks, in.type == EP_F16, s.scale);
}

template <typename T>
void launch_round(const float *sums, int64_t n, const Scale *scale, void *out, int sm_count, cudaStream_t stream) {
    const int grid = (int)std::min<int64_t>(ep::ceil_div(n, 1024), (int64_t)sm_count * 8);
    entropy_round<T><<<grid, 256, 0, stream>>>(sums, n, scale, static_cast<T *>(out));
}

int backward_run(ep_ctx *ctx, Inputs &in, const Backward &s, const Given &given, const Wanted &out) {
    if (in.type == EP_F32)
        launch_weights<float>(ctx, in, s, given, out.dweight);
    else if (in.type == EP_BF16)
        launch_weights<__nv_bfloat16>(ctx, in, s, given, out.dweight);
    else
        launch_weights<__half>(ctx, in, s, given, out.dweight);
    EP_CUDA(ctx, cudaGetLastError());
    in.kernels += 2;
    Operand x, w;
    int rc = operands(ctx, in, s.x, s.w, &x, &w);
    if (rc != EP_OK) return rc;
    Operand clean = x;   // x as dW reads it where a row that takes no part holds an infinity or a NaN
    if (out.dweight) {
        const bool direct = x.base == in.x;
        const Packed f = ep::packed_form(in.rows, in.n_in, in.type);
        const int grid = (int)std::min<int64_t>(ep::ceil_div(in.rows, 8), (int64_t)ctx->sm_count * 8);
        entropy_clean<uint16_t><<<grid, 256, 0, in.stream>>>(direct ? (const uint16_t *)in.x : nullptr, in.ldx, in.rows, in.n_in, in.targets,
                                                             given.lse, in.classes, s.scale, (uint16_t *)s.x, f.ld, f.parts, f.part_stride);
        EP_CUDA(ctx, cudaGetLastError());
        ++in.kernels;
        if (direct) clean = Operand{s.x, in.type, in.rows, in.n_in, f.ld, 1, 0};
    }
    const Pieces &p = s.pieces;
    const bool f32 = in.type == EP_F32;
    const size_t size = ep::type_size(in.type);
    const float *factor = in.type == EP_F16 ? &s.scale->down : nullptr;
    int64_t slab = 0;
    for (int64_t row0 = 0; row0 < in.rows; row0 += p.rows) {
        const int64_t rows = std::min(p.rows, in.rows - row0);
        const Operand xr = rows_of(x, row0, rows);
        char *dx_rows = out.dx ? static_cast<char *>(out.dx) + row0 * in.n_in * size : nullptr;
        for (int class0 = 0; class0 < in.classes; class0 += p.classes) {
            const int classes = std::min(p.classes, in.classes - class0);
            rc = logits_of(ctx, in, x, w, row0, rows, class0, classes, s.logits, s.share);
            if (rc != EP_OK) return rc;
            const Packed f = ep::packed_form(rows, classes, in.type);
            const dim3 grid((unsigned)ep::ceil_div(f.ld, G_CHUNKS * 8), (unsigned)s.slabs);
            auto kernel = f32 ? entropy_slopes<float> : in.type == EP_BF16 ? entropy_slopes<__nv_bfloat16> : entropy_slopes<__half>;
            kernel<<<grid, 256, 0, in.stream>>>(s.logits, f.ld, rows, classes, class0, in.bias, in.bias_type, in.targets + row0,
                                                given.lse + row0, s.weights + row0, s.scale, out.dx || out.dweight ? s.g : nullptr,
                                                f.part_stride, out.dbias ? s.part + slab * in.classes + class0 : nullptr, in.classes);
            EP_CUDA(ctx, cudaGetLastError());
            ++in.kernels;
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
            if (in.type == EP_BF16)
                launch_round<__nv_bfloat16>(s.dx, rows * in.n_in, s.scale, dx_rows, ctx->sm_count, in.stream);
            else
                launch_round<__half>(s.dx, rows * in.n_in, s.scale, dx_rows, ctx->sm_count, in.stream);
            EP_CUDA(ctx, cudaGetLastError());
            ++in.kernels;
        }
        slab += s.slabs;
    }
    if (out.dweight && p.across > 1 && !f32) {
        const int64_t n = (int64_t)in.classes * in.n_in;
        if (in.type == EP_BF16)
            launch_round<__nv_bfloat16>(s.dweight, n, s.scale, out.dweight, ctx->sm_count, in.stream);
        else
            launch_round<__half>(s.dweight, n, s.scale, out.dweight, ctx->sm_count, in.stream);
        EP_CUDA(ctx, cudaGetLastError());
        ++in.kernels;
    }
    if (out.dbias) {
        rc = ep::sum_partials(ctx, s.part, (int)slab, in.classes, out.dbias, in.stream);
        if (rc != EP_OK) return rc;
        ++in.kernels;
    }
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
    const ForwardSpace s = forward_space(ctx, rows, n_in, classes, in_type, in.aligned, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes)
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    Timed tm(ctx, in.stream, EP_TIMER_ENTROPY);
    rc = forward_run(ctx, in, s, loss, row_loss, lse, reinterpret_cast<long long *>(counted));
    tm.end(in.kernels);
    return rc;
}

size_t ep_cross_entropy_backward_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t n_in, int32_t classes, int32_t in_type,
                                                 int32_t is_aligned) {
    if (!ctx || !entropy_shape_ok(rows, n_in, classes) || !float_type(in_type)) return 0;
    return backward_space(ctx, rows, n_in, classes, in_type, is_aligned != 0, nullptr).bytes;
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
    const Backward s = backward_space(ctx, rows, n_in, classes, in_type, in.aligned, workspace);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes)
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    Timed tm(ctx, in.stream, EP_TIMER_ENTROPY);
    rc = backward_run(ctx, in, s, Given{lse, dloss, drow_loss, reinterpret_cast<const long long *>(counted)}, Wanted{dx, dweight, dbias});
    tm.end(in.kernels);
    return rc;
}

}  // extern "C"
