// Root-mean-square norm with the residual's addition and an optional 8-bit output, its backward pass, and the 8-bit
// output on its own.
//
// One pass over the data: a row stays with the L threads that share it (in registers, in the backward pass in shared
// memory), between the sum that gives its scale and the product with it, so every input is read once and every output
// written once.  All of these kernels are bound by HBM bandwidth for many rows and by launch latency for few.  Measured
// (of 6464 GB/s, a plain copy): 169343 x 128 fp32 with residual to bf16 50 us, 6.1 TB/s; backward of 2449029 x 128 bf16
// 425 us, 5.9 TB/s; one row of 1024 to 8 bits 4 us.
#include "ep_common.cuh"
#include "rows.cuh"

#include <algorithm>
#include <type_traits>

using namespace eprow;

namespace {

// L <= 32: a block of 256 threads has 256 / L rows at a time.  L > 32: the block is L threads and has one.
template <int L>
constexpr int block_threads() { return L > 32 ? L : 256; }

template <typename O>
constexpr float largest() { return std::is_same_v<O, i8> ? 127.f : 448.f; }   // of an 8-bit type

// rho = 1 / sqrt(mean(h^2) + eps) of a row, from this thread's share `ss` of the sum of squares.  Where the fp32 squares
// leave the range that is safe for their sum (a row of magnitudes below 1e-15 or above 1e18, or of zeros) they are taken
// of the row times a power of two instead; all threads that reduce together take that turn together.  A row of zeros
// with eps = 0 has rho = 0, so that it stays zero.  each(f) calls f with every h of this thread.
template <int L, typename Each>
__device__ __forceinline__ float row_rho(float ss, float per_column, float eps, float *slots, int &turn, Each each) {
    const float mean = reduce_row<L, OpSum>(ss, slots, turn) * per_column;
    float rho = rsqrtf(mean + eps);
    const bool rare = !(mean + eps > 1e-30f && mean < 1e36f);
    if (__any_sync(FULL, rare)) {
        float top = 0.f;
        each([&](float h) { top = fmaxf(top, fabsf(h)); });
        top = reduce_row<L, OpMaxNumber>(top, slots, turn);
        // (with eps > 0 magnitudes below 2^-87 do not count beside it; 2^60 keeps eps s^2 finite)
        const int up = min(max(-ilogbf(fmaxf(top, 1.17549435e-38f)), -100), eps > 0.f ? 60 : 126);
        const float s = scalbnf(1.f, up);
        ss = 0.f;
        each([&](float h) { ss = fmaf(h * s, h * s, ss); });
        const float scaled = reduce_row<L, OpSum>(ss, slots, turn) * per_column + eps * s * s;
        if (rare && scaled == 0.f)
            rho = 0.f;
        else if (rare)
            rho = scaled == scaled ? fminf(s * rsqrtf(scaled), 3.4e38f) : scaled;
    }
    return rho;
}

// NORM: the norm; otherwise the rows are only brought to 8 bits.
template <typename T, typename O, typename Lay, bool NORM>
__global__ void __launch_bounds__(block_threads<Lay::L>()) norm_rows(const T *x, const T *residual, const void *weight,
                                                                     int weight_type, int64_t rows, int d, float eps, O *out,
                                                                     float *scale, T *hidden) {
    constexpr int L = Lay::L, V = Lay::V, N = Lay::N;
    constexpr int GROUPS = block_threads<L>() / L;
    __shared__ float slots[L > 32 ? 64 : 1];
    int turn = 0;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    float g[V][N];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = Lay::col(lane, j, i);
            g[j][i] = NORM && weight && c < d ? load_param(weight, weight_type, c) : 1.f;
        }
    // the loop is the same for all threads of a warp (they reduce together); rows past the end are empty
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < rows; first += (int64_t)gridDim.x * GROUPS) {
        const int64_t row = first + group, at = row * d;
        const bool mine = row < rows;
        float h[V][N];
        Lay::load_if(mine, x + at, lane, d, 0.f, h);
        if (NORM && residual) {
            float r[V][N];
            Lay::load_if(mine, residual + at, lane, d, 0.f, r);
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) h[j][i] += r[j][i];
        }
        if (NORM && hidden && mine) Lay::store(hidden + at, lane, d, h);
        if (NORM) {
            float ss = 0.f;
            auto each = [&](auto f) {
#pragma unroll
                for (int j = 0; j < V; ++j)
#pragma unroll
                    for (int i = 0; i < N; ++i) f(h[j][i]);
            };
            each([&](float v) { ss = fmaf(v, v, ss); });
            const float rho = row_rho<L>(ss, 1.f / (float)d, eps, slots, turn, each);
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) h[j][i] = h[j][i] * rho * g[j][i];
        }
        if constexpr (sizeof(O) == 1) {
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) top = OpMax::apply(top, fabsf(h[j][i]));
            const float s = reduce_row<L, OpMax>(top, slots, turn) / largest<O>();
            if (std::is_same_v<O, i8> && !(s < INFINITY)) {   // integers have no NaN: the scale alone says so
                Lay::set(0.f, h);
            } else if (s > 0.f && s < 1.17549435e-38f) {   // no finite reciprocal worth multiplying by: divide
#pragma unroll
                for (int j = 0; j < V; ++j)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        h[j][i] = h[j][i] / s;   // (s has few bits: past the largest integer by half of it at most)
                        if constexpr (std::is_same_v<O, i8>) h[j][i] = fminf(fmaxf(h[j][i], -127.f), 127.f);
                    }
            } else {
                const float inverse = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
                for (int j = 0; j < V; ++j)
#pragma unroll
                    for (int i = 0; i < N; ++i) h[j][i] *= inverse;
            }
            if (lane == 0 && mine) scale[row] = s;
        }
        if (mine) Lay::store(out + at, lane, d, h);
    }
}

// How many rows a thread's copies run ahead of it, plus one.  Three rows of three inputs keep 50 to 150 KB in flight per
// SM whatever the registers allow (without the copies: 2449029 x 128 bf16 in 605 us, half of the memory's rate).  1: rows
// too wide for it, or not in 16-byte chunks, are read straight into registers.
template <typename Lay>
constexpr int stages() { return !Lay::VEC || block_threads<Lay::L>() > 256 || Lay::V > 4 ? 1 : Lay::V > 2 ? 2 : 3; }
template <typename T, typename D, typename Lay>
constexpr size_t ring_bytes() { return stages<Lay>() == 1 ? 0 : (size_t)stages<Lay>() * 3 * Lay::V * block_threads<Lay::L>() * 16; }

// dx of every row; the block's share of dweight goes to part[blockIdx.x][d] (or to dweight itself when it is alone).
template <typename T, typename D, typename Lay>
__global__ void __launch_bounds__(block_threads<Lay::L>()) norm_rows_backward(const D *dout, const T *hidden, const void *weight,
                                                                              int weight_type, const T *dhidden, int64_t rows,
                                                                              int d, float eps, T *dx, float *part) {
    constexpr int L = Lay::L, V = Lay::V, N = Lay::N, S = stages<Lay>();
    constexpr int THREADS = block_threads<L>(), GROUPS = THREADS / L;
    __shared__ float slots[L > 32 ? 64 : 1];
    extern __shared__ uint4 ring[];                        // [S][3][V][THREADS]
    float *fold = reinterpret_cast<float *>(ring);         // then [GROUPS][V * L * N] where GROUPS > 1
    ep_let_next_launch_start();
    int turn = 0;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const float per_column = 1.f / (float)d;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    float g[V][N], dg[V][N];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = Lay::col(lane, j, i);
            g[j][i] = weight && c < d ? load_param(weight, weight_type, c) : 1.f;
            dg[j][i] = 0.f;
        }
    auto fetch = [&](int64_t row, int s) {
        uint4 *to = ring + (size_t)s * 3 * V * THREADS + threadIdx.x;
        if (row < rows) {
            copy_row<Lay>(to, THREADS, hidden + row * d, lane, d);
            copy_row<Lay>(to + V * THREADS, THREADS, dout + row * d, lane, d);
            if (dhidden) copy_row<Lay>(to + 2 * V * THREADS, THREADS, dhidden + row * d, lane, d);
        }
        copies_end_group();
    };
    // the gradient of one row, from its chunks: called the same by all threads of a warp
    auto work = [&](int64_t row, auto hj, auto yj, auto oj) {
        const bool mine = row < rows;
        float ss = 0.f, ah = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float h[N], y[N];
            hj(j, h);
            yj(j, y);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ss = fmaf(h[i], h[i], ss);
                ah = fmaf(y[i] * g[j][i], h[i], ah);
            }
        }
        const float rho = row_rho<L>(ss, per_column, eps, slots, turn, [&](auto f) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float h[N];
                hj(j, h);
#pragma unroll
                for (int i = 0; i < N; ++i) f(h[i]);
            }
        });
        const float back = rho * (reduce_row<L, OpSum>(ah, slots, turn) * per_column);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float h[N], y[N], o[N];
            hj(j, h);
            yj(j, y);
            oj(j, o);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float unit = h[i] * rho;
                o[i] = fmaf(rho, y[i] * g[j][i] - unit * back, o[i]);
                dg[j][i] = fmaf(y[i], unit, dg[j][i]);
            }
            if (mine) Lay::store_part(dx + row * d, lane, j, d, o);
        }
    };
    if constexpr (S > 1) {
        int64_t ahead = (int64_t)blockIdx.x * GROUPS + group;
#pragma unroll
        for (int s = 0; s < S - 1; ++s, ahead += step) fetch(ahead, s);
        int s = 0;
        for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < rows; first += step, ahead += step) {
            fetch(ahead, s == 0 ? S - 1 : s - 1);   // into the slots of the row before
            copies_wait<S - 1>();
            const uint4 *from = ring + (size_t)s * 3 * V * THREADS + threadIdx.x;
            const int64_t row = first + group;
            const bool mine = row < rows;
            work(
                row, [&](int j, float(&v)[N]) { copied_chunk<Lay, T>(from, THREADS, mine, lane, j, d, 0.f, v); },
                [&](int j, float(&v)[N]) { copied_chunk<Lay, D>(from + V * THREADS, THREADS, mine, lane, j, d, 0.f, v); },
                [&](int j, float(&v)[N]) { copied_chunk<Lay, T>(from + 2 * V * THREADS, THREADS, mine && dhidden, lane, j, d, 0.f, v); });
            s = s + 1 == S ? 0 : s + 1;
        }
        copies_wait<0>();
        __syncthreads();   // the ring becomes the fold
    } else {
        for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < rows; first += step) {
            const int64_t row = first + group, at = row * d;
            const bool mine = row < rows;
            float h[V][N], y[V][N], o[V][N];
            Lay::load_if(mine, hidden + at, lane, d, 0.f, h);
            Lay::load_if(mine, dout + at, lane, d, 0.f, y);
            Lay::load_if(mine && dhidden, dhidden + at, lane, d, 0.f, o);
            auto held = [](const float(&a)[V][N]) {
                return [&a](int j, float(&v)[N]) {
#pragma unroll
                    for (int i = 0; i < N; ++i) v[i] = a[j][i];
                };
            };
            work(row, held(h), held(y), held(o));
        }
    }
    if (!part) return;
    float *to = part + (size_t)blockIdx.x * d;
    if constexpr (GROUPS == 1) {
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (Lay::col(lane, j, i) < d) to[Lay::col(lane, j, i)] = dg[j][i];
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) fold[group * Lay::WIDE + Lay::col(lane, j, i)] = dg[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
            float s = 0.f;
#pragma unroll 4
            for (int q = 0; q < GROUPS; ++q) s += fold[q * Lay::WIDE + c];
            to[c] = s;
        }
    }
}

// A block sums 32 columns: 32 x 32 threads, thread (c, r) the rows r, r + 32, ... in fp64; then a warp per column.
__global__ void __launch_bounds__(1024) fold_partials(const float *parts, int n, int cols, float *out) {
    __shared__ double s[32][33];
    const int lane = threadIdx.x & 31, r0 = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    ep_wait_for_launch_before();
    double t = 0.0;
    if (c < cols)
        for (int r = r0; r < n; r += 32 * 16) {   // 16 loads at a time, none of them alone at the end
            float v[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = r + 32 * q < n ? parts[(size_t)(r + 32 * q) * cols + c] : 0.f;
#pragma unroll
            for (int q = 0; q < 16; ++q) t += (double)v[q];
        }
    s[r0][lane] = t;
    __syncthreads();
    t = s[lane][r0];   // a warp per column now
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) t += __shfl_xor_sync(FULL, t, o);
    if (lane == 0 && blockIdx.x * 32 + r0 < cols) out[blockIdx.x * 32 + r0] = (float)t;
}

constexpr int MAX_D = 16384;
constexpr int FORWARD_BLOCKS_PER_SM = 8, BACKWARD_BLOCKS_PER_SM = 4;   // about what their registers let stay resident

template <int L>
int grid_for(const ep_ctx *ctx, int64_t rows, int per_sm, int alone = 1) {
    constexpr int groups = block_threads<L>() / L;
    if (rows <= (int64_t)groups * alone) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(ep::ceil_div(rows, groups), (int64_t)ctx->sm_count * per_sm));
}

struct NormArgs {
    ep_ctx *ctx;
    const void *x, *residual, *weight;
    int weight_type;
    int64_t rows;
    int d;
    float eps;
    void *out;
    float *scale;
    void *hidden;
    bool vec;
    cudaStream_t stream;
};

template <typename T, typename O, bool NORM>
struct NormLaunch {
    static constexpr int MAX_WIDTH = MAX_D;
    const NormArgs &a;
    template <typename Lay>
    int run() const {
        norm_rows<T, O, Lay, NORM><<<grid_for<Lay::L>(a.ctx, a.rows, FORWARD_BLOCKS_PER_SM), block_threads<Lay::L>(), 0, a.stream>>>(
            (const T *)a.x, (const T *)a.residual, a.weight, a.weight_type, a.rows, a.d, a.eps, (O *)a.out, a.scale, (T *)a.hidden);
        EP_CUDA(a.ctx, cudaGetLastError());
        return EP_OK;
    }
};

template <typename T, typename O, bool NORM>
int launch_norm(const NormArgs &a) {
    return with_layout<T>(a.d, a.vec, NormLaunch<T, O, NORM>{a});
}

template <typename T>
int launch_norm_out(const NormArgs &a, int out_type) {
    if constexpr (sizeof(T) == 4) {
        if (out_type == EP_BF16) return launch_norm<T, __nv_bfloat16, true>(a);
        if (out_type == EP_F16) return launch_norm<T, __half, true>(a);
    }
    if (out_type == EP_E4M3) return launch_norm<T, e4m3, true>(a);
    if (out_type == EP_I8) return launch_norm<T, i8, true>(a);
    return launch_norm<T, T, true>(a);
}

template <typename T>
int launch_quantize(const NormArgs &a, int out_type) {
    return out_type == EP_I8 ? launch_norm<T, i8, false>(a) : launch_norm<T, e4m3, false>(a);
}

struct BackArgs {
    ep_ctx *ctx;
    const void *dout, *hidden, *weight;
    int weight_type;
    const void *dhidden;
    int64_t rows;
    int d;
    float eps;
    void *dx;
    float *dweight, *parts;
    bool vec;
    cudaStream_t stream;
    int kernels;
};

template <typename T, typename D>
struct BackLaunch {
    static constexpr int MAX_WIDTH = MAX_D;
    BackArgs &a;
    template <typename Lay>
    int run() const {
        constexpr int threads = block_threads<Lay::L>();
        constexpr size_t fold = threads == Lay::L ? 0 : sizeof(float) * (threads / Lay::L) * Lay::WIDE;
        constexpr size_t smem = std::max(fold, ring_bytes<T, D, Lay>());
        // (two rounds of one block are quicker than two blocks and the fold after them: 128 x 64 fp32 in 3.9 us against 4.5)
        const int grid = grid_for<Lay::L>(a.ctx, a.rows, BACKWARD_BLOCKS_PER_SM, a.dweight ? 2 : 1);
        float *part = !a.dweight ? nullptr : grid == 1 ? a.dweight : a.parts;
        if (smem > 40 * 1024)   // (static shared memory counts too)
            EP_CUDA(a.ctx, cudaFuncSetAttribute(norm_rows_backward<T, D, Lay>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        norm_rows_backward<T, D, Lay><<<grid, threads, smem, a.stream>>>((const D *)a.dout, (const T *)a.hidden, a.weight,
                                                                         a.weight_type, (const T *)a.dhidden, a.rows, a.d, a.eps,
                                                                         (T *)a.dx, part);
        EP_CUDA(a.ctx, cudaGetLastError());
        a.kernels = 1;
        if (part && grid > 1) {
            a.kernels = 2;
            return ep::sum_partials(a.ctx, a.parts, grid, a.d, a.dweight, a.stream);
        }
        return EP_OK;
    }
};

template <typename T, typename D>
int launch_backward(BackArgs &a) {
    return with_layout<T>(a.d, a.vec, BackLaunch<T, D>{a});
}

}  // namespace

namespace ep {

int sum_partials(ep_ctx *ctx, const float *parts, int n, int cols, float *out, cudaStream_t stream) {
    EP_CUDA(ctx, launch_early(fold_partials, dim3((unsigned)ceil_div(cols, 32)), dim3(1024), 0, stream, parts, n, cols, out));
    return EP_OK;
}

}  // namespace ep

using namespace ep;

namespace {

bool norm_shape_ok(int64_t rows, int d) { return rows >= 0 && rows < (1ll << 31) && d >= 1 && d <= MAX_D; }
bool element_aligned(const void *p, int type) { return !p || aligned(p, (size_t)type_size(type)); }
bool all16(std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if (!aligned(p, 16)) return false;
    return true;
}

int norm_call(ep_ctx *ctx, bool norm, const void *x, int x_type, const void *residual, const void *weight, int weight_type,
              int64_t rows, int d, float eps, void *out, int out_type, float *scale, void *hidden, cudaStream_t stream) {
    NormArgs a{ctx, x, residual, weight, weight_type, rows, d, eps, out, scale, hidden, false, stream};
    a.vec = d % (16 / type_size(x_type)) == 0 && all16({x, residual, out, hidden});
    DeviceGuard guard(ctx->device);
    Timed tm(ctx, stream, EP_TIMER_NORM);
    int rc;
    if (!norm)
        rc = x_type == EP_F32    ? launch_quantize<float>(a, out_type)
             : x_type == EP_BF16 ? launch_quantize<__nv_bfloat16>(a, out_type)
                                 : launch_quantize<__half>(a, out_type);
    else
        rc = x_type == EP_F32    ? launch_norm_out<float>(a, out_type)
             : x_type == EP_BF16 ? launch_norm_out<__nv_bfloat16>(a, out_type)
                                 : launch_norm_out<__half>(a, out_type);
    tm.end(rc == EP_OK ? 1 : 0);
    return rc;
}

}  // namespace

extern "C" {

int ep_rms_norm(ep_ctx *ctx, const void *x, int32_t x_type, const void *residual, const void *weight,
                int32_t weight_type, int64_t rows, int32_t d, float eps, void *out, int32_t out_type, float *scale,
                void *hidden, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (!norm_shape_ok(rows, d)) return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld or d %d out of range", (long long)rows, d);
    if (!float_type(x_type) || (weight && !float_type(weight_type)) ||
        !(out_type == x_type || eight_bits(out_type) || (x_type == EP_F32 && float_type(out_type))))
        return fail(ctx, EP_ERR_INVALID_ARG, "no norm from type %d to type %d", x_type, out_type);
    if (!(eps >= 0.f) || eps > 3e38f) return fail(ctx, EP_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (rows == 0) return EP_OK;
    if (eight_bits(out_type) != (scale != nullptr))
        return fail(ctx, EP_ERR_INVALID_ARG, "scale goes with an 8-bit output, and with no other");
    if (!x || !out || !element_aligned(x, x_type) || !element_aligned(residual, x_type) || !element_aligned(out, out_type) ||
        !element_aligned(hidden, x_type) || !element_aligned(weight, weight ? weight_type : EP_E4M3) || !aligned(scale, 4))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    return norm_call(ctx, true, x, x_type, residual, weight, weight_type, rows, d, eps, out, out_type, scale, hidden,
                     static_cast<cudaStream_t>(cuda_stream));
}

int ep_quantize_rows_to(ep_ctx *ctx, const void *x, int32_t x_type, int64_t rows, int32_t d, void *q, int32_t q_type, float *scale,
                        void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (!norm_shape_ok(rows, d)) return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld or d %d out of range", (long long)rows, d);
    if (!float_type(x_type) || !eight_bits(q_type))
        return fail(ctx, EP_ERR_INVALID_ARG, "rows of type %d cannot be brought to 8 bits of type %d", x_type, q_type);
    if (rows == 0) return EP_OK;
    if (!x || !q || !scale || !element_aligned(x, x_type) || !aligned(scale, 4))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    return norm_call(ctx, false, x, x_type, nullptr, nullptr, EP_F32, rows, d, 0.f, q, q_type, scale, nullptr,
                     static_cast<cudaStream_t>(cuda_stream));
}

int ep_quantize_rows(ep_ctx *ctx, const void *x, int32_t x_type, int64_t rows, int32_t d, void *q, float *scale,
                     void *cuda_stream) {
    return ep_quantize_rows_to(ctx, x, x_type, rows, d, q, EP_E4M3, scale, cuda_stream);
}

size_t ep_rms_norm_backward_workspace_bytes(const ep_ctx *ctx, int64_t rows, int32_t d) {
    if (!ctx || !norm_shape_ok(rows, d)) return 0;
    Arena a(nullptr);
    a.take<float>((size_t)ctx->sm_count * BACKWARD_BLOCKS_PER_SM * d);
    return a.used;
}

int ep_rms_norm_backward(ep_ctx *ctx, const void *dout, int32_t dout_type, const void *hidden, int32_t h_type,
                         const void *weight, int32_t weight_type, const void *dhidden, int64_t rows, int32_t d, float eps,
                         void *dx, float *dweight, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!ctx) return EP_ERR_INVALID_ARG;
    if (!norm_shape_ok(rows, d)) return fail(ctx, EP_ERR_INVALID_ARG, "rows %lld or d %d out of range", (long long)rows, d);
    if (!float_type(h_type) || (weight && !float_type(weight_type)) ||
        !(dout_type == h_type || (h_type == EP_F32 && float_type(dout_type))))
        return fail(ctx, EP_ERR_INVALID_ARG, "no norm gradient from type %d to type %d", dout_type, h_type);
    if (!(eps >= 0.f) || eps > 3e38f) return fail(ctx, EP_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (!aligned(dweight, 4)) return fail(ctx, EP_ERR_INVALID_ARG, "misaligned pointer");
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    DeviceGuard guard(ctx->device);
    if (rows == 0) {
        if (dweight) EP_CUDA(ctx, cudaMemsetAsync(dweight, 0, sizeof(float) * (size_t)d, stream));
        return EP_OK;
    }
    if (!dout || !hidden || !dx || !element_aligned(dout, dout_type) || !element_aligned(hidden, h_type) ||
        !element_aligned(dhidden, h_type) || !element_aligned(dx, h_type) ||
        !element_aligned(weight, weight ? weight_type : EP_E4M3))
        return fail(ctx, EP_ERR_INVALID_ARG, "null or misaligned pointer");
    if (dweight && (!workspace || !aligned(workspace, 256) ||
                    workspace_bytes < ep_rms_norm_backward_workspace_bytes(ctx, rows, d)))
        return fail(ctx, EP_ERR_WORKSPACE, "workspace too small or misaligned");
    BackArgs a{ctx, dout, hidden, weight, weight_type, dhidden, rows, d, eps, dx, dweight, static_cast<float *>(workspace),
               false, stream, 0};
    a.vec = d % (16 / type_size(h_type)) == 0 && all16({dout, hidden, dhidden, dx});
    Timed tm(ctx, stream, EP_TIMER_NORM);
    int rc;
    if (h_type == EP_BF16)
        rc = launch_backward<__nv_bfloat16, __nv_bfloat16>(a);
    else if (h_type == EP_F16)
        rc = launch_backward<__half, __half>(a);
    else if (dout_type == EP_BF16)
        rc = launch_backward<float, __nv_bfloat16>(a);
    else if (dout_type == EP_F16)
        rc = launch_backward<float, __half>(a);
    else
        rc = launch_backward<float, float>(a);
    tm.end(rc == EP_OK ? a.kernels : 0);
    return rc;
}

}  // extern "C"
