// Device helpers of the row-wise kernels (norm.cu, route.cu) and of the products' epilogues (linear.cu): element
// types, accesses of 16-byte chunks, and sums and maxima over the threads that share a row.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "embedpart.h"

namespace eprow {

constexpr unsigned FULL = 0xffffffffu;

// 2^x, e^x and 1 / x by the special function unit: within a few units of 2^-22 of themselves (times |x| 2^-24 more for
// e^x), results below 2^-126 are zero.
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float exp_fast(float x) { return exp2_fast(x * 1.44269504f); }
__device__ __forceinline__ float reciprocal_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Two floats that go through one instruction (the fp32 pipe takes pairs; each is rounded as by itself).
struct Pair {
    unsigned long long v;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit Pair(float both) : Pair(both, both) {}
    __device__ __forceinline__ void get(float &lo, float &hi) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
};
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
struct e4m3 {
    uint8_t bits;
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(e4m3 v) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(v.bits, __NV_E4M3)));
}

// Every rounding is to nearest, ties to even; e4m3 saturates at 448 (its callers scale to that range first).
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ e4m3 from_f32<e4m3>(float v) {
    e4m3 r;
    r.bits = __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3);
    return r;
}

// Two floats to two e4m3 (a in the low byte).
__device__ __forceinline__ uint16_t to_e4m3_pair(float a, float b) {
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// One vector parameter (a norm's weight, a product's bias) of type EP_F32, EP_BF16 or EP_F16.
__device__ __forceinline__ float load_param(const void *p, int type, int64_t i) {
    if (type == EP_F32) return static_cast<const float *>(p)[i];
    if (type == EP_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}

template <int BYTES>
struct Raw;
template <>
struct Raw<1> { using type = uint8_t; };
template <>
struct Raw<2> { using type = uint16_t; };
template <>
struct Raw<4> { using type = uint32_t; };
template <>
struct Raw<8> { using type = uint2; };
template <>
struct Raw<16> { using type = uint4; };
template <>
struct Raw<32> { using type = uint4; };

// N consecutive elements at column `col` of a row of `width` elements.  vec: the row starts on a boundary of the
// whole access and width is a multiple of N, so the chunk is one access, all of it inside the row or none of it.
// Elements past the row's end read as `fill`.
template <int N, typename T>
__device__ __forceinline__ void load_chunk(const T *row, int col, int width, bool vec, float fill, float (&v)[N]) {
    if (vec) {
        if (col < width) {
            alignas(16) T e[N];
            constexpr int B = N * (int)sizeof(T);
            using R = typename Raw<B>::type;
            constexpr int PIECES = B > 16 ? B / 16 : 1;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) reinterpret_cast<R *>(e)[i] = reinterpret_cast<const R *>(row + col)[i];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = to_f32(e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = fill;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = col + i < width ? to_f32(row[col + i]) : fill;
    }
}

template <int N, typename T>
__device__ __forceinline__ void store_chunk(T *row, int col, int width, bool vec, const float (&v)[N]) {
    if (vec) {
        if (col < width) {
            alignas(16) T e[N];
            constexpr int B = N * (int)sizeof(T);
            using R = typename Raw<B>::type;
            constexpr int PIECES = B > 16 ? B / 16 : 1;
            if constexpr (sizeof(T) == 1 && N % 2 == 0) {   // (8 bits are converted two at a time)
#pragma unroll
                for (int i = 0; i < N; i += 2) reinterpret_cast<uint16_t *>(e)[i / 2] = to_e4m3_pair(v[i], v[i + 1]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) e[i] = from_f32<T>(v[i]);
            }
#pragma unroll
            for (int i = 0; i < PIECES; ++i) reinterpret_cast<R *>(row + col)[i] = reinterpret_cast<const R *>(e)[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (col + i < width) row[col + i] = from_f32<T>(v[i]);
    }
}

// WORDS consecutive 32-bit words from any byte address on, by 16-byte accesses and shifts.  The accesses reach up to 15
// bytes to either side: the caller has made sure that [p & ~15, + 4 WORDS + 16) belongs to the matrix.
template <int WORDS>
__device__ __forceinline__ void load_words_anywhere(const void *p, uint32_t (&out)[WORDS]) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    const uint4 *from = reinterpret_cast<const uint4 *>(b & ~uintptr_t(15));
    uint32_t w[WORDS + 4];
#pragma unroll
    for (int q = 0; q < WORDS / 4 + 1; ++q) {
        const uint4 v = from[q];
        w[4 * q] = v.x, w[4 * q + 1] = v.y, w[4 * q + 2] = v.z, w[4 * q + 3] = v.w;
    }
    const bool one = b & 4, two = b & 8;
#pragma unroll
    for (int i = 0; i < WORDS + 3; ++i) w[i] = one ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < WORDS + 1; ++i) w[i] = two ? w[i + 2] : w[i];
    const unsigned bits = (unsigned)(b & 3) * 8;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) out[i] = __funnelshift_r(w[i], w[i + 1], bits);
}
// N elements of a row from p on, of which the first `inside` (at least 1) belong to it; the others come out as zero bits.
// begin, end: the matrix.
template <int N, typename T>
__device__ __forceinline__ void load_elements_anywhere(const T *p, int inside, const T *begin, const T *end, T (&e)[N]) {
    constexpr int BYTES = N * (int)sizeof(T);
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) & ~uintptr_t(15);
    if (a >= reinterpret_cast<uintptr_t>(begin) && a + BYTES + 16 <= reinterpret_cast<uintptr_t>(end)) {
        union {
            uint32_t w[BYTES / 4];
            T t[N];
        } u;
        load_words_anywhere(p, u.w);
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = i < inside ? u.t[i] : T{};
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = i < inside ? p[i] : T{};
    }
}

// ---- sums and maxima over the L threads of a row -------------------------------------------------
// L <= 32: neighbouring lanes of one warp (all 32 lanes of the warp call together).  L > 32: the whole block; `slots`
// is then shared memory of 2 x 32 floats used in turn (`turn` flips with every call), one barrier per call.
struct OpSum {
    static __device__ __forceinline__ float apply(float a, float b) { return a + b; }
    static constexpr float none = 0.f;
};
struct OpMax {   // NaN if either is: a row that holds one has no largest magnitude to scale by
    static __device__ __forceinline__ float apply(float a, float b) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
        return r;
    }
    static constexpr float none = -INFINITY;
};
struct OpMaxNumber {   // NaN only if both are
    static __device__ __forceinline__ float apply(float a, float b) { return fmaxf(a, b); }
    static constexpr float none = -INFINITY;
};

template <int L, typename Op>
__device__ __forceinline__ float reduce_row(float v, float *slots, int &turn) {
    constexpr int W = L < 32 ? L : 32;
#pragma unroll
    for (int o = W / 2; o >= 1; o >>= 1) v = Op::apply(v, __shfl_xor_sync(FULL, v, o));
    if constexpr (L > 32) {
        float *s = slots + turn * 32;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
        __syncthreads();
        float t = (threadIdx.x & 31) < L / 32 ? s[threadIdx.x & 31] : Op::none;
#pragma unroll
        for (int o = L / 64; o >= 1; o >>= 1) t = Op::apply(t, __shfl_xor_sync(FULL, t, o));
        v = __shfl_sync(FULL, t, 0);
    }
    return v;
}

// ---- how a row lies over the L threads that share it ------------------------------------------------
// V x N columns to each thread.  VEC: chunks of N columns (16 bytes of the input type) dealt out in turn; every row
// starts on a 16-byte boundary and holds whole chunks.  Otherwise single columns dealt out in turn, so that neighbouring
// lanes access neighbouring elements wherever the row starts.  Rows have more than LOW columns: what lies below is not
// checked against the row's end.
template <int L_, int V_, int N_, bool VEC_, int LOW_>
struct Layout {
    static constexpr int L = L_, V = V_, N = N_, WIDE = L_ * V_ * N_;
    static constexpr bool VEC = VEC_;
    static __device__ __forceinline__ int col(int lane, int j, int i) {
        return VEC ? (j * L + lane) * N + i : (j * N + i) * L + lane;
    }
    // The thread that holds column c, and the column's place j * N + i there (any c; a place past the thread's own for
    // columns past the layout).
    static __device__ __forceinline__ int owner(int c) { return VEC ? c / N % L : c % L; }
    static __device__ __forceinline__ int index(int c) { return VEC ? c / N / L * N + c % N : c / L; }
    static __device__ __forceinline__ bool inside(int lane, int j, int i, int width) {
        return (VEC ? (j + 1) * L * N : (j * N + i + 1) * L) <= LOW_ || col(lane, j, i) < width;
    }
    template <typename T>
    static __device__ __forceinline__ void load(const T *row, int lane, int width, float fill, float (&v)[V_][N_]) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (VEC) {
                if (inside(lane, j, 0, width))
                    load_chunk(row, col(lane, j, 0), 1 << 30, true, fill, v[j]);
                else {
#pragma unroll
                    for (int i = 0; i < N; ++i) v[j][i] = fill;
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) v[j][i] = inside(lane, j, i, width) ? to_f32(row[col(lane, j, i)]) : fill;
            }
        }
    }
    template <typename T>
    static __device__ __forceinline__ void store(T *row, int lane, int width, const float (&v)[V_][N_]) {
#pragma unroll
        for (int j = 0; j < V; ++j) store_part(row, lane, j, width, v[j]);
    }
    template <typename T>
    static __device__ __forceinline__ void store_part(T *row, int lane, int j, int width, const float (&v)[N_]) {
        if constexpr (VEC) {
            if (inside(lane, j, 0, width)) store_chunk(row, col(lane, j, 0), 1 << 30, true, v);
        } else if constexpr (sizeof(T) == 1) {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const uint16_t two = to_e4m3_pair(v[i], v[i + 1]);
                if (inside(lane, j, i, width)) row[col(lane, j, i)].bits = (uint8_t)two;
                if (inside(lane, j, i + 1, width)) row[col(lane, j, i + 1)].bits = (uint8_t)(two >> 8);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (inside(lane, j, i, width)) row[col(lane, j, i)] = from_f32<T>(v[i]);
        }
    }
    // A row that is not there (or is not to be read) is all `fill`.
    template <typename T>
    static __device__ __forceinline__ void load_if(bool there, const T *row, int lane, int width, float fill, float (&v)[V_][N_]) {
        if (there)
            load(row, lane, width, fill, v);
        else
            set(fill, v);
    }
    static __device__ __forceinline__ void set(float fill, float (&v)[V_][N_]) {
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) v[j][i] = fill;
    }
};

// ---- rows on their way to shared memory ---------------------------------------------------------------
// A thread's own chunks of a row (VEC layouts), copied asynchronously several rows ahead: each thread reads back only
// what it copied itself, so nothing has to be synchronised, and the bytes in flight do not cost registers.  `slots` is
// this thread's first 16-byte slot, slots of one chunk index lie `threads` apart.
template <int BYTES>
__device__ __forceinline__ void copy_async(void *to, const void *from) {
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

template <typename Lay, typename T>
__device__ __forceinline__ void copy_row(uint4 *slots, int threads, const T *row, int lane, int width) {
#pragma unroll
    for (int j = 0; j < Lay::V; ++j)
        if (Lay::inside(lane, j, 0, width))
            copy_async<Lay::N * (int)sizeof(T)>(slots + j * threads, row + Lay::col(lane, j, 0));
}
// Chunk j of a row copied by copy_row; `fill` where the row has no such chunk.
template <typename Lay, typename T>
__device__ __forceinline__ void copied_chunk(const uint4 *slots, int threads, bool there, int lane, int j, int width, float fill,
                                             float (&v)[Lay::N]) {
    if (there && Lay::inside(lane, j, 0, width))
        load_chunk(reinterpret_cast<const T *>(slots + j * threads), 0, 1 << 30, true, fill, v);
    else {
#pragma unroll
        for (int i = 0; i < Lay::N; ++i) v[i] = fill;
    }
}

// `bytes` (up to 16) of 16, the rest zero.
__device__ __forceinline__ void copy_async_some(void *to, const void *from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes)
                 : "memory");
}

// One input of a kernel that goes over its rows in steps of a whole grid, THREADS / L rows a block: rows on their way to
// shared memory S - 1 steps ahead.  VEC layouts as above.  Other layouts of up to 32 threads a row: a warp copies
// the 16-byte pieces that its rows lie in, whatever their alignment, and its threads pick their elements (the input
// itself has to start on a 16-byte boundary: `on`).  What is left reads straight into registers.
template <typename T, typename Lay, int THREADS>
struct RowStream {
    static constexpr bool SPAN = !Lay::VEC && Lay::L <= 32;
    static constexpr int S = Lay::VEC || SPAN ? 3 : 1;
    static __host__ __device__ constexpr int span_bytes(int width) { return ((32 / Lay::L) * width * (int)sizeof(T) + 30) / 16 * 16; }
    static __host__ __device__ constexpr int ring_bytes(int width) {
        return Lay::VEC ? S * Lay::V * THREADS * 16 : SPAN ? S * (THREADS / 32) * span_bytes(width) : 0;
    }
    const T *base;
    int64_t rows;
    int width, lane, group, stage;
    bool on;
    char *mine, *shown;   // VEC: this thread's first slot; otherwise this warp's first span; and that of the row of next()

    __device__ __forceinline__ RowStream(char *ring, const T *input, int64_t n, int w, int lane_, int group_, bool spans)
        : base(input), rows(n), width(w), lane(lane_), group(group_), stage(0), on(Lay::VEC || (SPAN && spans)) {
        mine = Lay::VEC ? ring + threadIdx.x * 16 : ring + (threadIdx.x >> 5) * span_bytes(w);
    }
    __device__ __forceinline__ char *at(int s) const {
        return mine + s * (Lay::VEC ? Lay::V * THREADS * 16 : (THREADS / 32) * span_bytes(width));
    }
    // Starts the copy of the step whose first row (of the block) is `first` into stage s.
    __device__ __forceinline__ void fetch(int64_t first, int s) {
        if constexpr (Lay::VEC) {
            if (first + group < rows) copy_row<Lay>(reinterpret_cast<uint4 *>(at(s)), THREADS, base + (first + group) * width, lane, width);
            copies_end_group();
        } else if constexpr (SPAN) {
            if (!on) return;
            const int64_t row = first + (group & ~(32 / Lay::L - 1));
            if (row < rows) {
                const int64_t start = row * width * (int64_t)sizeof(T), from = start & ~int64_t(15);
                const int length = (int)min(rows - row, (int64_t)(32 / Lay::L)) * width * (int)sizeof(T) + (int)(start - from);
                const bool last = rows - row <= 32 / Lay::L;   // the last piece must not reach past the input
                const char *src = reinterpret_cast<const char *>(base) + from;
                char *dst = at(s);
                for (int p = (threadIdx.x & 31) * 16; p < length; p += 512)
                    copy_async_some(dst + p, src + p, last ? min(length - p, 16) : 16);
            }
            copies_end_group();
        }
    }
    __device__ __forceinline__ void begin(int64_t first, int64_t step) {
#pragma unroll
        for (int s = 0; s < S - 1; ++s) fetch(first + s * step, s);
    }
    // The row of this step: there = it is to be read.  Called by all threads of a warp.
    __device__ __forceinline__ void next(int64_t first, int64_t step, bool there, float fill, float (&v)[Lay::V][Lay::N]) {
        const int64_t row = first + group;
        if (on) {
            if constexpr (SPAN) __syncwarp();   // every lane has read what the next copy overwrites
            fetch(first + (S - 1) * step, stage == 0 ? S - 1 : stage - 1);
            copies_wait<S - 1>();
            if constexpr (Lay::VEC) {
#pragma unroll
                for (int j = 0; j < Lay::V; ++j)
                    copied_chunk<Lay, T>(reinterpret_cast<const uint4 *>(at(stage)), THREADS, there, lane, j, width, fill, v[j]);
            } else {
                __syncwarp();
                const int64_t first_row = first + (group & ~(32 / Lay::L - 1));
                const int shift = (int)(first_row * width * (int64_t)sizeof(T) & 15);
                Lay::load_if(there, reinterpret_cast<const T *>(at(stage) + shift) + (int)(row - first_row) * width, lane, width, fill, v);
            }
            shown = at(stage);
            stage = stage + 1 == S ? 0 : stage + 1;
        } else {
            Lay::load_if(there, base + row * width, lane, width, fill, v);
        }
    }
    // Element c of the row that next() has delivered (after the threads of the row have met).
    __device__ __forceinline__ float element(int64_t first, int c) const {
        if (!on) return to_f32(base[(first + group) * width + c]);
        if constexpr (Lay::VEC) {
            const int q = c / Lay::N;
            return to_f32(reinterpret_cast<const T *>(shown + ((q / Lay::L) * THREADS + q % Lay::L - lane) * 16)[c % Lay::N]);
        } else {
            const int64_t first_row = first + (group & ~(32 / Lay::L - 1));
            const int shift = (int)(first_row * width * (int64_t)sizeof(T) & 15);
            return to_f32(reinterpret_cast<const T *>(shown + shift)[(int)(first + group - first_row) * width + c]);
        }
    }
    __device__ __forceinline__ void end() const { copies_wait<0>(); }
};

// Calls f.run<Layout>() with the layout for rows of `width` elements of T.  About 16 columns per thread: fewer steps of
// the sums across threads than with one chunk each, and as many loads in flight (2449029 rows of 32 fp32 logits routed in
// 218 us with 4 columns a thread, 152 with 16, all else equal).
template <typename T, typename F>
int with_layout(int width, bool vec, F f) {
    constexpr int N = 16 / (int)sizeof(T);
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            if (width <= 4) return f.template run<Layout<1, 1, N, true, 0>>();
            if (width <= 16) return f.template run<Layout<1, 4, N, true, 4>>();
            if (width <= 32) return f.template run<Layout<2, 4, N, true, 16>>();
            if (width <= 64) return f.template run<Layout<4, 4, N, true, 32>>();
            if (width <= 128) return f.template run<Layout<8, 4, N, true, 64>>();
            if (width <= 256) return f.template run<Layout<16, 4, N, true, 128>>();
            if (width <= 512) return f.template run<Layout<32, 4, N, true, 256>>();
            if (width <= 1024) return f.template run<Layout<32, 8, N, true, 512>>();
            if (width <= 2048) return f.template run<Layout<256, 2, N, true, 1024>>();
            if (width <= 4096) return f.template run<Layout<256, 4, N, true, 2048>>();
            if constexpr (F::MAX_WIDTH > 4096) {
                if (width <= 8192) return f.template run<Layout<512, 4, N, true, 4096>>();
                return f.template run<Layout<512, 8, N, true, 8192>>();
            }
        } else {
            if (width <= 8) return f.template run<Layout<1, 1, N, true, 0>>();
            if (width <= 16) return f.template run<Layout<1, 2, N, true, 8>>();
            if (width <= 32) return f.template run<Layout<2, 2, N, true, 16>>();
            if (width <= 64) return f.template run<Layout<4, 2, N, true, 32>>();
            if (width <= 128) return f.template run<Layout<8, 2, N, true, 64>>();
            if (width <= 256) return f.template run<Layout<16, 2, N, true, 128>>();
            if (width <= 512) return f.template run<Layout<32, 2, N, true, 256>>();
            if (width <= 1024) return f.template run<Layout<32, 4, N, true, 512>>();
            if (width <= 2048) return f.template run<Layout<256, 1, N, true, 1024>>();
            if (width <= 4096) return f.template run<Layout<256, 2, N, true, 2048>>();
            if constexpr (F::MAX_WIDTH > 4096) {
                if (width <= 8192) return f.template run<Layout<256, 4, N, true, 4096>>();
                return f.template run<Layout<512, 4, N, true, 8192>>();
            }
        }
        return 0;
    }
    if (width <= 4) return f.template run<Layout<1, 1, 4, false, 0>>();
    if (width <= 16) return f.template run<Layout<2, 2, 4, false, 4>>();
    if (width <= 32) return f.template run<Layout<4, 2, 4, false, 16>>();
    if (width <= 48) return f.template run<Layout<4, 3, 4, false, 32>>();
    if (width <= 64) return f.template run<Layout<8, 2, 4, false, 48>>();
    if (width <= 96) return f.template run<Layout<8, 3, 4, false, 64>>();
    if (width <= 128) return f.template run<Layout<8, 4, 4, false, 96>>();
    if (width <= 192) return f.template run<Layout<16, 3, 4, false, 128>>();
    if (width <= 256) return f.template run<Layout<16, 4, 4, false, 192>>();
    if (width <= 320) return f.template run<Layout<16, 5, 4, false, 256>>();
    if (width <= 384) return f.template run<Layout<32, 3, 4, false, 320>>();
    if (width <= 512) return f.template run<Layout<32, 4, 4, false, 384>>();
    if (width <= 768) return f.template run<Layout<32, 6, 4, false, 512>>();
    if (width <= 1024) return f.template run<Layout<32, 8, 4, false, 768>>();
    if (width <= 2048) return f.template run<Layout<256, 2, 4, false, 1024>>();
    if (width <= 4096) return f.template run<Layout<256, 4, 4, false, 2048>>();
    if constexpr (F::MAX_WIDTH > 4096) {
        if (width <= 8192) return f.template run<Layout<512, 4, 4, false, 4096>>();
        return f.template run<Layout<512, 8, 4, false, 8192>>();
    }
    return 0;
}

}  // namespace eprow
