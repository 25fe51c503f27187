// ii_norm: the norm after a block, its gate and scale, the residual stream and
// the norm before the next block, in one pass over the rows.
//
// A group of threads holds a row in registers, so that each input is read once
// and each output written once whatever the norms need of the row. Squares are
// summed in 64 bits: a sum of squares of 32-bit values passes float's range on
// both sides, and the additions cost nothing beside the memory. The norm before
// the next block takes the stream as it was before its rounding.
//
// Bound by memory: 16384 x 8192, normalised before and after, with a gate for each
// element and a stream of 32 bits, 334 us, 5.6 TB/s; a copy of 2 GiB reaches 4.9.
// 65536 rows of 1001, read by the element, 162 us, 3.2 TB/s.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

template <class T, class S>
struct Norm {
    const T *x, *gate, *post_weight, *post_bias, *weight, *bias;
    const S* residual;
    S* sum;
    T* out;
    int64_t x_stride, gate_stride, residual_stride, sum_stride, out_stride;
    int32_t m, n, kind;
    bool post;
    float scale, eps, offset;
};

// Eight elements as they lie in memory.
template <class V>
union Eight {
    V at[8];
    u32x4 word[sizeof(V) / 2];
    __device__ Eight() {}
};

// Keeps the compiler from holding what it made of x before.
__device__ inline void anew(float& x) { asm volatile("" : "+v"(x)); }

// The sum over the kThreads threads of a row, in the order of their places, so
// that it is alike in all of them. `turn` tells one sum's room from the next's.
template <int kThreads>
__device__ inline double row_sum(double v, int turn) {
#pragma unroll
    for (int d = 1; d < std::min(kThreads, 64); d *= 2) v += __shfl_xor(v, d);
    if constexpr (kThreads > 64) {
        __shared__ double part[2][kThreads / 64];
        if (threadIdx.x % 64 == 0) part[turn % 2][threadIdx.x / 64] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) v += part[turn % 2][w];
    }
    return v;
}

// kThreads threads hold a row, kWords words of 8 elements each: words are
// whole (kWide), or a word's elements lie kThreads apart.
template <class T, class S, int kThreads, int kWords, bool kWide, bool kLayer>
__global__ __launch_bounds__(kThreads > 256 ? kThreads : 256) void norm_rows(Norm<T, S> p) {
    constexpr int kBlock = kThreads > 256 ? kThreads : 256, kRows = kBlock / kThreads;
    // several rows a wave: addresses of their own, whole words only
    constexpr bool kPart = kThreads < 64;
    static_assert((kRows == 1 || kThreads <= 64) && (!kPart || (kWide && kWords == 1)));
    const int t = threadIdx.x % kThreads;
    // a thread's first element, and how far the others are from it
    const int first = kWide ? t * 8 : t;
    const auto away = [](int w, int j) {
        return kWide ? w * kThreads * 8 + j : (w * 8 + j) * kThreads;
    };
    // Rows are read and written by buffer instructions, which give zeros past a
    // row's end and leave out what would be written there.
    const auto get = [&](auto* from, int w) {
        using V = std::remove_const_t<std::remove_pointer_t<decltype(from)>>;
        Eight<V> v;
        if constexpr (kPart) {
#pragma unroll
            for (int h = 0; h < (int)sizeof(v) / 16; ++h)
                v.word[h] = first < p.n ? reinterpret_cast<const u32x4*>(from + first)[h] : u32x4{};
            return v;
        }
        const Rsrc row = buffer(from, (int64_t)p.n * (int)sizeof(V));
        if constexpr (kWide) {
#pragma unroll
            for (int h = 0; h < (int)sizeof(v) / 16; ++h)
                v.word[h] = __builtin_amdgcn_raw_buffer_load_b128(
                    row, (first + away(w, 0)) * (int)sizeof(V) + h * 16, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int offset = (first + away(w, j)) * (int)sizeof(V);
                if constexpr (sizeof(V) == 4)
                    v.at[j] = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b32(row, offset, 0, 0));
                else
                    v.at[j] = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b16(row, offset, 0, 0));
            }
        }
        return v;
    };
    const auto put = [&](auto* to, int w, const float (&from)[8]) {
        using V = std::remove_pointer_t<decltype(to)>;
        Eight<V> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.at[j] = (V)from[j];
        if constexpr (kPart) {
#pragma unroll
            for (int h = 0; h < (int)sizeof(v) / 16; ++h)
                if (first < p.n) reinterpret_cast<u32x4*>(to + first)[h] = v.word[h];
            return;
        }
        const Rsrc row = buffer(to, (int64_t)p.n * (int)sizeof(V));
        if constexpr (kWide) {
#pragma unroll
            for (int h = 0; h < (int)sizeof(v) / 16; ++h)
                __builtin_amdgcn_raw_buffer_store_b128(
                    v.word[h], row, (first + away(w, 0)) * (int)sizeof(V) + h * 16, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int offset = (first + away(w, j)) * (int)sizeof(V);
                if constexpr (sizeof(V) == 4)
                    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v.at[j]), row,
                                                          offset, 0, 0);
                else
                    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v.at[j]), row,
                                                          offset, 0, 0);
            }
        }
    };
    int turn = 0;
    // Past the row's end y is 0 but for what a mean took off it.
    const auto normalise = [&](float (&y)[kWords][8], const T* weight, const T* bias) {
        double mean = 0, squares = 0;
        if constexpr (kLayer) {
#pragma unroll
            for (int w = 0; w < kWords; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) mean += first + away(w, j) < p.n ? y[w][j] : 0.0f;
            mean = row_sum<kThreads>(mean, turn++) / p.n;
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (kLayer) anew(y[w][j]);
                const double d = kLayer && first + away(w, j) >= p.n ? 0.0 : (double)y[w][j] - mean;
                squares = fma(d, d, squares);
            }
        const double root = 1.0 / sqrt(row_sum<kThreads>(squares, turn++) / p.n + (double)p.eps);
        // The mean as two floats: rounded to one it is off by 2^-24 of itself, which
        // is steps of the result where the deviation is that much smaller. y - mu is
        // exact there, so what is left of the mean comes off after it, with the product.
        const float r = (float)root, mu = (float)mean, rest = (float)(mean - mu) * r;
        if (r > 0x1p-100f && r < 0x1p100f) {
#pragma unroll
            for (int w = 0; w < kWords; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) y[w][j] = kLayer ? fmaf(y[w][j] - mu, r, -rest) : y[w][j] * r;
        } else {  // what 32 bits cannot hold, of the root or of y - mean
#pragma unroll
            for (int w = 0; w < kWords; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    anew(y[w][j]);
                    y[w][j] = (float)(((double)y[w][j] - mean) * root);
                }
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            if (weight) {
                const auto a = get(weight, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[w][j] *= (float)a.at[j] + p.offset;
            }
            if (bias) {
                const auto b = get(bias, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[w][j] += (float)b.at[j];
            }
        }
    };

    int mine = threadIdx.x / kThreads;
    if (!kPart) mine = __builtin_amdgcn_readfirstlane(mine);  // alike in a wave
    for (int64_t i = (int64_t)blockIdx.x * kRows + mine; i < p.m; i += (int64_t)gridDim.x * kRows) {
        // all loads are on their way before the first sum
        Eight<T> x[kWords], g[kWords];
        Eight<S> r[kWords];
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            x[w] = get(p.x + i * p.x_stride, w);
            if (p.gate) g[w] = get(p.gate + i * p.gate_stride, w);
            if (p.residual) r[w] = get(p.residual + i * p.residual_stride, w);
        }
        float y[kWords][8];
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[w][j] = (float)x[w].at[j];
        if (p.post) normalise(y, p.post_weight, p.post_bias);
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = y[w][j] * p.scale;
                if (p.gate) v *= (float)g[w].at[j];
                if (p.residual) v += (float)r[w].at[j];
                y[w][j] = v;
            }
            if (p.sum) put(p.sum + i * p.sum_stride, w, y[w]);
        }
        if (p.out) {
            normalise(y, p.weight, p.bias);
#pragma unroll
            for (int w = 0; w < kWords; ++w) put(p.out + i * p.out_stride, w, y[w]);
        }
    }
}

template <class T, class S, int kThreads, int kWords>
void rows_launch(const Norm<T, S>& p, bool wide, hipStream_t stream) {
    constexpr int kBlock = kThreads > 256 ? kThreads : 256;
    // a dispatch counts its work-items in 32 bits
    const uint32_t grid = (uint32_t)std::min<int64_t>(groups(p.m, kBlock / kThreads), 1 << 21);
    const bool layer = p.kind == II_NORM_LAYER;
    if (wide) {
        if (layer)
            norm_rows<T, S, kThreads, kWords, true, true><<<grid, kBlock, 0, stream>>>(p);
        else
            norm_rows<T, S, kThreads, kWords, true, false><<<grid, kBlock, 0, stream>>>(p);
    } else if constexpr (kThreads >= 64) {
        if (layer)
            norm_rows<T, S, kThreads, kWords, false, true><<<grid, kBlock, 0, stream>>>(p);
        else
            norm_rows<T, S, kThreads, kWords, false, false><<<grid, kBlock, 0, stream>>>(p);
    }
}

template <class T, class S>
void launch(const Norm<T, S>& p, bool wide, hipStream_t stream) {
    // Words of a row in as few threads as keep the loads of a row apart from the
    // next's, for some words each where that hides more: 16384 x 4096 with a
    // residual 91 us by 512 threads against 96 by 256 of two words, 16384 x 8192
    // normalised twice 333 by 256 of four against 338 by 512 of two, 2049 x 32768
    // 110 by 1024 of four against 120 by 512 of eight. Short rows share a wave:
    // 65536 x 128 13 us against 25 with a wave each.
    if (wide && p.n <= 128) return rows_launch<T, S, 16, 1>(p, wide, stream);
    if (wide && p.n <= 256) return rows_launch<T, S, 32, 1>(p, wide, stream);
    if (p.n <= 512) return rows_launch<T, S, 64, 1>(p, wide, stream);
    if (p.n <= 2048) return rows_launch<T, S, 256, 1>(p, wide, stream);
    if (p.n <= 4096) return rows_launch<T, S, 512, 1>(p, wide, stream);
    if (p.n <= 8192) return rows_launch<T, S, 256, 4>(p, wide, stream);
    if (p.n <= 16384) return rows_launch<T, S, 512, 4>(p, wide, stream);
    rows_launch<T, S, 1024, 4>(p, wide, stream);
}

template <class T, class S>
int run(const ii_norm_args& a, hipStream_t stream) {
    Norm<T, S> p;
    p.x = static_cast<const T*>(a.x);
    p.gate = static_cast<const T*>(a.gate);
    p.residual = static_cast<const S*>(a.residual);
    p.post_weight = static_cast<const T*>(a.post_weight);
    p.post_bias = static_cast<const T*>(a.post_bias);
    p.weight = static_cast<const T*>(a.weight);
    p.bias = static_cast<const T*>(a.bias);
    p.sum = static_cast<S*>(a.sum);
    p.out = static_cast<T*>(a.out);
    // the stride of a single row says nothing of how it can be read
    const auto stride = [&](int64_t s) { return a.m > 1 ? s : 0; };
    p.x_stride = stride(a.x_stride);
    p.gate_stride = stride(a.gate_stride);
    p.residual_stride = stride(a.residual_stride);
    p.sum_stride = stride(a.sum_stride);
    p.out_stride = stride(a.out_stride);
    p.m = (int32_t)a.m;
    p.n = (int32_t)a.n;
    p.kind = a.kind;
    p.post = a.post != 0;
    p.scale = a.scale;
    p.eps = a.eps;
    p.offset = a.offset;
    const auto word = [](const void* at, int64_t s, size_t size) {
        return !at || (reinterpret_cast<uintptr_t>(at) % 16 == 0 && s * size % 16 == 0);
    };
    const bool wide = a.n % 8 == 0 && word(p.x, p.x_stride, 2) && word(p.gate, p.gate_stride, 2) &&
                      word(p.residual, p.residual_stride, sizeof(S)) &&
                      word(p.sum, p.sum_stride, sizeof(S)) && word(p.out, p.out_stride, 2) &&
                      word(p.post_weight, 0, 2) && word(p.post_bias, 0, 2) &&
                      word(p.weight, 0, 2) && word(p.bias, 0, 2);
    launch(p, wide, stream);
    return launched("ii_norm");
}

int check(const ii_norm_args& a) {
    const char* fn = "ii_norm";
    if (!half_type(a.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, a.dtype);
    if (a.stream_dtype != a.dtype && a.stream_dtype != II_F32)
        return fail(II_EINVAL, "%s: stream_dtype %d", fn, a.stream_dtype);
    if (a.kind != II_NORM_RMS && a.kind != II_NORM_LAYER)
        return fail(II_EINVAL, "%s: kind %d", fn, a.kind);
    if (a.post != 0 && a.post != 1) return fail(II_EINVAL, "%s: post is %d", fn, a.post);
    if (a.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, a.reserved);
    if (a.m < 0 || a.m > INT32_MAX || a.n < 0 || a.n > 32768)
        return fail(II_EINVAL, "%s: %lld rows of %lld elements", fn, (long long)a.m, (long long)a.n);
    if (!std::isfinite(a.scale) || !std::isfinite(a.offset) || !std::isfinite(a.eps) || a.eps < 0)
        return fail(II_EINVAL, "%s: scale %g, eps %g, offset %g", fn, a.scale, a.eps, a.offset);
    if (!a.m || !a.n) return II_OK;  // operands of no elements may be NULL
    if (!a.post && (a.post_weight || a.post_bias))
        return fail(II_EINVAL, "%s: post_weight or post_bias without post", fn);
    if (!a.out && (a.weight || a.bias)) return fail(II_EINVAL, "%s: weight or bias without out", fn);
    if (!a.out && !a.sum) return fail(II_EINVAL, "%s: neither sum nor out", fn);
    if (a.x_stride < 0 || a.gate_stride < 0 || a.residual_stride < 0)
        return fail(II_EINVAL, "%s: a stride is negative", fn);
    if (a.m > 1 && ((a.sum && a.sum_stride < a.n) || (a.out && a.out_stride < a.n)))
        return fail(II_EINVAL, "%s: rows of sum or out meet (strides %lld, %lld, %lld elements)", fn,
                    (long long)a.sum_stride, (long long)a.out_stride, (long long)a.n);
    const uint64_t m = a.m, n = a.n, wide = a.stream_dtype == II_F32 ? 4 : 2;
    struct Operand {
        const char* what;
        const void* p;
        uint64_t rows;
        int64_t stride;
        uint64_t size;
        bool need;
        Rows r;
    } ops[] = {{"sum", a.sum, m, a.sum_stride, wide, false, {}},
               {"out", a.out, m, a.out_stride, 2, false, {}},
               {"x", a.x, m, a.x_stride, 2, true, {}},
               {"residual", a.residual, m, a.residual_stride, wide, false, {}},
               {"gate", a.gate, m, a.gate_stride, 2, false, {}},
               {"post_weight", a.post_weight, 1, 0, 2, false, {}},
               {"post_bias", a.post_bias, 1, 0, 2, false, {}},
               {"weight", a.weight, 1, 0, 2, false, {}},
               {"bias", a.bias, 1, 0, 2, false, {}}};
    for (Operand& o : ops) {
        if (!o.p && !o.need) continue;
        uint64_t stride;
        if (__builtin_mul_overflow((uint64_t)(o.rows > 1 ? o.stride : 0), o.size, &stride))
            return fail(II_EOVERFLOW, "%s: the stride of %s", fn, o.what);
        const int rc = check_rows(fn, o.what, o.p, o.rows, n * o.size, stride, o.size, &o.r);
        if (rc) return rc;
    }
    if (const int rc = check_apart(fn, "out", ops[0].r, ops[1].r)) return rc;
    for (int w = 0; w < 2; ++w)
        for (int i = 2; i < 9; ++i) {
            const Rows &to = ops[w].r, &from = ops[i].r;
            // each element is read by the thread that then writes it
            const bool same = (w == 0 && i == 3) || (w == 1 && i == 2);
            if (same && to.at == from.at && (m == 1 || to.stride == from.stride)) continue;
            if (const int rc = check_apart(fn, ops[i].what, to, from)) return rc;
        }
    return II_OK;
}

}  // namespace
}  // namespace ii

extern "C" int ii_norm(const ii_norm_args* a, hipStream_t stream) {
    if (!a) return ii::fail(II_EINVAL, "ii_norm: args is NULL");
    {
        const ii::Checks checks;
        if (const int rc = ii::check(*a)) return rc;
    }
    if (!a->m || !a->n) return II_OK;
    const bool wide = a->stream_dtype == II_F32;
    if (a->dtype == II_BF16)
        return wide ? ii::run<__bf16, float>(*a, stream) : ii::run<__bf16, __bf16>(*a, stream);
    return wide ? ii::run<_Float16, float>(*a, stream) : ii::run<_Float16, _Float16>(*a, stream);
}
