// ii_linear: products with weight matrices, and their epilogue.
#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

template <class T>
struct Linear {
    const T *x, *w, *w2, *bias, *bias2, *residual;
    void* out;
    int64_t x_stride, w_stride, w2_stride, residual_stride, out_stride;
    int32_t m, n, k, act;
    bool out_f32;
};

__device__ inline float activate(float y, int act) {
    switch (act) {
    case II_ACT_RELU: return y < 0 ? 0.0f : y;  // NaN stays
    case II_ACT_SILU: return y / (1.0f + expf(-y));
    case II_ACT_GELU: return 0.5f * y * (1.0f + erff(y * 0.70710678118654752f));
    }
    return y;
}

template <class T, bool kGated>
__device__ inline void put(const Linear<T>& p, int64_t i, int64_t j, float y, float z) {
    if (p.bias) y += (float)p.bias[j];
    y = activate(y, p.act);
    if (kGated) {
        if (p.bias2) z += (float)p.bias2[j];
        y *= z;
    }
    if (p.residual) y += (float)p.residual[i * p.residual_stride + j];
    if (p.out_f32)
        static_cast<float*>(p.out)[i * p.out_stride + j] = y;
    else
        static_cast<T*>(p.out)[i * p.out_stride + j] = (T)y;
}

// 64 tokens by 64 weight rows a workgroup of four waves, 32 elements of k at
// a time through LDS, every element loaded by itself: rows at any address.
constexpr int kElemTile = 64, kElemK = 32, kElemPad = 8;

template <class T>
__device__ inline void stage_elements(T (*to)[kElemK + kElemPad], const T* from, int64_t stride,
                                      int64_t row0, int64_t rows, int64_t k0, int64_t k) {
    const int t = threadIdx.x, r = t / 4, c = t % 4 * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        T v = (T)0.0f;
        if (row0 + r < rows && k0 + c + j < k) v = from[(row0 + r) * stride + k0 + c + j];
        to[r][c + j] = v;
    }
}

template <class T, bool kGated>
__global__ __launch_bounds__(256) void linear_elements(Linear<T> p) {
    using x8 = typename Vec<T>::x8;
    __shared__ T xs[kElemTile][kElemK + kElemPad];
    __shared__ T ws[kGated ? 2 : 1][kElemTile][kElemK + kElemPad];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, part = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * kElemTile, m0 = (int64_t)blockIdx.y * kElemTile;
    f32x4 acc[kGated ? 2 : 1][4] = {};
    for (int64_t k0 = 0; k0 < p.k; k0 += kElemK) {
        stage_elements(xs, p.x, p.x_stride, m0, p.m, k0, p.k);
        stage_elements(ws[0], p.w, p.w_stride, n0, p.n, k0, p.k);
        if (kGated) stage_elements(ws[kGated], p.w2, p.w2_stride, n0, p.n, k0, p.k);
        __syncthreads();
#pragma unroll
        for (int g = 0; g <= (kGated ? 1 : 0); ++g) {
            const x8 a = *reinterpret_cast<const x8*>(&ws[g][wave * 16 + row][part * 8]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                acc[g][t] = mfma16(a, *reinterpret_cast<const x8*>(&xs[t * 16 + row][part * 8]),
                                   acc[g][t]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t i = m0 + t * 16 + row, j = n0 + wave * 16 + part * 4 + r;
            if (i < p.m && j < p.n) put<T, kGated>(p, i, j, acc[0][t][r], acc[kGated][t][r]);
        }
}

template <class T, bool kGated>
void launch(const Linear<T>& p, hipStream_t stream) {
    const dim3 grid((p.n + kElemTile - 1) / kElemTile, (p.m + kElemTile - 1) / kElemTile);
    linear_elements<T, kGated><<<grid, 256, 0, stream>>>(p);
}

template <class T>
int run(const ii_linear_args& a, hipStream_t stream) {
    Linear<T> p;
    p.x = static_cast<const T*>(a.x);
    p.w = static_cast<const T*>(a.w);
    p.w2 = static_cast<const T*>(a.w2);
    p.bias = static_cast<const T*>(a.bias);
    p.bias2 = static_cast<const T*>(a.bias2);
    p.residual = static_cast<const T*>(a.residual);
    p.out = a.out;
    p.x_stride = a.x_stride;
    p.w_stride = a.w_stride;
    p.w2_stride = a.w2_stride;
    p.residual_stride = a.residual_stride;
    p.out_stride = a.out_stride;
    p.m = (int32_t)a.m;
    p.n = (int32_t)a.n;
    p.k = (int32_t)a.k;
    p.act = a.act;
    p.out_f32 = a.out_dtype == II_F32;
    if (p.w2)
        launch<T, true>(p, stream);
    else
        launch<T, false>(p, stream);
    return launched("ii_linear");
}

int check(const ii_linear_args& a) {
    const char* fn = "ii_linear";
    constexpr int64_t most = INT32_MAX;
    if (!half_type(a.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, a.dtype);
    if (a.out_dtype != a.dtype && a.out_dtype != II_F32)
        return fail(II_EINVAL, "%s: out_dtype %d", fn, a.out_dtype);
    if (a.act < II_ACT_NONE || a.act > II_ACT_GELU)
        return fail(II_EINVAL, "%s: act %d", fn, a.act);
    if (a.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, a.reserved);
    if (a.m < 0 || a.n < 0 || a.k < 0 || a.m > most || a.n > most || a.k > most)
        return fail(II_EINVAL, "%s: sizes %lld, %lld, %lld", fn, (long long)a.m, (long long)a.n,
                    (long long)a.k);
    if (a.bias2 && !a.w2) return fail(II_EINVAL, "%s: bias2 without w2", fn);
    if (a.x_stride < 0 || a.w_stride < 0 || a.w2_stride < 0 || a.residual_stride < 0)
        return fail(II_EINVAL, "%s: a stride is negative", fn);
    if (a.m > 1 && a.out_stride < a.n)
        return fail(II_EINVAL, "%s: rows of out meet (stride %lld, %lld columns)", fn,
                    (long long)a.out_stride, (long long)a.n);
    if (!a.m || !a.n) return II_OK;
    const uint64_t m = a.m, n = a.n, k = a.k, size = 2, osize = a.out_dtype == II_F32 ? 4 : 2;
    Rows out, r;
    int rc = check_rows(fn, "out", a.out, m, n * osize, (m > 1 ? a.out_stride : 0) * osize, osize,
                        &out);
    if (rc) return rc;
    const struct {
        const char* what;
        const void* p;
        uint64_t rows, width, stride;
        bool need;
    } ins[] = {{"x", a.x, m, k, (uint64_t)a.x_stride, true},
               {"w", a.w, n, k, (uint64_t)a.w_stride, true},
               {"w2", a.w2, n, k, (uint64_t)a.w2_stride, false},
               {"bias", a.bias, 1, n, 0, false},
               {"bias2", a.bias2, 1, n, 0, false},
               {"residual", a.residual, m, n, (uint64_t)a.residual_stride, false}};
    for (const auto& in : ins) {
        if (!in.p && !in.need) continue;
        uint64_t stride;
        if (__builtin_mul_overflow(in.rows > 1 ? in.stride : 0, size, &stride))
            return fail(II_EOVERFLOW, "%s: the stride of %s", fn, in.what);
        rc = check_rows(fn, in.what, in.p, in.rows, in.width * size, stride, size, &r);
        if (rc) return rc;
        if (in.p == a.residual && in.p == a.out && a.out_dtype == a.dtype &&
            (m == 1 || a.residual_stride == a.out_stride) && in.rows == m && in.width == n)
            continue;  // each element is read by the lane that then writes it
        rc = check_apart(fn, in.what, out, r);
        if (rc) return rc;
    }
    return check_work(fn, a.work, a.work_bytes);
}

}  // namespace
}  // namespace ii

extern "C" int ii_linear(const ii_linear_args* a, hipStream_t stream) {
    if (!a) return ii::fail(II_EINVAL, "ii_linear: args is NULL");
    if (const int rc = ii::check(*a)) return rc;
    if (!a->m || !a->n) return II_OK;
    return a->dtype == II_BF16 ? ii::run<__bf16>(*a, stream) : ii::run<_Float16>(*a, stream);
}
