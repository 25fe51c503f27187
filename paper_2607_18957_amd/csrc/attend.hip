// ii_attend: attention of new tokens over a paged key/value cache.
#include <cmath>

#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

struct Attend {
    const uint8_t *q, *k, *v, *k_scale, *v_scale;
    uint8_t* out;
    int64_t q_row, q_head, out_row, out_head;  // strides, bytes
    int64_t page_stride, head_stride, token_stride;
    int64_t scale_page_stride, scale_head_stride, scale_token_stride;
    const int32_t *pages, *lengths, *q_start;
    int64_t pages_stride, capacity;  // capacity: keys a table's columns hold
    int64_t rows, window, num_pages;
    int32_t seqs, heads, group, page_bits;
    float scale;
};

template <class T, bool kQuant>
__device__ inline float kept(const Attend& p, const uint8_t* base, const uint8_t* scales,
                             int64_t page, int head, int64_t row, int d) {
    const uint8_t* at = base + page * p.page_stride + head * p.head_stride + row * p.token_stride;
    if (!kQuant) return (float)reinterpret_cast<const T*>(at)[d];
    const uint32_t e = scales[page * p.scale_page_stride + head * p.scale_head_stride +
                              row * p.scale_token_stride + d / 32];
    return __builtin_amdgcn_cvt_f32_fp8(at[d], 0) * __builtin_bit_cast(float, e ? e << 23 : 0x400000u);
}

// One wave a (row, query head): 64 keys at a time, a lane a key for the
// scores, a lane a few positions for the values.
template <class T, bool kQuant, int kDim>
__global__ __launch_bounds__(64) void attend_rows(Attend p) {
    __shared__ float qs[kDim], ps[64];
    __shared__ int64_t at[64];
    const int lane = threadIdx.x, head = blockIdx.y, kv = head / p.group;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        // the row's sequence
        int64_t seq = row, first = row, end = row + 1;
        if (p.q_start) {
            seq = -1;
            for (int b = 0; b < p.seqs; ++b)
                if (p.q_start[b] <= row && row < p.q_start[b + 1]) {
                    seq = b;
                    first = p.q_start[b];
                    end = p.q_start[b + 1];
                }
        }
        if (seq < 0 || seq >= p.seqs) continue;
        const int64_t pos = (int64_t)p.lengths[seq] - (end - first) + (row - first);
        const int64_t stop = min(pos + 1, p.capacity);
        const int64_t start = p.window ? max((int64_t)0, pos - p.window + 1) : 0;
        const T* q = reinterpret_cast<const T*>(p.q + row * p.q_row + head * p.q_head);
        __syncthreads();
        for (int d = lane; d < kDim; d += 64) qs[d] = (float)q[d];
        __syncthreads();
        float top = -INFINITY, sum = 0, acc[kDim / 64] = {};
        for (int64_t j0 = start; j0 < stop; j0 += 64) {
            const int64_t j = j0 + lane;
            float s = -INFINITY;
            int64_t page = -1;
            if (j < stop) page = p.pages[seq * p.pages_stride + (j >> p.page_bits)];
            const int64_t r = j & (((int64_t)1 << p.page_bits) - 1);
            if (page >= 0 && page < p.num_pages) {
                s = 0;
                for (int d = 0; d < kDim; ++d)
                    s += qs[d] * kept<T, kQuant>(p, p.k, p.k_scale, page, kv, r, d);
                s *= p.scale;
            } else {
                page = -1;
            }
            float m = s;
            for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
            const float next = fmaxf(top, m);
            if (next == -INFINITY) continue;  // nothing seen yet: alike in every lane
            const float keep = expf(top - next), w = page < 0 ? 0.0f : expf(s - next);
            top = next;
            __syncthreads();
            ps[lane] = w;
            at[lane] = page < 0 ? -1 : page << p.page_bits | r;
            __syncthreads();
            sum = sum * keep + w;
            for (int i = 0; i < kDim / 64; ++i) {
                acc[i] *= keep;
                for (int t = 0; t < 64; ++t)
                    if (at[t] >= 0)
                        acc[i] += ps[t] * kept<T, kQuant>(p, p.v, p.v_scale, at[t] >> p.page_bits, kv,
                                                          at[t] & (((int64_t)1 << p.page_bits) - 1),
                                                          lane + 64 * i);
            }
        }
        for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
        T* out = reinterpret_cast<T*>(p.out + row * p.out_row + head * p.out_head);
        for (int i = 0; i < kDim / 64; ++i) out[lane + 64 * i] = (T)(sum == 0 ? 0.0f : acc[i] / sum);
    }
}

template <class T, bool kQuant>
void launch(const Attend& p, int dim, hipStream_t stream) {
    const dim3 grid((uint32_t)std::min<int64_t>(p.rows, 1 << 20), p.heads);
    if (dim == 64)
        attend_rows<T, kQuant, 64><<<grid, 64, 0, stream>>>(p);
    else
        attend_rows<T, kQuant, 128><<<grid, 64, 0, stream>>>(p);
}

int run(const ii_attend_args& a, const ii_cache& c, hipStream_t stream) {
    const char* fn = "ii_attend";
    CacheRows held;
    int rc = check_cache(fn, c, &held);
    if (rc) return rc;
    if (!half_type(a.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, a.dtype);
    const bool quant = c.dtype == II_FP8_E4M3;
    if (!quant && c.dtype != a.dtype)
        return fail(II_EINVAL, "%s: a cache of type %d, queries of type %d", fn, c.dtype, a.dtype);
    if (a.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, a.reserved);
    if (a.heads < 1 || a.heads % c.heads || a.heads > 65535)
        return fail(II_EINVAL, "%s: %d query heads over %d cache heads", fn, a.heads, c.heads);
    if (a.rows < 0 || a.rows > INT32_MAX || a.seqs < 0 || a.seqs > 65535 || a.max_q < 0 ||
        a.max_len < 0 || a.window < 0)
        return fail(II_EINVAL, "%s: a size is out of range", fn);
    if (a.columns < 0 || a.columns > ((int64_t)1 << 40) / c.page || a.pages_stride < 0)
        return fail(II_EINVAL, "%s: a page table of %lld columns, stride %lld", fn,
                    (long long)a.columns, (long long)a.pages_stride);
    if (!std::isfinite(a.scale)) return fail(II_EINVAL, "%s: scale is not finite", fn);
    if (!a.q_start && a.rows != a.seqs)
        return fail(II_EINVAL, "%s: %lld rows for %lld sequences without q_start", fn,
                    (long long)a.rows, (long long)a.seqs);
    if (!a.rows || !a.seqs) return II_OK;
    Rows q, out, table, lengths, starts;
    if ((rc = check_heads(fn, "out", a.out, a.rows, a.heads, c.dim, a.out_row_stride,
                          a.out_head_stride, 2, true, &out)) ||
        (rc = check_heads(fn, "q", a.q, a.rows, a.heads, c.dim, a.q_row_stride, a.q_head_stride, 2,
                          false, &q)) ||
        (rc = check_rows(fn, "pages", a.pages, a.seqs, (uint64_t)a.columns * 4,
                         a.seqs > 1 ? (uint64_t)a.pages_stride * 4 : 0, 4, &table)) ||
        (rc = check_rows(fn, "lengths", a.lengths, 1, (uint64_t)a.seqs * 4, 0, 4, &lengths)) ||
        (rc = check_rows(fn, "q_start", a.q_start, a.q_start ? 1 : 0, ((uint64_t)a.seqs + 1) * 4, 0,
                         4, &starts)) ||
        (rc = check_work(fn, a.work, a.work_bytes)) || (rc = check_apart(fn, "q", out, q)) ||
        (rc = check_apart(fn, "pages", out, table)) ||
        (rc = check_apart(fn, "lengths", out, lengths)) ||
        (rc = check_apart(fn, "q_start", out, starts)))
        return rc;
    for (const Rows& r : held.all)
        if ((rc = check_apart(fn, "the cache", out, r))) return rc;
    const int64_t size = quant ? 1 : 2;
    Attend p;
    p.q = static_cast<const uint8_t*>(a.q);
    p.k = static_cast<const uint8_t*>(c.k);
    p.v = static_cast<const uint8_t*>(c.v);
    p.k_scale = c.k_scale;
    p.v_scale = c.v_scale;
    p.out = static_cast<uint8_t*>(a.out);
    p.q_row = a.q_row_stride * 2;
    p.q_head = a.q_head_stride * 2;
    p.out_row = a.out_row_stride * 2;
    p.out_head = a.out_head_stride * 2;
    p.page_stride = c.page_stride * size;
    p.head_stride = c.head_stride * size;
    p.token_stride = c.token_stride * size;
    p.scale_page_stride = c.scale_page_stride;
    p.scale_head_stride = c.scale_head_stride;
    p.scale_token_stride = c.scale_token_stride;
    p.pages = a.pages;
    p.lengths = a.lengths;
    p.q_start = a.q_start;
    p.pages_stride = a.pages_stride;
    p.capacity = a.columns * c.page;
    p.rows = a.rows;
    p.window = a.window;
    p.num_pages = c.pages;
    p.seqs = (int32_t)a.seqs;
    p.heads = a.heads;
    p.group = a.heads / c.heads;
    p.page_bits = __builtin_ctz(c.page);
    p.scale = a.scale;
    if (a.dtype == II_BF16)
        quant ? launch<__bf16, true>(p, c.dim, stream) : launch<__bf16, false>(p, c.dim, stream);
    else
        quant ? launch<_Float16, true>(p, c.dim, stream) : launch<_Float16, false>(p, c.dim, stream);
    return launched(fn);
}

}  // namespace
}  // namespace ii

extern "C" int ii_attend(const ii_attend_args* a, const ii_cache* c, hipStream_t stream) {
    if (!a || !c) return ii::fail(II_EINVAL, "ii_attend: an argument is NULL");
    return ii::run(*a, *c, stream);
}
