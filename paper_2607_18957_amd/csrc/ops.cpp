// Argument checks of the operators.
#include "ops.h"

#include <algorithm>

namespace ii {

static thread_local AllocInfo found;  // nothing between calls

Checks::Checks() { found = AllocInfo{}; }
Checks::~Checks() { found = AllocInfo{}; }

int check_rows(const char* fn, const char* what, const void* p, uint64_t rows, uint64_t width,
               uint64_t stride, uint64_t align, Rows* r) {
    *r = Rows{reinterpret_cast<uint64_t>(p), rows, width, stride};
    if (!rows || !width) return II_OK;
    if (!p) return fail(II_EINVAL, "%s: %s is NULL", fn, what);
    if (r->at % align || (rows > 1 && stride % align))
        return fail(II_EALIGN, "%s: %s (%#llx, stride %llu bytes) is not a multiple of %llu bytes",
                    fn, what, (unsigned long long)r->at, (unsigned long long)stride,
                    (unsigned long long)align);
    uint64_t span, end;
    if (__builtin_mul_overflow(rows - 1, stride, &span) ||
        __builtin_add_overflow(span, width, &span) || __builtin_add_overflow(r->at, span, &end))
        return fail(II_EOVERFLOW, "%s: %s: %llu rows of %llu bytes at stride %llu", fn, what,
                    (unsigned long long)rows, (unsigned long long)width,
                    (unsigned long long)stride);
    if (found.kind == AllocInfo::kDevice && found.extent && r->at >= found.base &&
        end <= found.base + found.size)
        return II_OK;
    found = alloc_info(r->at);
    if (!reachable(found, r->at, end))
        return fail(II_EINVAL, "%s: %s [%#llx, +%llu bytes) is not memory the device can reach: "
                    "not inside one device allocation or one pinned host allocation", fn, what,
                    (unsigned long long)r->at, (unsigned long long)span);
    return II_OK;
}

int check_apart(const char* fn, const char* what, const Rows& w, const Rows& r) {
    if (!w.rows || !w.width || !r.rows || !r.width) return II_OK;
    if (w.end() <= r.at || r.end() <= w.at) return II_OK;
    if (w.rows > 1 && r.rows > 1 && w.stride == r.stride && w.width <= w.stride) {
        const uint64_t s = w.stride;
        const uint64_t d = w.at >= r.at ? (w.at - r.at) % s : (s - (r.at - w.at) % s) % s;
        if (d >= r.width && d + w.width <= s) return II_OK;
    }
    return fail(II_EOVERLAP, "%s: what is written overlaps %s", fn, what);
}

int check_span(const char* fn, const char* what, const Axis* axes, int n, uint64_t width,
               bool apart, uint64_t* span, Nest* nest) {
    Axis by[3];
    int live = 0;
    for (int i = 0; i < n; ++i) {
        if (axes[i].count <= 1) continue;
        if (axes[i].stride < 0) return fail(II_EINVAL, "%s: a stride of %s is negative", fn, what);
        int j = live++;
        for (; j > 0 && by[j - 1].stride > axes[i].stride; --j) by[j] = by[j - 1];
        by[j] = axes[i];
    }
    uint64_t end = width;
    for (int i = 0; i < live; ++i) {
        if (apart && (uint64_t)by[i].stride < end)
            return fail(II_EINVAL, "%s: rows of %s meet (stride %lld bytes, %llu held)", fn, what,
                        (long long)by[i].stride, (unsigned long long)end);
        uint64_t more;
        if (__builtin_mul_overflow((uint64_t)by[i].count - 1, (uint64_t)by[i].stride, &more) ||
            __builtin_add_overflow(end, more, &end) || end > INT64_MAX)
            return fail(II_EOVERFLOW, "%s: the extent of %s", fn, what);
    }
    *span = end;
    if (nest) {
        nest->width = width;
        nest->axes = live;
        std::copy(by, by + live, nest->by);
    }
    return II_OK;
}

bool nests_meet(const Nest& a, const Nest& b) {
    const auto extent = [](const Nest& x) {
        uint64_t e = x.width;
        for (int i = 0; i < x.axes; ++i) e += (uint64_t)(x.by[i].count - 1) * x.by[i].stride;
        return e;
    };
    // distances, as the arrays may end past the last address
    if (b.at >= a.at ? b.at - a.at >= extent(a) : a.at - b.at >= extent(b)) return false;
    if (!a.axes || !b.axes || a.by[a.axes - 1].stride != b.by[b.axes - 1].stride) return true;
    // Place i of a against place j of b along this axis: what lies inside a
    // place is shorter than the stride, so it meets that of i - j = q or q + 1,
    // b being q strides and a part of one after a.
    Nest x = a, y = b;
    const Axis& ax = a.by[--x.axes];
    const Axis& bx = b.by[--y.axes];
    const int64_t s = ax.stride, d = (int64_t)(b.at - a.at);  // less than 2^63 apart
    const int64_t q = d >= 0 ? d / s : -((-d + s - 1) / s);
    for (int64_t i = q; i <= q + 1; ++i) {
        if (i >= ax.count || i <= -bx.count) continue;
        x.at = a.at + (uint64_t)(i * s);
        if (nests_meet(x, y)) return true;
    }
    return false;
}

int check_heads(const char* fn, const char* what, const void* p, int64_t tokens, int64_t heads,
                int64_t dim, int64_t token_stride, int64_t head_stride, int size, bool written,
                Rows* r, Nest* nest) {
    if (!tokens) {
        *r = Rows{};
        return II_OK;
    }
    int64_t ts, hs;
    if (__builtin_mul_overflow(token_stride, (int64_t)size, &ts) ||
        __builtin_mul_overflow(head_stride, (int64_t)size, &hs))
        return fail(II_EOVERFLOW, "%s: the strides of %s", fn, what);
    if ((tokens > 1 && ts % 16) || (heads > 1 && hs % 16))
        return fail(II_EALIGN, "%s: strides of %s (%lld, %lld bytes) are not multiples of 16 bytes",
                    fn, what, (long long)ts, (long long)hs);
    const Axis axes[2] = {{tokens, ts}, {heads, hs}};
    uint64_t token, span;
    int rc = check_span(fn, what, axes + 1, 1, dim * size, written, &token);
    if (!rc) rc = check_span(fn, what, axes, 2, dim * size, written, &span, nest);
    if (rc) return rc;
    if (nest) nest->at = reinterpret_cast<uint64_t>(p);
    // tokens one after another, or one range
    if (tokens > 1 && token <= (uint64_t)ts) return check_rows(fn, what, p, tokens, token, ts, 16, r);
    return check_rows(fn, what, p, 1, span, 0, 16, r);
}

int check_heads_apart(const char* fn, const char* what, const Rows& written, const Nest& w,
                      const Rows& read, const Nest& r) {
    if (!written.rows || !read.rows) return II_OK;
    // rows of what is read may meet each other, which nests_meet does not expect
    uint64_t end = r.width;
    bool apart = true;
    for (int i = 0; i < r.axes; ++i) {
        apart &= (uint64_t)r.by[i].stride >= end;
        end += (uint64_t)(r.by[i].count - 1) * r.by[i].stride;
    }
    if (apart && !nests_meet(w, r)) return II_OK;
    return check_apart(fn, what, written, read);
}

int check_cache(const char* fn, const ii_cache& c, bool written, CacheRows* held) {
    const bool quant = c.dtype == II_FP8_E4M3;
    if (!quant && !half_type(c.dtype)) return fail(II_EINVAL, "%s: cache of type %d", fn, c.dtype);
    if (c.heads < 1) return fail(II_EINVAL, "%s: cache of %d heads", fn, c.heads);
    if (c.dim != 64 && c.dim != 128) return fail(II_EINVAL, "%s: heads of %d elements", fn, c.dim);
    if (c.page < 1 || (c.page & (c.page - 1)))
        return fail(II_EINVAL, "%s: pages of %d tokens, not a power of two", fn, c.page);
    if (c.pages < 0 || c.pages > INT32_MAX)
        return fail(II_EINVAL, "%s: %lld pages", fn, (long long)c.pages);
    *held = CacheRows{};
    if (!c.pages) return II_OK;
    const int64_t size = quant ? 1 : 2;
    const char* const what[4] = {"the cache's k", "the cache's v", "k_scale", "v_scale"};
    const void* const at[4] = {c.k, c.v, c.k_scale, c.v_scale};
    const int arrays = quant ? 4 : 2;
    uint64_t span[4];
    Nest nest[4];
    for (int i = 0; i < arrays; ++i) {
        Axis axes[3] = {{c.pages, c.page_stride}, {c.heads, c.head_stride}, {c.page, c.token_stride}};
        if (i >= 2) {
            axes[0].stride = c.scale_page_stride;
            axes[1].stride = c.scale_head_stride;
            axes[2].stride = c.scale_token_stride;
        }
        const int64_t align = i < 2 ? 16 : c.dim / 32;
        for (Axis& a : axes) {
            if (__builtin_mul_overflow(a.stride, i < 2 ? size : 1, &a.stride))
                return fail(II_EOVERFLOW, "%s: the strides of %s", fn, what[i]);
            if (a.count > 1 && a.stride % align)
                return fail(II_EALIGN, "%s: a stride of %s (%lld bytes) is not a multiple of %lld "
                            "bytes", fn, what[i], (long long)a.stride, (long long)align);
        }
        const int rc = check_span(fn, what[i], axes, 3, i < 2 ? c.dim * size : c.dim / 32, true,
                                  &span[i], &nest[i]);
        if (rc) return rc;
        nest[i].at = reinterpret_cast<uint64_t>(at[i]);
        for (int j = 0; j < i && written; ++j)
            if (at[i] && at[j] && nests_meet(nest[i], nest[j]))
                return fail(II_EOVERLAP, "%s: %s and %s meet", fn, what[j], what[i]);
    }
    for (int i = 0; i < arrays; ++i) {
        const int rc = check_rows(fn, what[i], at[i], 1, span[i], 0, i < 2 ? 16 : c.dim / 32,
                                  &held->all[i]);
        if (rc) return rc;
    }
    return II_OK;
}

int check_move(const char* fn, const ii_cache& c, const ii_tokens& f, bool write, TokenRows* r) {
    CacheRows& held = r->cache;
    int rc = check_cache(fn, c, write, &held);
    if (rc) return rc;
    if (!half_type(f.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, f.dtype);
    if (c.dtype != II_FP8_E4M3 && c.dtype != f.dtype)
        return fail(II_EINVAL, "%s: a cache of type %d, tokens of type %d", fn, c.dtype, f.dtype);
    if (f.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, f.reserved);
    if (f.tokens < 0 || f.tokens > (int64_t)1 << 40)
        return fail(II_EINVAL, "%s: %lld tokens", fn, (long long)f.tokens);
    if (!f.tokens) return II_OK;
    Rows &slots = r->slots, *rows = r->kv;
    Nest* nest = r->nest;
    rc = check_rows(fn, "slots", f.slots, 1, (uint64_t)f.tokens * 8, 0, 8, &slots);
    if (rc) return rc;
    const int64_t ts[2] = {f.k_token_stride, f.v_token_stride};
    const int64_t hs[2] = {f.k_head_stride, f.v_head_stride};
    void* const at[2] = {f.k, f.v};
    const char* const what[2] = {"k", "v"};
    for (int i = 0; i < 2; ++i) {
        rc = check_heads(fn, what[i], at[i], f.tokens, c.heads, c.dim, ts[i], hs[i], 2, !write,
                         &rows[i], &nest[i]);
        if (rc) return rc;
    }
    for (int i = 0; i < 2; ++i) {
        if (!write && (rc = check_apart(fn, "slots", rows[i], slots))) return rc;
        for (const Rows& r : held.all) {
            rc = write ? check_apart(fn, what[i], r, rows[i]) : check_apart(fn, "the cache", rows[i], r);
            if (rc) return rc;
        }
    }
    if (write)
        for (const Rows& r : held.all)
            if ((rc = check_apart(fn, "slots", r, slots))) return rc;
    if (!write && nests_meet(nest[0], nest[1])) return fail(II_EOVERLAP, "%s: k and v meet", fn);
    return II_OK;
}

int check_work(const char* fn, const void* work, uint64_t bytes, Rows* r) {
    *r = Rows{};
    if (!work && !bytes) return II_OK;
    const int rc = check_rows(fn, "work", work, 1, bytes, 0, 16, r);
    if (r->width > II_WORK_BYTES) r->width = II_WORK_BYTES;
    return rc;
}

int launched(const char* fn) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? II_OK : fail(II_EHIP, "%s: %s", fn, hipGetErrorString(e));
}

}  // namespace ii
