// Argument checks that the operators share.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "ii_internal.h"
#include "ii_ops.h"
#include "reach.h"

namespace ii {

// Rows of memory an operator touches: `rows` rows of `width` bytes, `stride`
// bytes apart.
struct Rows {
    uint64_t at = 0, rows = 0, width = 0, stride = 0;
    uint64_t end() const { return rows && width ? at + (rows - 1) * stride + width : at; }
};

// One call's checks. The allocation found last is kept until the call's end:
// ranges of one allocation, one after another, cost one query.
struct Checks {
    Checks();
    ~Checks();
};

// Form *r and check it: present, aligned, no overflow, inside one allocation
// the device reaches. Empty ranges pass whatever their address.
int check_rows(const char* fn, const char* what, const void* p, uint64_t rows, uint64_t width,
               uint64_t stride, uint64_t align, Rows* r);

// What is written may not meet what is read. Rows at one stride whose columns
// are apart (slices of a fused buffer) do not.
int check_apart(const char* fn, const char* what, const Rows& written, const Rows& read);

// [count][stride] axes around a contiguous row of `width` bytes, strides in
// bytes: *span receives the bytes from the first to the last, and what no two
// rows share (`apart`) is required of memory that is written. *nest (if not
// NULL) receives the axes of more than one place, the least stride first.
struct Axis {
    int64_t count, stride;
};
struct Nest {
    uint64_t at, width;
    int axes;
    Axis by[3];
};
int check_span(const char* fn, const char* what, const Axis* axes, int n, uint64_t width,
               bool apart, uint64_t* span, Nest* nest = nullptr);

// Whether two arrays, each with rows apart, share a byte. Exact where strides
// agree from the largest down to where one array's rows lie within the other's
// gaps (arrays of one shape in one buffer, in any order of axes); where they do
// not agree, arrays whose extents meet count as meeting.
bool nests_meet(const Nest& a, const Nest& b);

// [tokens][heads][dim] of `size`-byte elements at strides in elements.
int check_heads(const char* fn, const char* what, const void* p, int64_t tokens, int64_t heads,
                int64_t dim, int64_t token_stride, int64_t head_stride, int size, bool written,
                Rows* r, Nest* nest = nullptr);

// check_apart for heads: those of one token may lie between another array's.
int check_heads_apart(const char* fn, const char* what, const Rows& written, const Nest& w,
                      const Rows& read, const Nest& r);

// The memory of a cache: keys, values and their scales (empty without them).
struct CacheRows {
    Rows all[4];
};
int check_cache(const char* fn, const ii_cache& c, bool written, CacheRows* held);

// Tokens on their way into a cache (write) or out of it.
struct TokenRows {
    CacheRows cache;
    Rows kv[2], slots;  // slots and kv are empty without tokens
    Nest nest[2];       // of kv, with tokens
};
int check_move(const char* fn, const ii_cache& c, const ii_tokens& f, bool write, TokenRows* r);

// Groups of `size` that hold n things; in 64 bits, as n + size - 1 need not fit n's type.
constexpr int64_t groups(int64_t n, int64_t size) { return (n + size - 1) / size; }

inline bool half_type(int32_t dtype) { return dtype == II_BF16 || dtype == II_F16; }

// Scratch of split work: counters first, each zero between calls, then the
// partial results.
constexpr uint64_t kWorkCounters = 16384;
constexpr uint64_t kWorkHead = kWorkCounters * 4;
// *r: what a call may write of it, to be kept apart from its other operands.
int check_work(const char* fn, const void* work, uint64_t bytes, Rows* r);

int launched(const char* fn);

}  // namespace ii
