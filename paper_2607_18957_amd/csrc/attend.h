// What the kernels of ii_attend share.
#pragma once

#include <cmath>
#include <type_traits>

#include "ops.h"
#include "ops_device.h"

namespace ii {

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

__device__ inline bf16x2 unpack(uint32_t codes, float scale, bf16x2, bool high) {
    return high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
}
__device__ inline f16x2 unpack(uint32_t codes, float scale, f16x2, bool high) {
    return high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, true)
                : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, false);
}
// Four keys of 16 positions each for 16 lanes: lane i addresses 4 positions of
// key i / 4 and gets position i of the four keys.
template <class T>
__device__ inline typename Vec<T>::x4 read_transposed(const T* at) {
    using Lds = __attribute__((address_space(3))) s16x4;
    return __builtin_bit_cast(typename Vec<T>::x4,
                              __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(void*)at));
}

template <class T>
__device__ inline bool not_finite(typename Vec<T>::x8 v) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) bad |= !(fabsf((float)v[i]) <= 3.4e38f);
    return bad;
}

// What is added to the exponents of weights, in bits, sums and totals alike, so
// that the largest weight is 2^15 where the running maximum may be `grow` bits
// behind: f16 has 11 bits of a weight down to 2^-14 alone and loses it below
// 2^-25, and 131072 keys 2^-26 of the largest make 1/512 of a result. bf16 has
// float's range.
//
// The product with the values takes weights of 16 bits, rounded once each, which
// brings the error against 64 bits from 1.65e-3 (the result's own rounding to
// bf16) to 2.1e-3. A second product with what the rounding left out brings it
// back, but takes a prompt of 8000 tokens 786 us against 618, 48 sequences of up
// to 8192 keys 99 against 94, 128 of up to 1500 58 against 52.
template <class T>
constexpr float lift(float grow) {
    return std::is_same_v<T, _Float16> ? 15.0f - grow : 0.0f;
}

// Where a sequence's queries and keys are.
struct Seq {
    int64_t first, len;  // its first row; keys
    int32_t n;           // queries
};
__device__ inline Seq sequence(const Attend& p, int b) {
    Seq s;
    int64_t end = b + 1;
    s.first = b;
    if (p.q_start) {
        s.first = p.q_start[b];
        end = p.q_start[b + 1];
    }
    s.len = p.lengths[b];
    // queries outside the rows are left out; the last row stays the last key's
    if (end < s.first || end > p.rows || s.first < 0) end = s.first = 0;
    s.n = (int32_t)(end - s.first);
    return s;
}

// The keys that the queries t_first .. t_last of a sequence see: all of [lo,
// hi) by some query, those of [lo_max, hi_min) by every one.
struct Reach {
    int64_t lo, hi, lo_max, hi_min;
};
__device__ inline Reach reach_of(const Attend& p, const Seq& seq, int t_first, int t_last) {
    const int64_t pos0 = seq.len - seq.n + t_first, pos1 = seq.len - seq.n + t_last;
    Reach r;
    r.lo = p.window ? max((int64_t)0, pos0 - p.window + 1) : 0;
    r.hi = max((int64_t)0, min(pos1 + 1, p.capacity));
    r.lo_max = p.window ? max((int64_t)0, pos1 - p.window + 1) : 0;
    r.hi_min = max((int64_t)0, min(pos0 + 1, p.capacity));
    return r;
}

// Parts of a reach, of part_keys keys or more, at most parts_most.
__device__ inline int parts_of(const Reach& r, int parts_most, int part_keys) {
    const int64_t keys = max((int64_t)0, r.hi - r.lo);
    return (int)max((int64_t)1, min((int64_t)parts_most, (keys + part_keys - 1) / part_keys));
}

// Scratch of results that are split over keys.
struct AttendWork {
    uint32_t* counters = nullptr;
    float* partial = nullptr;
    uint64_t floats = 0;
};

// Attention of the sequences with more than least_rows (query, head of a
// group) rows (attend_many.hip); max_q queries and `reach` keys at most are
// expected of a sequence.
void attend_many(const Attend& p, int dtype, bool quant, int dim, int64_t max_q, int64_t reach,
                 int least_rows, const AttendWork& work, hipStream_t stream);

}  // namespace ii
