// How a paged cache keeps values in 8 bits, for the kernels that write it.
#pragma once

#include "ii_ops.h"
#include "ops_device.h"

namespace ii {

struct CacheAt {
    uint8_t* at[2];  // keys, values; bytes
    uint8_t* scale[2];
    int64_t page_stride, head_stride, token_stride;  // bytes
    int64_t scale_page_stride, scale_head_stride, scale_token_stride;
    int64_t pages;
    int32_t page_bits;
};

inline CacheAt cache_at(const ii_cache& c) {
    const int size = c.dtype == II_FP8_E4M3 ? 1 : 2;
    CacheAt d;
    d.at[0] = static_cast<uint8_t*>(c.k);
    d.at[1] = static_cast<uint8_t*>(c.v);
    d.scale[0] = c.k_scale;
    d.scale[1] = c.v_scale;
    d.page_stride = c.page_stride * size;
    d.head_stride = c.head_stride * size;
    d.token_stride = c.token_stride * size;
    d.scale_page_stride = c.scale_page_stride;
    d.scale_head_stride = c.scale_head_stride;
    d.scale_token_stride = c.scale_token_stride;
    d.pages = c.pages;
    d.page_bits = __builtin_ctz(c.page);
    return d;
}

// Exponent (biased) of a block's scale from the bits of its largest finite
// magnitude: amax = 1.f * 2^E fits 448 = 1.75 * 2^8 at 2^(E - 8), or needs
// one more if f > 0.75.
__device__ inline uint32_t scale_exponent(uint32_t amax) {
    const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffff) > 0x600000);
    return e < 1 ? 1 : e;  // at most 247
}

// Codes of this lane's eight elements of a block of 32, which four neighbouring
// lanes hold and agree about; *exponent receives the scale's.
template <class T>
__device__ inline u32x2 quantise(const float (&x)[8], uint32_t* exponent) {
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = __builtin_bit_cast(uint32_t, x[j]) & 0x7fffffff;
        if (b < 0x7f800000 && b > amax) amax = b;
    }
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
    const uint32_t e = scale_exponent(amax);
    const float inverse = __builtin_bit_cast(float, (254 - e) << 23);
    // 2^8 times a code above 240 is past the largest f16
    const float most = __is_same(T, _Float16) && e == 127 + 8 ? 240.0f : 448.0f;
    uint32_t code[2] = {};
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        float y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t b = __builtin_bit_cast(uint32_t, x[j + i]) & 0x7fffffff;
            y[i] = b < 0x7f800000 ? fminf(fmaxf(x[j + i] * inverse, -most), most)
                                  : __builtin_nanf("");
        }
        int& w = reinterpret_cast<int&>(code[j / 4]);
        w = j % 4 ? __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, true)
                  : __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, false);
    }
    *exponent = e;
    return u32x2{code[0], code[1]};
}

}  // namespace ii
