// ii_cache_write and ii_cache_read: a paged key/value cache, quantised as it
// is written.
//
// A block of 32 elements x gets the scale 2^e, e the least with max |x| <=
// 448 * 2^e over its finite elements, and codes e4m3(x * 2^-e). Both the
// scale and the product are exact, so the codes are the definition's, bit for
// bit, at any precision.
//
// Bound by memory: each lane moves 16 bytes of activations (8 elements) of
// keys or of values, four lanes hold a block and agree on its scale by two
// exchanges, so reads and writes of a head's row are contiguous. 16384 tokens
// of 8 heads of 128: written in 25 us, 4.0 TB/s (the vector units are busy in
// three quarters of the cycles), read in 20, 5.1 TB/s; kept as they are, 134 MB
// moved by each, 42 us together (with inputs that the last pass left in caches;
// in 8 bits 46).
#include "cache_device.h"
#include "ops.h"

namespace ii {
namespace {

struct Tokens {
    uint8_t* at[2];
    int64_t token_stride[2], head_stride[2];  // bytes
    const int64_t* slots;
    int64_t tokens;
    int32_t heads, dim;
};

constexpr int kThreads = 256;

template <class T, bool kQuant, bool kWrite>
__global__ __launch_bounds__(kThreads) void cache_move(CacheAt c, Tokens f) {
    using x8 = typename Vec<T>::x8;
    const int per_head = f.dim / 8;
    const int64_t per_token = (int64_t)per_head * f.heads;
    const int64_t unit = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int kv = blockIdx.y;
    const int64_t token = unit / per_token;
    const bool live = token < f.tokens;
    const int in = (int)(unit - token * per_token), head = in / per_head, part = in % per_head;
    // every lane takes part in the exchanges below; blocks are four
    // neighbouring lanes of one token
    const int64_t slot = live ? f.slots[token] : -1;
    const int64_t page = slot >> c.page_bits;
    const bool kept = slot >= 0 && page < c.pages;
    const int64_t row = slot & (((int64_t)1 << c.page_bits) - 1);
    const int64_t at = page * c.page_stride + head * c.head_stride + row * c.token_stride;
    const int64_t sat = page * c.scale_page_stride + head * c.scale_head_stride +
                        row * c.scale_token_stride + part / 4;
    x8* user = reinterpret_cast<x8*>(f.at[kv] + token * f.token_stride[kv] +
                                     head * f.head_stride[kv] + part * 16);
    if (!kQuant) {
        u32x4* mine = reinterpret_cast<u32x4*>(c.at[kv] + at + part * 16);
        u32x4* theirs = reinterpret_cast<u32x4*>(user);
        if (kWrite) {
            if (kept) *mine = *theirs;
        } else if (live) {
            *theirs = kept ? *mine : u32x4{};
        }
        return;
    }
    if (kWrite) {
        x8 v = {};
        if (kept) v = *user;
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
        uint32_t e;
        const u32x2 code = quantise<T>(x, &e);
        if (kept) {
            *reinterpret_cast<u32x2*>(c.at[kv] + at + part * 8) = code;
            if (part % 4 == 0) c.scale[kv][sat] = (uint8_t)e;
        }
    } else if (live) {
        x8 v = {};
        if (kept) {
            const u32x2 code = *reinterpret_cast<const u32x2*>(c.at[kv] + at + part * 8);
            // 2^(e - 127); an exponent of 0 (2^-127) is below float's normal range
            const uint32_t e = c.scale[kv][sat];
            const float scale = __builtin_bit_cast(float, e ? e << 23 : 0x400000u);
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(code[j / 4], false);
                const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(code[j / 4], true);
                v[j] = (T)(lo[0] * scale);
                v[j + 1] = (T)(lo[1] * scale);
                v[j + 2] = (T)(hi[0] * scale);
                v[j + 3] = (T)(hi[1] * scale);
            }
        }
        *user = v;
    }
}

template <class T>
void launch(const CacheAt& c, const Tokens& f, bool quant, bool write, hipStream_t stream) {
    // a dispatch counts its work-items in 32 bits
    const int64_t per_token = (int64_t)f.heads * (f.dim / 8);
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 31) / per_token);
    for (int64_t t0 = 0; t0 < f.tokens; t0 += most) {
        Tokens part = f;
        part.tokens = std::min(most, f.tokens - t0);
        part.slots += t0;
        for (int i = 0; i < 2; ++i) part.at[i] += t0 * f.token_stride[i];
        const dim3 grid((uint32_t)((part.tokens * per_token + kThreads - 1) / kThreads), 2);
        if (quant && write)
            cache_move<T, true, true><<<grid, kThreads, 0, stream>>>(c, part);
        else if (quant)
            cache_move<T, true, false><<<grid, kThreads, 0, stream>>>(c, part);
        else if (write)
            cache_move<T, false, true><<<grid, kThreads, 0, stream>>>(c, part);
        else
            cache_move<T, false, false><<<grid, kThreads, 0, stream>>>(c, part);
    }
}

int move(const char* fn, const ii_cache* ca, const ii_tokens* tk, bool write, hipStream_t stream) {
    if (!ca || !tk) return fail(II_EINVAL, "%s: an argument is NULL", fn);
    const ii_cache& c = *ca;
    const ii_tokens& f = *tk;
    {
        const Checks checks;
        TokenRows r;
        if (const int rc = check_move(fn, c, f, write, &r)) return rc;
    }
    if (!f.tokens) return II_OK;
    const CacheAt d = cache_at(c);
    Tokens t;
    for (int i = 0; i < 2; ++i) {
        t.at[i] = static_cast<uint8_t*>(i ? f.v : f.k);
        t.token_stride[i] = (i ? f.v_token_stride : f.k_token_stride) * 2;
        t.head_stride[i] = (i ? f.v_head_stride : f.k_head_stride) * 2;
    }
    t.slots = f.slots;
    t.tokens = f.tokens;
    t.heads = c.heads;
    t.dim = c.dim;
    const bool quant = c.dtype == II_FP8_E4M3;
    if (f.dtype == II_BF16)
        launch<__bf16>(d, t, quant, write, stream);
    else
        launch<_Float16>(d, t, quant, write, stream);
    return launched(fn);
}

}  // namespace
}  // namespace ii

extern "C" int ii_cache_write(const ii_cache* cache, const ii_tokens* from, hipStream_t stream) {
    return ii::move("ii_cache_write", cache, from, true, stream);
}

extern "C" int ii_cache_read(const ii_cache* cache, const ii_tokens* to, hipStream_t stream) {
    return ii::move("ii_cache_read", cache, to, false, stream);
}
