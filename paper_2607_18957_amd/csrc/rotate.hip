// ii_rotate and ii_cache_append: heads turned by their token's position, keys
// on their way into a paged cache.
//
// A wave takes a token, or a part of its heads. It forms the sines of the
// token's rot / 2 angles once, a lane each, and leaves them in LDS; then heads
// pass through it, each in dim / 8 lanes of 8 elements, which find the other
// halves of their pairs in LDS or beside them.
//
// Angles and products are held in 64 bits, which run at the rate of 32 here: the
// angle of a far position would lose its last digits, and a key would be rounded
// to the wrong 8-bit code where it lies next to the middle of two. The way from
// 64 bits to a result is one rounding: through a float whose last bit remembers
// what was cut off (round_odd).
//
// Bound by memory.
#include <algorithm>
#include <cmath>

#include "cache_device.h"
#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

struct Heads {
    const uint8_t* x;
    uint8_t* out;
    int64_t x_token, x_head, out_token, out_head;  // bytes
    int32_t heads;
};

struct Rotate {
    const int64_t *positions, *slots;
    const double* freqs;
    double magnitude;
    int64_t tokens;
    int32_t rot, layout, lanes, at_once, splits;  // lanes of a head, heads a wave takes at once
};

constexpr int kWaves = 4;

// cos and sin of position * freq: the product in two doubles, whole turns taken
// off it with 2 pi in two doubles.
__device__ inline void turn_of(double position, double freq, double* c, double* s) {
    constexpr double kTurn = 6.283185307179586477, kRest = 2.4492935982947064e-16;
    constexpr double kTurns = 0.15915494309189533577, kHalfTurns = 0.31830988618379067154;
    const double p = position * freq, low = fma(position, freq, -p);
    const double n = rint(p * kTurns);
    const double r = fma(-n, kRest, fma(-n, kTurn, p)) + low;
    sincospi(r * kHalfTurns, s, c);
}

// y as a float that rounds on to fewer bits as y itself does: cut off, with the
// last bit set if anything was.
__device__ inline float round_odd(double y) {
    const float f = (float)y;
    const uint32_t b = __builtin_bit_cast(uint32_t, f);
    const double back = f;
    const bool inexact = back != y && (b & 0x7fffffff) < 0x7f800000;
    const uint32_t step = fabs(y) > fabs(back) ? 1 : ~0u;
    return __builtin_bit_cast(float, inexact && !(b & 1) ? b + step : b);
}

// LDS written by this wave is read by it after this.
__device__ inline void wave_meets() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Heads 0 .. q.heads - 1 are q's; with kAppend those of keys and of values
// follow, which go to the cache.
template <class T, bool kAppend, bool kQuant>
__global__ __launch_bounds__(kWaves * 64) void rotate_heads(Rotate p, Heads q, Heads k, Heads v,
                                                            CacheAt c) {
    using x8 = typename Vec<T>::x8;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int pairs = p.rot / 2;
    using f64x2 = __attribute__((ext_vector_type(2))) double;
    f64x2* turns = reinterpret_cast<f64x2*>(lds + wave * (pairs * 16 + 1024));
    T* room = reinterpret_cast<T*>(turns + pairs);

    const int mine = lane / p.lanes, first = lane % p.lanes * 8;  // head, its first element here
    const bool used = mine < p.at_once;
    const bool turned = first < p.rot;
    const bool halves = p.layout == II_ROTARY_HALF;
    const int total = q.heads + (kAppend ? 2 * k.heads : 0);
    const int step = p.at_once * p.splits;
    const int64_t units = p.tokens * p.splits;
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units;
         unit += (int64_t)gridDim.x * kWaves) {
        const int64_t token = unit / p.splits;
        int base = (int)(unit - token * p.splits) * p.at_once;
        int64_t slot = -1;
        if (kAppend) slot = p.slots[token];
        const int64_t page = slot >> c.page_bits;
        const bool kept = kAppend && slot >= 0 && page < c.pages;
        const int64_t row = slot & (((int64_t)1 << c.page_bits) - 1);

        const auto load = [&](int h) {
            u32x4 x = {};
            if (!used || h >= total) return x;
            const uint8_t* from;
            if (!kAppend || h < q.heads)
                from = q.x + token * q.x_token + h * q.x_head;
            else if (!kept)
                return x;
            else if (h < q.heads + k.heads)
                from = k.x + token * k.x_token + (h - q.heads) * k.x_head;
            else
                from = v.x + token * v.x_token + (h - q.heads - k.heads) * v.x_head;
            return *reinterpret_cast<const u32x4*>(from + first * 2);
        };
        u32x4 next = load(base + mine);

        const double position = (double)p.positions[token];
        for (int i = lane; i < pairs; i += 64) {
            double co, si;
            turn_of(position, p.freqs[i], &co, &si);
            turns[i] = f64x2{co * p.magnitude, si * p.magnitude};
        }
        wave_meets();
        double co[8], si[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = first + j;
            co[j] = 1;
            si[j] = 0;
            if (e < p.rot) {
                const f64x2 t = turns[halves ? (e < pairs ? e : e - pairs) : e / 2];
                co[j] = t[0];
                si[j] = (halves ? e < pairs : j % 2 == 0) ? -t[1] : t[1];
            }
        }

        for (; base < total; base += step) {
            const int h = base + mine;
            const u32x4 raw = next;
            next = load(h + step);
            const x8 x = __builtin_bit_cast(x8, raw);
            // the others of the pairs
            x8 o;
            if (halves) {
                *reinterpret_cast<u32x4*>(room + lane * 8) = raw;
                wave_meets();
                const T* head = room + (used ? mine * p.lanes * 8 : 0);
                if (pairs % 8 == 0) {
                    const int e = first < pairs ? first + pairs : first - pairs;
                    o = *reinterpret_cast<const x8*>(head + (turned ? e : first));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = first + j;
                        o[j] = head[e >= p.rot ? e : e < pairs ? e + pairs : e - pairs];
                    }
                }
                wave_meets();  // read before the next head's are written
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = x[j ^ 1];
            }
            const bool value = kAppend && h >= q.heads + k.heads;
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double t = fma((double)(float)x[j], co[j], (double)(float)o[j] * si[j]);
                y[j] = value || first + j >= p.rot ? (float)x[j] : round_odd(t);
            }
            if (!kAppend || h < q.heads) {
                if (used && h < total) {
                    x8 out;
#pragma unroll
                    for (int j = 0; j < 8; ++j) out[j] = (T)y[j];
                    *reinterpret_cast<x8*>(q.out + token * q.out_token + h * q.out_head + first * 2) = out;
                }
            }
            if constexpr (kAppend) {
                // four neighbouring lanes hold a block, of one head
                uint32_t exponent = 0;
                u32x2 code = {};
                if (kQuant) code = quantise<T>(y, &exponent);
                if (used && kept && h >= q.heads && h < total) {
                    const int kh = value ? h - q.heads - k.heads : h - q.heads;
                    const int64_t at = page * c.page_stride + kh * c.head_stride + row * c.token_stride;
                    uint8_t* to = (value ? c.at[1] : c.at[0]) + at;
                    if (kQuant) {
                        *reinterpret_cast<u32x2*>(to + first) = code;
                        if (first % 32 == 0)
                            (value ? c.scale[1] : c.scale[0])[page * c.scale_page_stride +
                                                              kh * c.scale_head_stride +
                                                              row * c.scale_token_stride + first / 32] =
                                (uint8_t)exponent;
                    } else {
                        x8 out;
#pragma unroll
                        for (int j = 0; j < 8; ++j) out[j] = value ? x[j] : (T)y[j];
                        *reinterpret_cast<x8*>(to + first * 2) = out;
                    }
                }
            }
        }
        wave_meets();  // sines read before the next token's are written
    }
}

Heads heads_of(const ii_turn& t) {
    Heads h;
    h.x = static_cast<const uint8_t*>(t.x);
    h.out = static_cast<uint8_t*>(t.out);
    h.x_token = t.x_token_stride * 2;
    h.x_head = t.x_head_stride * 2;
    h.out_token = t.out_token_stride * 2;
    h.out_head = t.out_head_stride * 2;
    h.heads = t.heads;
    return h;
}

// How `heads` heads of each token are given to waves.
dim3 shape(Rotate* p, const ii_rotary& r, int64_t tokens, int64_t heads, int dim) {
    p->positions = r.positions;
    p->freqs = r.freqs;
    p->magnitude = r.magnitude;
    p->tokens = tokens;
    p->rot = r.rot_dim;
    p->layout = r.layout;
    p->lanes = dim / 8;
    p->at_once = 64 / p->lanes;
    // enough waves to fill the card, though each forms its token's sines again
    const int64_t rounds = groups(heads, p->at_once);
    p->splits = (int32_t)std::max<int64_t>(1, std::min(rounds, 4096 / std::max<int64_t>(tokens, 1)));
    return dim3((uint32_t)std::min<int64_t>(groups(tokens * p->splits, kWaves), 1 << 20));
}

int check_rotary(const char* fn, const ii_rotary& r, int64_t tokens, int dim, Rows (&held)[2]) {
    if (r.rot_dim < 0 || r.rot_dim > dim || r.rot_dim % 2)
        return fail(II_EINVAL, "%s: rot_dim %d of heads of %d elements", fn, r.rot_dim, dim);
    if (r.layout != II_ROTARY_HALF && r.layout != II_ROTARY_INTERLEAVED)
        return fail(II_EINVAL, "%s: layout %d", fn, r.layout);
    if (!std::isfinite(r.magnitude)) return fail(II_EINVAL, "%s: magnitude %g", fn, r.magnitude);
    if (r.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, r.reserved);
    if (!tokens) return II_OK;
    int rc = check_rows(fn, "positions", r.positions, 1, (uint64_t)tokens * 8, 0, 8, &held[0]);
    if (!rc) rc = check_rows(fn, "freqs", r.freqs, 1, (uint64_t)r.rot_dim * 4, 0, 8, &held[1]);
    return rc;
}

// x and out of heads to be turned; out may be x itself.
int check_turn(const char* fn, const ii_turn& t, Rows* x, Rows* out) {
    if (!half_type(t.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, t.dtype);
    if (t.heads < 1 || t.heads > 1 << 28) return fail(II_EINVAL, "%s: %d heads", fn, t.heads);
    if (t.dim < 8 || t.dim > 512 || t.dim % 8)
        return fail(II_EINVAL, "%s: heads of %d elements", fn, t.dim);
    if (t.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, t.reserved);
    if (t.tokens < 0 || t.tokens > (int64_t)1 << 40)
        return fail(II_EINVAL, "%s: %lld tokens", fn, (long long)t.tokens);
    int rc = check_heads(fn, "x", t.x, t.tokens, t.heads, t.dim, t.x_token_stride, t.x_head_stride, 2,
                         false, x);
    if (!rc)
        rc = check_heads(fn, "out", t.out, t.tokens, t.heads, t.dim, t.out_token_stride,
                         t.out_head_stride, 2, true, out);
    if (rc) return rc;
    // a head is read by the lanes of a wave before any of them writes it
    if (t.x == t.out && (t.tokens <= 1 || t.x_token_stride == t.out_token_stride) &&
        (t.heads <= 1 || t.x_head_stride == t.out_head_stride))
        return II_OK;
    return check_apart(fn, "x", *out, *x);
}

template <class T>
void turn(const ii_turn& t, const ii_rotary& r, hipStream_t stream) {
    Rotate p = {};
    const dim3 grid = shape(&p, r, t.tokens, t.heads, t.dim);
    const Heads h = heads_of(t);
    rotate_heads<T, false, false><<<grid, kWaves * 64, kWaves * (p.rot * 8 + 1024), stream>>>(
        p, h, Heads{}, Heads{}, CacheAt{});
}

int rotate(const ii_turn* t, const ii_rotary* r, hipStream_t stream) {
    const char* fn = "ii_rotate";
    if (!t || !r) return fail(II_EINVAL, "%s: an argument is NULL", fn);
    {
        const Checks checks;
        Rows x, out, held[2];
        int rc = check_turn(fn, *t, &x, &out);
        if (rc || (rc = check_rotary(fn, *r, t->tokens, t->dim, held))) return rc;
        if ((rc = check_apart(fn, "positions", out, held[0])) ||
            (rc = check_apart(fn, "freqs", out, held[1])))
            return rc;
    }
    if (!t->tokens) return II_OK;
    if (t->dtype == II_BF16)
        turn<__bf16>(*t, *r, stream);
    else
        turn<_Float16>(*t, *r, stream);
    return launched(fn);
}

template <class T>
void put(const ii_cache& c, const ii_tokens& f, const ii_rotary& r, const ii_turn* q,
         hipStream_t stream) {
    Rotate p = {};
    const Heads h = q ? heads_of(*q) : Heads{};
    const dim3 grid = shape(&p, r, f.tokens, h.heads + 2 * (int64_t)c.heads, c.dim);
    p.slots = f.slots;
    const Heads k = {static_cast<const uint8_t*>(f.k), nullptr, f.k_token_stride * 2,
                     f.k_head_stride * 2, 0, 0, c.heads};
    const Heads v = {static_cast<const uint8_t*>(f.v), nullptr, f.v_token_stride * 2,
                     f.v_head_stride * 2, 0, 0, c.heads};
    const uint32_t lds = kWaves * (p.rot * 8 + 1024);
    if (c.dtype == II_FP8_E4M3)
        rotate_heads<T, true, true><<<grid, kWaves * 64, lds, stream>>>(p, h, k, v, cache_at(c));
    else
        rotate_heads<T, true, false><<<grid, kWaves * 64, lds, stream>>>(p, h, k, v, cache_at(c));
}

int append(const ii_cache* c, const ii_tokens* f, const ii_rotary* r, const ii_turn* q,
           hipStream_t stream) {
    const char* fn = "ii_cache_append";
    if (!c || !f || !r) return fail(II_EINVAL, "%s: an argument is NULL", fn);
    {
        const Checks checks;
        TokenRows t;
        Rows x, out, held[2];
        int rc = check_move(fn, *c, *f, true, &t);
        if (rc || (rc = check_rotary(fn, *r, f->tokens, c->dim, held))) return rc;
        if (c->heads > 1 << 28) return fail(II_EINVAL, "%s: cache of %d heads", fn, c->heads);
        if (q) {
            if (q->dtype != f->dtype || q->tokens != f->tokens || q->dim != c->dim)
                return fail(II_EINVAL, "%s: q of type %d, %lld tokens, %d elements; keys of type %d, "
                            "%lld, %d", fn, q->dtype, (long long)q->tokens, q->dim, f->dtype,
                            (long long)f->tokens, c->dim);
            if ((rc = check_turn(fn, *q, &x, &out))) return rc;
        }
        const struct {
            const char* what;
            const Rows& r;
        } read[] = {{"k", t.kv[0]}, {"v", t.kv[1]}, {"slots", t.slots}, {"positions", held[0]},
                    {"freqs", held[1]}, {"q", x}};
        for (const auto& in : read) {
            for (const Rows& w : t.cache.all)
                if ((rc = check_apart(fn, in.what, w, in.r))) return rc;
            if (&in.r != &x && (rc = check_apart(fn, in.what, out, in.r))) return rc;
        }
        for (const Rows& w : t.cache.all)
            if ((rc = check_apart(fn, "the cache", out, w))) return rc;
    }
    if (!f->tokens) return II_OK;
    if (f->dtype == II_BF16)
        put<__bf16>(*c, *f, *r, q, stream);
    else
        put<_Float16>(*c, *f, *r, q, stream);
    return launched(fn);
}

}  // namespace
}  // namespace ii

extern "C" int ii_rotate(const ii_turn* heads, const ii_rotary* rotary, hipStream_t stream) {
    return ii::rotate(heads, rotary, stream);
}

extern "C" int ii_cache_append(const ii_cache* cache, const ii_tokens* from, const ii_rotary* rotary,
                               const ii_turn* q, hipStream_t stream) {
    return ii::append(cache, from, rotary, q, stream);
}

extern "C" int ii_rotary_freqs(int32_t rot_dim, double base, double factor, double low, double high,
                               int64_t original, double* freqs) {
    const char* fn = "ii_rotary_freqs";
    if (rot_dim < 0 || rot_dim > 1 << 20 || rot_dim % 2)
        return ii::fail(II_EINVAL, "%s: rot_dim %d", fn, rot_dim);
    if (!(base > 0) || !(factor > 0) || !std::isfinite(base) || !std::isfinite(factor))
        return ii::fail(II_EINVAL, "%s: base %g, factor %g", fn, base, factor);
    if (original < 0 || (original && (!std::isfinite(low) || !std::isfinite(high) || !(high > low))))
        return ii::fail(II_EINVAL, "%s: original %lld, low %g, high %g", fn, (long long)original, low,
                        high);
    if (rot_dim && !freqs) return ii::fail(II_EINVAL, "%s: freqs is NULL", fn);
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        double keep = 0;
        if (original) {
            const double turns = (double)original * f / 6.283185307179586477;
            keep = std::min(std::max((turns - low) / (high - low), 0.0), 1.0);
        }
        freqs[i] = keep * f + (1 - keep) * f / factor;
    }
    return II_OK;
}
