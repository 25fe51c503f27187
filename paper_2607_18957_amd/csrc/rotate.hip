// ii_rotate and ii_cache_append: heads turned by their token's position, keys
// on their way into a paged cache.
//
// A wave takes a token, or a part of its heads. It forms the sines of the
// token's rot / 2 angles once, a lane each, and leaves them in LDS; then heads
// pass through it, each in dim / 8 lanes of 8 elements, which find the other
// halves of their pairs in LDS or beside them.
//
// Angles and sines are held in 64 bits: the angle of a far position would lose its
// last digits. Products of 32 bits are enough for results of 16, but a key that is
// quantised would be rounded to the wrong code where it lies next to the middle of
// two, so its products are held in 64 bits too, which run at the rate of 32 here;
// the way from there is one rounding, through a float whose last bit remembers what
// was cut off (round_odd).
//
// Bound by memory: 8191 tokens of 32 heads of 128, turned in half of each, 29.7 us,
// 4.5 TB/s; 16384 tokens appended to an 8-bit cache, 32 query and 8 key heads,
// 92 us, 4.0 TB/s. The loads of four rounds are on their way, 4 KB a wave: with one
// these took 36 and 117 us, with eight, which leave fewer waves, 29 and 103.
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
constexpr int kAhead = 4;  // rounds whose loads are on their way

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

// Bytes of LDS of a wave.
__host__ __device__ constexpr int lds_of(int rot, bool quant) {
    return 1024 + (rot / 2 + rot / 2 % 2) * 8 + (quant ? rot * 8 : 0);
}

// Rounds of as many heads as a wave holds: those of q, then with kAppend those of
// keys and of values, which go to the cache.
template <class T, bool kAppend, bool kQuant>
__global__ __launch_bounds__(kWaves * 64) void rotate_heads(Rotate p, Heads q, Heads k, Heads v,
                                                            CacheAt c) {
    using x8 = typename Vec<T>::x8;
    using f32x2 = __attribute__((ext_vector_type(2))) float;
    using f64x2 = __attribute__((ext_vector_type(2))) double;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int pairs = p.rot / 2;
    // sines in 64 bits if keys are quantised, in 32, and a wave's heads
    char* const at = lds + wave * lds_of(p.rot, kQuant);
    T* room = reinterpret_cast<T*>(at);
    f32x2* turns = reinterpret_cast<f32x2*>(at + 1024);
    f64x2* turns64 = reinterpret_cast<f64x2*>(at + 1024 + pairs * 8 + pairs % 2 * 8);

    const int mine = lane / p.lanes, first = lane % p.lanes * 8;  // head, its first element here
    const bool used = mine < p.at_once;
    const bool halves = p.layout == II_ROTARY_HALF;
    // where the others of this lane's pairs are, and its own sines
    const T* head = room + (used ? mine * p.lanes * 8 : 0);
    const bool words = pairs % 8 == 0;
    const int across = first >= p.rot ? first : first < pairs ? first + pairs : first - pairs;
    const auto sines = [&](auto* from, int j) {
        const int e = first + j;
        auto t = from[halves ? (e < pairs ? e : e - pairs) : e / 2];
        if (halves ? e < pairs : j % 2 == 0) t[1] = -t[1];
        return t;
    };
    const auto others = [&](u32x4 raw) {
        const x8 x = __builtin_bit_cast(x8, raw);
        x8 o;
        if (halves) {
            *reinterpret_cast<u32x4*>(room + lane * 8) = raw;
            wave_meets();
            if (words) {
                o = *reinterpret_cast<const x8*>(head + across);
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
        return o;
    };

    const int q_rounds = (q.heads + p.at_once - 1) / p.at_once;
    const int kv_rounds = kAppend ? (k.heads + p.at_once - 1) / p.at_once : 0;
    const int rounds = q_rounds + 2 * kv_rounds;
    const int64_t units = p.tokens * p.splits;
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units;
         unit += (int64_t)gridDim.x * kWaves) {
        const int64_t token = unit / p.splits;
        int round = (int)(unit - token * p.splits);
        int64_t slot = -1;
        if (kAppend) slot = p.slots[token];
        const int64_t page = slot >> c.page_bits;
        const bool kept = kAppend && slot >= 0 && page < c.pages;
        const int64_t row = slot & (((int64_t)1 << c.page_bits) - 1);

        const auto load = [&](int r) {
            u32x4 x = {};
            const uint8_t* from;
            int h = r * p.at_once + mine;
            if (!kAppend || r < q_rounds) {
                if (r >= rounds || !used || h >= q.heads) return x;
                from = q.x + token * q.x_token + h * q.x_head;
            } else {
                h -= q_rounds * p.at_once;
                const bool of_k = r < q_rounds + kv_rounds;
                if (!of_k) h -= kv_rounds * p.at_once;
                if (r >= rounds || !used || !kept || h >= k.heads) return x;
                if (of_k)
                    from = k.x + token * k.x_token + h * k.x_head;
                else
                    from = v.x + token * v.x_token + h * v.x_head;
            }
            return *reinterpret_cast<const u32x4*>(from + first * 2);
        };
        u32x4 ahead[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ahead[i] = load(round + i * p.splits);

        const double position = (double)p.positions[token];
        for (int i = lane; i < pairs; i += 64) {
            double co, si;
            turn_of(position, p.freqs[i], &co, &si);
            co *= p.magnitude;
            si *= p.magnitude;
            turns[i] = f32x2{(float)co, (float)si};
            if (kQuant) turns64[i] = f64x2{co, si};
        }
        wave_meets();
        float co[8], si[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            co[j] = 1;
            si[j] = 0;
            if (first + j < p.rot) {
                const f32x2 t = sines(turns, j);
                co[j] = t[0];
                si[j] = t[1];
            }
        }

        const auto pass = [&](u32x4 raw) {
            const x8 x = __builtin_bit_cast(x8, raw);
            const bool of_q = round < q_rounds, of_k = round < q_rounds + kv_rounds;
            x8 y = x;
            if (of_q || (of_k && !kQuant)) {
                const x8 o = others(raw);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float t = fmaf((float)x[j], co[j], (float)o[j] * si[j]);
                    y[j] = first + j < p.rot ? (T)t : x[j];
                }
            }
            if (!kAppend || of_q) {
                const int h = round * p.at_once + mine;
                if (used && h < q.heads)
                    *reinterpret_cast<x8*>(q.out + token * q.out_token + h * q.out_head + first * 2) = y;
                return;
            }
            const int h = (round - q_rounds - (of_k ? 0 : kv_rounds)) * p.at_once + mine;
            const bool put = used && kept && h < k.heads;
            uint8_t* to = (of_k ? c.at[0] : c.at[1]) + page * c.page_stride + h * c.head_stride +
                          row * c.token_stride;
            if constexpr (kQuant) {
                float z[8];
                if (of_k) {
                    const x8 o = others(raw);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        z[j] = (float)x[j];
                        if (first + j < p.rot) {
                            const f64x2 t = sines(turns64, j);
                            z[j] = round_odd(fma((double)z[j], t[0], (double)(float)o[j] * t[1]));
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = (float)x[j];
                }
                // four neighbouring lanes hold a block, of one head
                uint32_t exponent;
                const u32x2 code = quantise<T>(z, &exponent);
                if (put) {
                    *reinterpret_cast<u32x2*>(to + first) = code;
                    if (first % 32 == 0)
                        (of_k ? c.scale[0] : c.scale[1])[page * c.scale_page_stride +
                                                         h * c.scale_head_stride +
                                                         row * c.scale_token_stride + first / 32] =
                            (uint8_t)exponent;
                }
            } else if (put) {
                *reinterpret_cast<x8*>(to + first * 2) = y;
            }
        };
        while (round < rounds) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i, round += p.splits) {
                if (round >= rounds) break;
                const u32x4 raw = ahead[i];
                ahead[i] = load(round + kAhead * p.splits);
                pass(raw);
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
dim3 shape(Rotate* p, const ii_rotary& r, int64_t tokens, int64_t q_heads, int64_t kv_heads, int dim) {
    p->positions = r.positions;
    p->freqs = r.freqs;
    p->magnitude = r.magnitude;
    p->tokens = tokens;
    p->rot = r.rot_dim;
    p->layout = r.layout;
    p->lanes = dim / 8;
    p->at_once = 64 / p->lanes;
    // enough waves to fill the card, though each forms its token's sines again
    const int64_t rounds = groups(q_heads, p->at_once) + 2 * groups(kv_heads, p->at_once);
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

// x and out of heads to be turned; out may be x itself. *nest: out's, with tokens.
int check_turn(const char* fn, const ii_turn& t, Rows* x, Rows* out, Nest* nest) {
    if (!half_type(t.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, t.dtype);
    if (t.heads < 1 || t.heads > 1 << 28) return fail(II_EINVAL, "%s: %d heads", fn, t.heads);
    if (t.dim < 8 || t.dim > 512 || t.dim % 8)
        return fail(II_EINVAL, "%s: heads of %d elements", fn, t.dim);
    if (t.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, t.reserved);
    if (t.tokens < 0 || t.tokens > (int64_t)1 << 40)
        return fail(II_EINVAL, "%s: %lld tokens", fn, (long long)t.tokens);
    Nest from;
    int rc = check_heads(fn, "x", t.x, t.tokens, t.heads, t.dim, t.x_token_stride, t.x_head_stride, 2,
                         false, x, &from);
    if (!rc)
        rc = check_heads(fn, "out", t.out, t.tokens, t.heads, t.dim, t.out_token_stride,
                         t.out_head_stride, 2, true, out, nest);
    if (rc) return rc;
    // a head is read by the lanes of a wave before any of them writes it
    if (t.x == t.out && (t.tokens <= 1 || t.x_token_stride == t.out_token_stride) &&
        (t.heads <= 1 || t.x_head_stride == t.out_head_stride))
        return II_OK;
    return check_heads_apart(fn, "x", *out, *nest, *x, from);
}

template <class T>
void turn(const ii_turn& t, const ii_rotary& r, hipStream_t stream) {
    Rotate p = {};
    const dim3 grid = shape(&p, r, t.tokens, t.heads, 0, t.dim);
    const Heads h = heads_of(t);
    rotate_heads<T, false, false><<<grid, kWaves * 64, kWaves * lds_of(p.rot, false), stream>>>(
        p, h, Heads{}, Heads{}, CacheAt{});
}

int rotate(const ii_turn* t, const ii_rotary* r, hipStream_t stream) {
    const char* fn = "ii_rotate";
    if (!t || !r) return fail(II_EINVAL, "%s: an argument is NULL", fn);
    {
        const Checks checks;
        Rows x, out, held[2];
        Nest nest;
        int rc = check_turn(fn, *t, &x, &out, &nest);
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
    const dim3 grid = shape(&p, r, f.tokens, h.heads, c.heads, c.dim);
    p.slots = f.slots;
    const Heads k = {static_cast<const uint8_t*>(f.k), nullptr, f.k_token_stride * 2,
                     f.k_head_stride * 2, 0, 0, c.heads};
    const Heads v = {static_cast<const uint8_t*>(f.v), nullptr, f.v_token_stride * 2,
                     f.v_head_stride * 2, 0, 0, c.heads};
    const bool quant = c.dtype == II_FP8_E4M3;
    const uint32_t lds = kWaves * lds_of(p.rot, quant);
    if (quant)
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
        Nest nest;
        int rc = check_move(fn, *c, *f, true, &t);
        if (rc || (rc = check_rotary(fn, *r, f->tokens, c->dim, held))) return rc;
        if (c->heads > 1 << 28) return fail(II_EINVAL, "%s: cache of %d heads", fn, c->heads);
        if (q) {
            if (q->dtype != f->dtype || q->tokens != f->tokens || q->dim != c->dim)
                return fail(II_EINVAL, "%s: q of type %d, %lld tokens, %d elements; keys of type %d, "
                            "%lld, %d", fn, q->dtype, (long long)q->tokens, q->dim, f->dtype,
                            (long long)f->tokens, c->dim);
            if ((rc = check_turn(fn, *q, &x, &out, &nest))) return rc;
        }
        const struct {
            const char* what;
            const Rows& r;
            const Nest* nest;
        } read[] = {{"k", t.kv[0], &t.nest[0]}, {"v", t.kv[1], &t.nest[1]}, {"slots", t.slots, nullptr},
                    {"positions", held[0], nullptr}, {"freqs", held[1], nullptr}, {"q", x, nullptr}};
        for (const auto& in : read) {
            for (const Rows& w : t.cache.all)
                if ((rc = check_apart(fn, in.what, w, in.r))) return rc;
            if (&in.r == &x) continue;
            // q may lie between the keys and values of its heads
            rc = in.nest ? check_heads_apart(fn, in.what, out, nest, in.r, *in.nest)
                         : check_apart(fn, in.what, out, in.r);
            if (rc) return rc;
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
