// ii_logprobs: log-probabilities of given tokens, entropy and the likeliest
// tokens, in one pass over the logits.
//
// Every thread keeps the running maximum m of its logits, s = sum 2^u and t = sum
// 2^u u, u = (z - m) / ln 2, a term of which is never below -0.54 however far apart
// the logits are; then log sum_j e^z_j = m + log s, and the entropy is log s - t ln 2
// / s. Sums of a tile are added up in 64 bits: a vocabulary is a long sum, and what
// it loses is in every result. A logit is kept as a key of 64 bits, its order above
// and its token's complement below, so that no two are alike and the order of
// arrival does not show.
//
// The likeliest tokens: of the largest logits of a wave's 64 threads, in order, the
// top-th is a bound that `top` tokens reach, and so is the least of the waves'
// (top / 4)-th. What reaches the larger bound, little more than `top` tokens of a
// tile, goes into a list in LDS; later tiles add what is above the list's top-th,
// which few are. Where many logits are alike a bound of keys takes its place: the
// top-th of the 256 threads' largest, of which at most `top` threads hold tokens
// that reach it. A list is cut to `top` by counting, for each key, those above it,
// after a bound of the same kind has left few.
//
// Bound by memory: 2047 x 128256 in bf16 101 us, 5.2 TB/s, where a logit takes some
// ten vector instructions, of which the exponential counts for four; in the first
// milliseconds of load the card takes up to 130. With the 5 or 20 likeliest, 240 and
// 257 us, the vector units bound it. Few rows are bound by the steps from a load to
// the last part's joining: 48 x 128256 with the 20 likeliest 22 us, 1 x 8192 with 5
// of them 8.8.
#include <algorithm>
#include <cmath>

#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

constexpr int kThreads = 256;
// Logits of a tile a thread: with 16, 2047 x 128256 took 106 us, 1 x 8192 11.4.
constexpr int kEach = 32;
constexpr int kTile = kThreads * kEach;
constexpr int kList = 2560;       // keys a list holds
constexpr int kPruned = 256;      // and how many beyond 3 top are put up with
constexpr float kLog2e = 1.44269504088896340736f;

struct Logprobs {
    const void* logits;
    const int64_t* targets;
    float *logprob, *entropy, *top_logprobs;
    int64_t* top_ids;
    int64_t stride, rows;  // elements
    int64_t part;          // elements of one, which may pass those of a vocabulary
    int32_t vocab, top, parts;
    float scale;
    uint32_t* counters;
    float* partial;
    uint32_t room;  // floats of a part in partial
};

// Sums of 2^u, and of u times that, u = (x - m) to2, x a logit; to2 is scale / ln 2.
struct Sums {
    float m;
    double s, t;
};
__device__ inline Sums no_sums() { return Sums{-INFINITY, 0, 0}; }

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The same relative to m; m is not below a.m. Without a finite logit there is
// nothing to move.
__device__ inline void move_to(Sums& a, float m, float to2) {
    if (a.m != m) {
        if (a.m == -INFINITY) {
            a.t = 0;
        } else {
            const float u = (a.m - m) * to2;
            const double c = exp2_of(u);
            a.t = c * (a.t + a.s * fmaxf(u, -3e38f));
            a.s *= c;
        }
        a.m = m;
    }
}
__device__ inline void join(Sums& a, Sums b, float to2) {
    const float m = fmaxf(a.m, b.m);
    move_to(a, m, to2);
    move_to(b, m, to2);
    a.s += b.s;
    a.t += b.t;
}

// Those of the workgroup's threads: their maximum, then all relative to it, in the
// order of lanes and waves. Called by all threads.
__device__ inline Sums sum_of(Sums a, float to2, Sums (&waves)[kThreads / 64]) {
    float most = a.m;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    move_to(a, most, to2);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        a.s += __shfl_xor(a.s, d);
        a.t += __shfl_xor(a.t, d);
    }
    __syncthreads();
    if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = a;
    __syncthreads();
    a = waves[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) join(a, waves[w], to2);
    return a;
}

// The order of floats in whole numbers (-0 as +0; NaN as -infinity), above the
// complement of the token, so that of equal logits the lower token is larger.
// No key is 0.
__device__ inline uint32_t order_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline uint64_t key_of(float x, int token) {
    if (!(x == x)) x = -INFINITY;
    return (uint64_t)order_of(x) << 32 | (uint32_t)~token;
}
__device__ inline float float_of(uint32_t order) {
    return __builtin_bit_cast(float, order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ inline float logit_of(uint64_t key) { return float_of((uint32_t)(key >> 32)); }

struct List {
    uint64_t key[kList];
    uint64_t sorted[II_MAX_TOP];
    uint64_t best[kThreads], least;  // of a tile
    uint32_t count, added[3], more, again;
    float room[2][kThreads / 64];
};

// How many of the n keys are above mine. n is even, or key[n] is 0.
__device__ inline int above(const uint64_t* key, int n, uint64_t mine) {
    using u64x2 = __attribute__((ext_vector_type(2))) uint64_t;
    int c = 0;
#pragma unroll 4
    for (int i = 0; i < (n + 1) / 2; ++i) {
        const u64x2 k = reinterpret_cast<const u64x2*>(key)[i];
        c += (k[0] > mine) + (k[1] > mine);
    }
    return c;
}

// A bound that `top` of the threads' values `mine` reach: the largest of the
// waves' top-th ones, or the least of the waves' (top / 4)-th, whichever is
// larger. Called by all threads; `room` is free before and after.
__device__ inline float bound_of(float mine, int top, float (&room)[2][kThreads / 64]) {
    const int lane = threadIdx.x % 64;
    // the wave's values in falling order, by exchanges of two sorted halves
#pragma unroll
    for (int k = 2; k <= 64; k *= 2)
#pragma unroll
        for (int d = k / 2; d > 0; d /= 2) {
            const float other = __shfl_xor(mine, d);
            const bool larger = ((lane & k) == 0) == ((lane & d) == 0);
            mine = larger ? fmaxf(mine, other) : fminf(mine, other);
        }
    constexpr int kWaves = kThreads / 64;
    const float one = __shfl(mine, top - 1), all = __shfl(mine, (top + kWaves - 1) / kWaves - 1);
    __syncthreads();
    if (lane == 0) {
        room[0][threadIdx.x / 64] = one;
        room[1][threadIdx.x / 64] = all;
    }
    __syncthreads();
    float most = room[0][0], least = room[1][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        most = fmaxf(most, room[0][w]);
        least = fminf(least, room[1][w]);
    }
    return fmaxf(most, least);
}

// Cuts the list to its `top` largest keys, in order. Called by all threads with
// what was written before them in place; they may read the list after it. Keys
// of 0, which may be many, come last.
__device__ inline void prune(List& l, int top) {
    __syncthreads();
    int n = (int)l.count;
    if (n > 2 * II_MAX_TOP) {
        // only what reaches a bound of the threads' largest can be among them
        constexpr int kEach = kList / kThreads;
        uint64_t mine[kEach], best = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = i * kThreads + threadIdx.x;
            mine[i] = at < n ? l.key[at] : 0;
            best = max(best, mine[i]);
        }
        const uint32_t bound = order_of(bound_of(best ? logit_of(best) : -INFINITY, top, l.room));
        int hits = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) hits += mine[i] && (uint32_t)(mine[i] >> 32) >= bound;
        if (threadIdx.x == 0) l.again = 0;
        __syncthreads();
        uint32_t place = 0;
        if (hits) place = atomicAdd(&l.again, (uint32_t)hits);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (mine[i] && (uint32_t)(mine[i] >> 32) >= bound) l.key[place++] = mine[i];
        __syncthreads();
        n = (int)l.again;
    }
    if (threadIdx.x < II_MAX_TOP) l.sorted[threadIdx.x] = 0;
    if (threadIdx.x == 0 && n % 2) l.key[n] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t mine = l.key[i];
        const int c = above(l.key, n, mine);
        if (c < top) l.sorted[c] = mine;
    }
    __syncthreads();
    const int left = min(n, top);
    if ((int)threadIdx.x < left) l.key[threadIdx.x] = l.sorted[threadIdx.x];
    if (threadIdx.x == 0) l.count = left;
    __syncthreads();
}

template <class T>
struct Word {  // 16 bytes of logits
    static constexpr int size = 16 / sizeof(T);
};

// Three workgroups a compute unit leave a lane 168 registers; of f32 with the
// likeliest one more is kept in scratch, read once a row.
template <class T, bool kTop>
__global__ __launch_bounds__(kThreads, 3) void logprobs_rows(Logprobs p) {
    constexpr int kWord = Word<T>::size, kWords = kEach / kWord;
    static_assert(II_MAX_TOP * kEach + II_MAX_TOP < kList - 1);
    using vec = __attribute__((ext_vector_type(kWord))) T;
    __shared__ __attribute__((aligned(16))) char lds[kTop ? sizeof(List) : 16];
    __shared__ Sums waves[kThreads / 64];
    List& list = *reinterpret_cast<List*>(lds);
    const int t = threadIdx.x;
    const float to2 = p.scale * kLog2e;
    const double unit = p.scale / (double)to2;  // of u in z

    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        // Words are whole ones of memory: tokens before the row's first and past
        // its last are left out of the word that they share with it.
        const T* logits = static_cast<const T*>(p.logits) + row * p.stride;
        const int lead = (int)(reinterpret_cast<uintptr_t>(logits) % 16 / sizeof(T));
        const vec* from = reinterpret_cast<const vec*>(logits - lead);
        const int64_t begin = blockIdx.x * p.part;
        const int64_t end = min(begin + p.part, (int64_t)p.vocab + lead);
        // asked for here, wanted at the end
        int64_t target = -1;
        float logit = 0;
        if (t == 0 && p.logprob) {
            target = p.targets[row];
            if (target >= 0 && target < p.vocab) logit = (float)logits[target];
        }
        Sums sums = no_sums();
        uint64_t bound = 0;
        if (kTop) {
            if (t == 0) list.count = list.added[0] = list.added[1] = list.added[2] = 0;
            __syncthreads();
        }
        int turn = 0;  // of three counters: one in use, one read, one cleared
        for (int64_t base = begin; base < end; base += kTile) {
            float x[kEach];
            const auto at = [&](int i) { return base + ((int64_t)(i / kWord) * kThreads + t) * kWord + i % kWord; };
            const bool whole = base >= lead && base + kTile <= end;
            if (whole) {
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    const vec v = from[at(w * kWord) / kWord];
#pragma unroll
                    for (int j = 0; j < kWord; ++j) x[w * kWord + j] = (float)v[j];
                }
            } else {
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    vec v = {};
                    if (at(w * kWord) < end) v = from[at(w * kWord) / kWord];
#pragma unroll
                    for (int j = 0; j < kWord; ++j) {
                        const int64_t e = at(w * kWord + j);
                        x[w * kWord + j] = e >= lead && e < end ? (float)v[j] : -INFINITY;
                    }
                }
            }
            float most = x[0];
#pragma unroll
            for (int i = 1; i < kEach; ++i) most = fmaxf(most, x[i]);
            move_to(sums, fmaxf(sums.m, most), to2);
            const float ref = sums.m == -INFINITY ? 0.0f : sums.m;
            float s = 0, below = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const float u = (x[i] - ref) * to2, e = exp2_of(u);
                s += e;
                below = fmaf(e, fmaxf(u, -3e38f), below);
            }
            sums.s += s;
            sums.t += below;
            if constexpr (kTop) {
                const int top = p.top;
                const auto real = [&](int i) { return whole || (at(i) >= lead && at(i) < end); };
                if ((int)list.count < top) {
                    const float reach = bound_of(most == most ? most : -INFINITY, top, list.room);
                    // below the keys of what reaches it
                    if (reach > -INFINITY) bound = max(bound, (uint64_t)order_of(reach) << 32);
                }
                // Logits from here on are above the bound: of those that equal a
                // token's the later ones are not. Without a bound all are.
                const float from_here = float_of((uint32_t)(bound >> 32) + ((uint32_t)bound != 0));
                uint32_t mask = 0;
                if (bound) {
#pragma unroll
                    for (int i = 0; i < kEach; ++i) mask |= (x[i] >= from_here ? 1u : 0u) << i;
                } else {
#pragma unroll
                    for (int i = 0; i < kEach; ++i) mask |= (real(i) ? 1u : 0u) << i;
                }
                int hits = __popc(mask);
                uint32_t place = 0;
                if (hits) place = atomicAdd(&list.added[turn], (uint32_t)hits);
                __syncthreads();
                uint32_t added = list.added[turn];
                turn = turn == 2 ? 0 : turn + 1;
                if (t == 0) list.added[turn == 2 ? 0 : turn + 1] = 0;
                const uint32_t held = list.count;
                if (added) {  // alike in all threads
                    if (added > 3 * (uint32_t)top + kPruned || held + added > kList - 2) {
                        // too many: the tile's own bound, unless fewer than
                        // `top` threads hold any
                        uint64_t mine = 0;
#pragma unroll
                        for (int i = 0; i < kEach; ++i)
                            if (real(i)) mine = max(mine, key_of(x[i], (int)(at(i) - lead)));
                        list.best[t] = mine;
                        if (t == 0) {
                            list.least = 0;
                            list.more = 0;
                        }
                        __syncthreads();
                        if (mine && above(list.best, kThreads, mine) == top - 1) list.least = mine;
                        __syncthreads();
                        if (list.least) bound = max(bound, list.least - 1);
                        prune(list, top);
                        mask = 0;
#pragma unroll
                        for (int i = 0; i < kEach; ++i)
                            mask |= (real(i) && key_of(x[i], (int)(at(i) - lead)) > bound ? 1u : 0u) << i;
                        hits = __popc(mask);
                        if (hits) place = atomicAdd(&list.more, (uint32_t)hits);
                        __syncthreads();
                        added = list.more;
                    }
                    place += list.count;
                    if (hits)
#pragma unroll
                        for (int i = 0; i < kEach; ++i)
                            if (mask >> i & 1) list.key[place++] = key_of(x[i], (int)(at(i) - lead));
                    __syncthreads();
                    if (t == 0) list.count += added;
                    __syncthreads();
                    if ((int)list.count > 3 * top + kPruned || (int)list.count - (int)added < top) {
                        prune(list, top);
                        if ((int)list.count >= top) bound = list.key[top - 1];
                    }
                }
            }
        }

        sums = sum_of(sums, to2, waves);
        if constexpr (kTop) {
            if (p.parts == 1 || (int)list.count > p.top) prune(list, p.top);
        }

        if (p.parts > 1) {
            // a part: m, s, t, then its keys
            const Rsrc parts = buffer(p.partial + row * p.parts * p.room,
                                      (int64_t)p.parts * p.room * 4);
            const uint32_t mine = blockIdx.x * p.room * 4;
            using f64x2 = __attribute__((ext_vector_type(2))) double;
            if (t == 0) {
                leave_part(parts, mine, f32x4{sums.m, 0, 0, 0});
                leave_part(parts, mine + 16, __builtin_bit_cast(f32x4, f64x2{sums.s, sums.t}));
            }
            using u64x2 = __attribute__((ext_vector_type(2))) uint64_t;
            if (kTop)
                for (int i = t * 2; i < p.top; i += kThreads * 2) {
                    const int n = (int)list.count;
                    leave_part(parts, mine + 32 + i * 8,
                               __builtin_bit_cast(f32x4, u64x2{i < n ? list.key[i] : 0,
                                                               i + 1 < n ? list.key[i + 1] : 0}));
                }
            if (!arrive_last(&p.counters[row], p.parts)) continue;
            // the sums of part t, asked for before the keys
            f32x4 m = {-INFINITY, 0, 0, 0}, st = {};
            if (t < p.parts) {
                m = take_part(parts, t * p.room * 4);
                st = take_part(parts, t * p.room * 4 + 16);
            }
            if constexpr (kTop) {
                // as many parts at once as the list has room for beside `top`
                const int pairs = (p.top + 1) / 2, step = max(1, (kList - 2 - p.top) / (2 * pairs));
                if (t == 0) list.count = 0;
                __syncthreads();
                for (int q0 = 0; q0 < p.parts; q0 += step) {
                    const int n = min(step, p.parts - q0), held = (int)list.count;
                    for (int i = t; i < n * pairs; i += kThreads) {
                        const u64x2 k = __builtin_bit_cast(
                            u64x2, take_part(parts, (q0 + i / pairs) * p.room * 4 + 32 + i % pairs * 16));
                        list.key[held + i * 2] = k[0];
                        list.key[held + i * 2 + 1] = k[1];
                    }
                    __syncthreads();
                    if (t == 0) list.count = held + n * pairs * 2;
                    __syncthreads();
                    prune(list, p.top);
                }
            }
            sums = no_sums();
            for (int q = t; q < p.parts; q += kThreads) {
                if (q != t) {
                    m = take_part(parts, q * p.room * 4);
                    st = take_part(parts, q * p.room * 4 + 16);
                }
                const f64x2 both = __builtin_bit_cast(f64x2, st);
                join(sums, Sums{m[0], both[0], both[1]}, to2);
            }
            sums = sum_of(sums, to2, waves);
        }

        // nothing but -infinity: every log-probability is -infinity, the entropy 0
        const bool none = sums.m == -INFINITY && sums.s == 0;
        // The exponentials were of z (1 + off), as scale / ln 2 was rounded: their
        // sum's logarithm is off by off times the mean of z - m, the same way in
        // every term, where other roundings cancel. unit / ln 2 is 1 - off.
        const double mean = none ? 0.0 : unit * (sums.t / sums.s);
        const double logs = none ? 0.0 : log(sums.s) + fma(mean * unit, 1.4426950408889634, -mean);
        const auto result = [&](float x) {
            return none ? -INFINITY : (float)(((double)x - sums.m) * p.scale - logs);
        };
        if (t == 0) {
            if (p.logprob) {
                p.logprob[row] = target >= 0 && target < p.vocab ? result(logit) : 0.0f;
            }
            if (p.entropy) {
                const double h = logs - mean;
                p.entropy[row] = h < 0 ? 0.0f : (float)h;
            }
        }
        if constexpr (kTop) {
            for (int i = t; i < p.top; i += kThreads) {
                // places past the vocabulary, which parts leave as 0
                const uint64_t k = i < (int)list.count ? list.key[i] : 0;
                p.top_ids[row * p.top + i] = k ? (int64_t)(uint32_t)~(uint32_t)k : -1;
                p.top_logprobs[row * p.top + i] = k ? result(logit_of(k)) : -INFINITY;
            }
        }
        __syncthreads();  // what LDS holds of this row has been read
    }
}

template <class T>
int run(const ii_logprobs_args& a, hipStream_t stream) {
    Logprobs p;
    p.logits = a.logits;
    p.targets = a.targets;
    p.logprob = a.logprob;
    p.entropy = a.entropy;
    p.top_ids = a.top_ids;
    p.top_logprobs = a.top_logprobs;
    p.stride = a.rows > 1 ? a.logits_stride : 0;
    p.rows = a.rows;
    p.vocab = (int32_t)a.vocab;
    p.top = a.top;
    p.scale = a.scale;
    p.room = (uint32_t)groups(8 + 2 * a.top, 4) * 4;
    p.counters = nullptr;
    p.partial = nullptr;
    // few rows are cut into parts of a tile or more, three workgroups a compute
    // unit: with four, which wait for one another, 48 x 128256 took 31.7 us
    // against 27.5, with two 28.0
    constexpr int64_t kWanted = 768;
    int64_t parts = 1;
    if (a.work_bytes > kWorkHead && a.rows <= (int64_t)kWorkCounters) {
        p.counters = static_cast<uint32_t*>(a.work);
        p.partial = reinterpret_cast<float*>(static_cast<char*>(a.work) + kWorkHead);
        const int64_t floats = (std::min<uint64_t>(a.work_bytes, II_WORK_BYTES) - kWorkHead) / 4;
        parts = std::min<int64_t>({groups(a.vocab, kTile), kWanted / a.rows, floats / (a.rows * p.room)});
        if (a.top) parts = std::min<int64_t>(parts, 1024 / a.top);
        parts = std::max<int64_t>(parts, 1);
    }
    // a row may begin inside a word
    p.part = groups(groups(a.vocab + 7, parts), kThreads) * kThreads;
    p.parts = (int32_t)groups(a.vocab + 7, p.part);
    const dim3 grid(p.parts, (uint32_t)std::min<int64_t>(a.rows, 65535));
    if (a.top)
        logprobs_rows<T, true><<<grid, kThreads, 0, stream>>>(p);
    else
        logprobs_rows<T, false><<<grid, kThreads, 0, stream>>>(p);
    return launched("ii_logprobs");
}

int check(const ii_logprobs_args& a) {
    const char* fn = "ii_logprobs";
    if (!half_type(a.dtype) && a.dtype != II_F32) return fail(II_EINVAL, "%s: dtype %d", fn, a.dtype);
    if (a.top < 0 || a.top > II_MAX_TOP) return fail(II_EINVAL, "%s: top is %d", fn, a.top);
    if (a.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, a.reserved);
    if (a.rows < 0 || a.rows > INT32_MAX || a.vocab < 1 || a.vocab > INT32_MAX)
        return fail(II_EINVAL, "%s: %lld rows of %lld logits", fn, (long long)a.rows,
                    (long long)a.vocab);
    // exponentials are taken of scale / ln 2 times a difference, which may be 0
    if (!std::isfinite(a.scale * kLog2e) || !(a.scale > 0))
        return fail(II_EINVAL, "%s: scale %g", fn, a.scale);
    if (!a.rows) return II_OK;  // operands of no elements may be NULL
    if (!a.targets != !a.logprob)
        return fail(II_EINVAL, "%s: logprob and targets go together", fn);
    if (!a.top_ids != !a.top || !a.top_logprobs != !a.top)
        return fail(II_EINVAL, "%s: top_ids and top_logprobs go with a top above 0", fn);
    if (!a.logprob && !a.entropy && !a.top)
        return fail(II_EINVAL, "%s: nothing is wanted", fn);
    if (a.logits_stride < 0) return fail(II_EINVAL, "%s: a stride is negative", fn);
    const uint64_t rows = a.rows, size = a.dtype == II_F32 ? 4 : 2;
    uint64_t stride;
    if (__builtin_mul_overflow((uint64_t)(rows > 1 ? a.logits_stride : 0), size, &stride))
        return fail(II_EOVERFLOW, "%s: the stride of logits", fn);
    Rows logits, targets, scratch, out[4];
    const uint64_t top = a.top;
    const struct {
        const char* what;
        const void* p;
        uint64_t bytes, align;
    } outs[4] = {{"logprob", a.logprob, rows * 4, 4},
                 {"entropy", a.entropy, rows * 4, 4},
                 {"top_ids", a.top_ids, rows * top * 8, 8},
                 {"top_logprobs", a.top_logprobs, rows * top * 4, 4}};
    int rc = check_rows(fn, "logits", a.logits, rows, (uint64_t)a.vocab * size, stride, size, &logits);
    if (!rc && a.targets) rc = check_rows(fn, "targets", a.targets, 1, rows * 8, 0, 8, &targets);
    if (!rc) rc = check_work(fn, a.work, a.work_bytes, &scratch);
    if (rc || (rc = check_apart(fn, "logits", scratch, logits)) ||
        (rc = check_apart(fn, "targets", scratch, targets)))
        return rc;
    for (int i = 0; i < 4; ++i) {
        if (!outs[i].p) continue;
        rc = check_rows(fn, outs[i].what, outs[i].p, 1, outs[i].bytes, 0, outs[i].align, &out[i]);
        if (rc || (rc = check_apart(fn, "logits", out[i], logits)) ||
            (rc = check_apart(fn, "targets", out[i], targets)) ||
            (rc = check_apart(fn, "work", out[i], scratch)))
            return rc;
        for (int j = 0; j < i; ++j)
            if ((rc = check_apart(fn, outs[j].what, out[i], out[j]))) return rc;
    }
    return II_OK;
}

}  // namespace
}  // namespace ii

extern "C" int ii_logprobs(const ii_logprobs_args* a, hipStream_t stream) {
    if (!a) return ii::fail(II_EINVAL, "ii_logprobs: args is NULL");
    {
        const ii::Checks checks;
        if (const int rc = ii::check(*a)) return rc;
    }
    if (!a->rows) return II_OK;
    if (a->dtype == II_F32) return ii::run<float>(*a, stream);
    return a->dtype == II_BF16 ? ii::run<__bf16>(*a, stream) : ii::run<_Float16>(*a, stream);
}
