// ii_adapt: low-rank adapters of many requests beside a shared projection,
// out[i] = base[i] + s_a B_a (A_a x[i]), a the adapter of row i.
//
// Rows of one adapter share what is read of it, so rows are taken in tiles of
// one adapter. A few rows, in any order, are gathered: a workgroup counts the
// rows of each adapter and finds which of them its tile of 16 has. Many are put into
// the order of their adapters first, by a kernel of one workgroup; their tiles have
// 32. Where there are more adapters than are counted, or no `work` to note the order
// in, a tile is 32 neighbours, with a pass for each adapter among them.
//
// h = A x is a sum over k that the waves of a workgroup, and workgroups, share.
// For the product with B, whose matrix instruction takes 16 bits, a row of h is
// cut into two or three parts of T, the second what the first's rounding left
// out: 16 bits of bf16 and 22 of f16 in two parts, more than a result of 16 bits
// shows, and all 24 in three, for a result of 32. Parts lie behind one another as
// one longer sum. f16 has little range: rows are brought to its middle by a power
// of two first.
//
// A kernel leaves the parts and the tiles' rows in `work`, a second one
// forms the columns of out, in waves that share nothing and never wait for one
// another. Without `work`, and where the sums are short, each workgroup of a tile's
// columns forms h again, in LDS.
//
// Many rows are bound by memory: 4099 x 4096 x 14336 with 8 adapters of rank 64 and
// a base of 32 bits 121 us, the second kernel 89 of them at 4.0 TB/s. Few are bound
// by the steps from one kernel's first load to the other's last store: 250 x 14336 x
// 4096 with 32 adapters of rank 16 20 us, 4 x 4096 x 4096 12, a call's cost on the
// host being 10.
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

constexpr int kMaxRank = 256;
// Rows that are gathered: 300 rows of 8 adapters take 14.6 us, put into order 17.3
// (4096 x 4096, rank 16); 700 in runs of 350, rank 64, to 14336 39.8 against 34.4,
// 1000 of 32 adapters in no order 26.7 against 22.3. (As neighbours 2000 of 32
// adapters took 109 us, in order 31.)
constexpr int kGathered = 512;
constexpr int kCounted = 1024;   // adapters (and none) whose rows are counted
constexpr int kUnit = 64;        // elements of k a wave takes at once

template <class T>
struct Adapt {
    const T *x, *a, *b;
    const int32_t *adapters, *ranks;
    const float* scales;
    const void* base;
    void* out;
    int64_t x_stride, a_stride, a_row, b_stride, b_row, base_stride, out_stride;
    int32_t m, n, k, rank, count;
    int32_t rankp;        // rank in whole words of 8
    int32_t parts, wide;  // parts of h; elements of a row of parts in LDS
    int32_t columns;      // of out, a workgroup's
    int32_t tiles, splits;  // workgroups that share k of a tile
    int32_t shares;       // workgroups that share its columns
    bool out_f32, base_f32;
    bool ordered;         // the tiles' rows are in memory before the first kernel
    uint32_t* counters;
    float* partial;       // [tiles][splits][rows of a tile][rankp]
    // what the first kernel leaves of each row of each tile
    T* held;              // [wide]
    float* factor;        // of a result
    int32_t *row, *id;    // -1: none
    int32_t* used;        // rows of A, columns of B
};

template <class T>
__device__ inline int adapter_of(const Adapt<T>& p, int64_t row) {
    const int a = p.adapters[row];
    return a >= 0 && a < p.count ? a : -1;
}
template <class T>
__device__ inline int rank_of(const Adapt<T>& p, int a) {
    return p.ranks ? min(max(p.ranks[a], 0), p.rank) : p.rank;
}

template <class T>
__device__ inline float scale_of(const Adapt<T>& p, int a) {
    return p.scales ? p.scales[a] : 1.0f;
}

// A tile's rows and their adapters, -1 for none; places past the last row have
// row -1.
template <int kTok>
struct Tile {
    int row[kTok], id[kTok], rank[kTok];
    float factor[kTok];  // of a result
};

// A workgroup's tile, and which of those that share it this is. The workgroups of
// a tile's columns are neighbours, so that its rows are read and written along;
// those of a tile's k are not. All on one XCD, so that its L2 need not hold every
// adapter, took 4099 rows x 4096 x 14336 from 122 us to 132.
struct Share {
    int tile, share;
};
__device__ inline Share share_of_columns(int shares) {
    return {(int)(blockIdx.x / shares), (int)(blockIdx.x % shares)};
}
__device__ inline Share share_of_k(int tiles) {
    return {(int)(blockIdx.x % tiles), (int)(blockIdx.x / tiles)};
}

// The rows of tile t of the gathered ones, false if there is none. Called by all
// threads.
template <class T, int kTok>
__device__ inline bool gather(const Adapt<T>& p, int t, Tile<kTok>& tile) {
    __shared__ int rows[kCounted];
    constexpr int kWords = kGathered / 64;
    const int lane = threadIdx.x % 64;
    int id[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const int j = i * 64 + lane;
        id[i] = -2;
        if (j < p.m) id[i] = adapter_of(p, j);
    }
    int mine = -2, from = 0;  // the tile's adapter; its rows from this one on
    if (p.count < kCounted) {
        // tiles in the order of adapters, those without one first
        for (int e = threadIdx.x; e <= p.count; e += blockDim.x) rows[e] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            if (i * 64 < p.m && i % (blockDim.x / 64) == threadIdx.x / 64 && id[i] >= -1)
                atomicAdd(&rows[id[i] + 1], 1);
        __syncthreads();
        int before = 0;
        for (int c0 = 0; c0 <= p.count && mine == -2; c0 += 64) {
            const int tiles = c0 + lane <= p.count ? (rows[c0 + lane] + kTok - 1) / kTok : 0;
            int to = tiles;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int v = __shfl_up(to, d);
                if (lane >= d) to += v;
            }
            to += before;
            const uint64_t here = __ballot(to - tiles <= t && t < to);
            if (here) {
                const int at = __builtin_ctzll(here);
                mine = c0 + at - 1;
                from = (t - __shfl(to - tiles, at)) * kTok;
            }
            before = __shfl(to, 63);
        }
        if (mine == -2) return false;
    } else {
        // too many adapters to count: the tile that begins with row t, if one does
        mine = adapter_of(p, t);
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const int past = min(max(t - i * 64, 0), 64);  // of this word, before t
            const uint64_t low = past == 64 ? ~0ull : (1ull << past) - 1;
            from += __popcll(__ballot(id[i] == mine) & low);
        }
        if (from % kTok) return false;
    }
    // asked for here, wanted later
    const int rank = mine < 0 ? 0 : rank_of(p, mine);
    const float factor = mine < 0 ? 0.0f : scale_of(p, mine);
    int found = 0;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        if (i * 64 >= p.m) break;
        const uint64_t same = __ballot(id[i] == mine);
        const int place = found + __popcll(same & ((1ull << lane) - 1)) - from;
        if (threadIdx.x < 64 && same >> lane & 1 && place >= 0 && place < kTok) {
            tile.row[place] = i * 64 + lane;
            tile.id[place] = mine;
        }
        found += __popcll(same);
    }
    if (threadIdx.x < kTok && (int)threadIdx.x >= found - from) {
        tile.row[threadIdx.x] = -1;
        tile.id[threadIdx.x] = -1;
    }
    if (threadIdx.x < kTok) {
        tile.rank[threadIdx.x] = rank;
        tile.factor[threadIdx.x] = factor;
    }
    __syncthreads();
    return true;
}

// Tile b of many rows, in the order that adapt_order has left, or as they come.
// False if it has none.
template <class T, int kTok>
__device__ inline bool of_many(const Adapt<T>& p, int b, Tile<kTok>& tile) {
    if (p.ordered && p.row[(int64_t)b * kTok] < 0) return false;
    if (threadIdx.x < kTok) {
        int64_t i = (int64_t)b * kTok + threadIdx.x;
        int id = -1;
        if (p.ordered) {
            id = p.id[i];
            i = p.row[i];
        } else {
            if (i >= p.m) i = -1;
            if (i >= 0) id = adapter_of(p, i);
        }
        tile.row[threadIdx.x] = (int)i;
        tile.id[threadIdx.x] = id;
        tile.rank[threadIdx.x] = id < 0 ? 0 : rank_of(p, id);
        tile.factor[threadIdx.x] = id < 0 ? 0.0f : scale_of(p, id);
    }
    __syncthreads();
    return true;
}

// Many rows in the order of their adapters, each adapter's from a tile's first
// place on: places without a row have row -1. One workgroup counts, adds up and
// puts them; rows of an adapter come in no order, which no result depends on, but
// 64 neighbours of one stay together.
constexpr int kOrderThreads = 1024;
template <class T, int kTok>
__global__ __launch_bounds__(kOrderThreads) void adapt_order(Adapt<T> p) {
    __shared__ int rows[kCounted], next[kCounted], waves[kOrderThreads / 64];
    const int t = threadIdx.x, lane = t % 64;
    rows[t] = 0;
    __syncthreads();
    // takes a place for each lane's adapter (0: none), the lanes of one together
    const auto take = [&](int* from, int id) {
        const int first = __builtin_amdgcn_readfirstlane(id);
        if (__ballot(id != first) == 0) {
            int at = 0;
            if (lane == 0 && first >= 0) at = atomicAdd(&from[first], 64);
            return __shfl(at, 0) + lane;
        }
        return id >= 0 ? atomicAdd(&from[id], 1) : 0;
    };
    // put(row, adapter), some rows' adapters asked for at once
    const auto each = [&](auto&& put) {
        constexpr int kAhead = 4;
        for (int64_t base = 0; base < p.m; base += kAhead * kOrderThreads) {
            int id[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t i = base + u * kOrderThreads + t;
                id[u] = i < p.m ? adapter_of(p, i) + 1 : -1;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) put(base + u * kOrderThreads + t, id[u]);
        }
    };
    each([&](int64_t, int id) { take(rows, id); });
    __syncthreads();
    static_assert(kCounted == kOrderThreads);
    const int held = t <= p.count ? rows[t] : 0, tiles = (held + kTok - 1) / kTok;
    int to = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(to, d);
        if (lane >= d) to += v;
    }
    if (lane == 63) waves[t / 64] = to;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kOrderThreads / 64; ++w) {
        if (w < t / 64) before += waves[w];
        total += waves[w];
    }
    const int first = (before + to - tiles) * kTok;
    next[t] = first;
    for (int e = first + held; e < first + tiles * kTok; ++e) {
        p.row[e] = -1;
        p.id[e] = -1;
    }
    for (int64_t e = (int64_t)total * kTok + t; e < (int64_t)p.tiles * kTok; e += kOrderThreads) {
        p.row[e] = -1;
        p.id[e] = -1;
    }
    __syncthreads();
    each([&](int64_t i, int id) {
        const int e = take(next, id);
        if (id >= 0) {
            p.row[e] = (int)i;
            p.id[e] = id - 1;
        }
    });
}

// The least adapter of the tile above a, or INT_MAX; its rank.
template <int kTok>
__device__ inline int next_adapter(const Tile<kTok>& tile, int a, int& rank) {
    static_assert(kTok <= 64);
    const int id = tile.id[threadIdx.x % kTok];
    int v = id > a ? id : INT32_MAX;
#pragma unroll
    for (int d = 1; d < kTok; d *= 2) v = min(v, __shfl_xor(v, d));
    v = __builtin_amdgcn_readfirstlane(v);
    const uint64_t here = __ballot(id == v);
    rank = here ? __builtin_amdgcn_readfirstlane(tile.rank[__builtin_ctzll(here) % kTok]) : 0;
    return v;
}

// 16 bytes at any multiple of an element: the same instruction at every alignment.
template <class V, class T>
__device__ inline V word_at(const T* from) {
    V v;
    static_assert(sizeof(V) == 16);
    __builtin_memcpy(&v, from, 16);
    return v;
}
// Elements of a row from `from` on, of which `left` are there, others zero.
template <class T>
__device__ inline typename Vec<T>::x8 some(const T* from, int64_t left) {
    typename Vec<T>::x8 v = {};
    if (left >= 8) return word_at<typename Vec<T>::x8>(from);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) v[j] = from[j];
    return v;
}

// Rows r0 .. r0 + kR * 16 of h of the tile's rows whose adapter is a, this
// workgroup's share of k, given to keep(token, rank, value).
template <class T, int kR, int kTT, int kWaves, class Keep>
__device__ inline void shrink(const Adapt<T>& p, const Tile<kTT * 16>& tile, int a, int rank, int r0, int split,
                              float* red, Keep&& keep) {
    using x8 = typename Vec<T>::x8;
    constexpr int kSums = kR * kTT * 256;
    const int lane = threadIdx.x % 64, row = lane % 16, part = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const T *ap[kR], *xp[kTT];
#pragma unroll
    for (int r = 0; r < kR; ++r)  // rows past the rank are left out below
        ap[r] = p.a + a * p.a_stride + min(r0 + r * 16 + row, max(rank - 1, 0)) * p.a_row + part * 8;
#pragma unroll
    for (int t = 0; t < kTT; ++t) xp[t] = p.x + max(tile.row[t * 16 + row], 0) * p.x_stride + part * 8;
    f32x4 acc[kR][kTT] = {};
    const int units = (int)groups(p.k, kUnit), whole = p.k / kUnit;
    // each wave takes neighbouring units: rows begin at few of the memory's
    // channels, and waves side by side would be at the same ones
    const int each = (units + kWaves * p.splits - 1) / (kWaves * p.splits);
    const int begin = (split * kWaves + wave) * each;
    const int end = min(begin + each, units), full = min(end, whole);
    constexpr int kAhead = kTT > 1 ? 2 : 4;  // units whose loads are on their way
    const auto take = [&](int u, x8(&av)[2][kR], x8(&xv)[2][kTT]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t k = (int64_t)u * kUnit + h * 32;
#pragma unroll
            for (int r = 0; r < kR; ++r) av[h][r] = word_at<x8>(ap[r] + k);
#pragma unroll
            for (int t = 0; t < kTT; ++t) xv[h][t] = word_at<x8>(xp[t] + k);
        }
    };
    const auto multiply = [&](const x8(&av)[2][kR], const x8(&xv)[2][kTT]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < kR; ++r)
#pragma unroll
                for (int t = 0; t < kTT; ++t) acc[r][t] = mfma16(av[h][r], xv[h][t], acc[r][t]);
    };
    if (rank > r0) {
        for (int u = begin; u < full; u += kAhead) {
            x8 av[kAhead][2][kR], xv[kAhead][2][kTT];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (u + i < full) take(u + i, av[i], xv[i]);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (u + i < full) multiply(av[i], xv[i]);
        }
        // what is left, past the last whole unit
        for (int u = max(begin, whole); u < end; ++u) {
            x8 av[2][kR], xv[2][kTT];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t k = (int64_t)u * kUnit + h * 32, left = p.k - k - part * 8;
#pragma unroll
                for (int r = 0; r < kR; ++r) av[h][r] = some(ap[r] + k, left);
#pragma unroll
                for (int t = 0; t < kTT; ++t) xv[h][t] = some(xp[t] + k, left);
            }
            multiply(av, xv);
        }
    }
    // red[wave][r][t][token][row of h]
#pragma unroll
    for (int r = 0; r < kR; ++r)
#pragma unroll
        for (int t = 0; t < kTT; ++t)
            *reinterpret_cast<f32x4*>(&red[wave * kSums + ((r * kTT + t) * 16 + row) * 16 + part * 4]) =
                acc[r][t];
    __syncthreads();
    for (int e = threadIdx.x; e < kSums; e += kWaves * 64) {
        float s = red[e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += red[w * kSums + e];
        const int token = e / 256 % kTT * 16 + e / 16 % 16, r = r0 + e / (256 * kTT) * 16 + e % 16;
        if (tile.id[token] == a && r < p.rankp) keep(token, r, r < rank ? s : 0.0f);
    }
    __syncthreads();
}

// h[token][rank] cut into parts of T, [token][part][rank], for the product with B.
template <class T, int kTok, int kThreads>
__device__ inline void cut(const Adapt<T>& p, Tile<kTok>& tile, const float* h, T* parts) {
    constexpr int kLanes = std::min(64, kThreads / kTok);
    const int token = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    if (token < kTok) {
        const float* mine = h + token * p.rankp;
        float up = 1, down = 1;
        if constexpr (std::is_same_v<T, _Float16>) {
            float most = 0;
            for (int r = lane; r < p.rankp; r += kLanes) most = fmaxf(most, fabsf(mine[r]));
#pragma unroll
            for (int d = 1; d < kLanes; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
            // the largest to 2^12 .. 2^13
            const int e = min(max((int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127 - 12, -100), 100);
            if (most > 0) {
                up = __builtin_bit_cast(float, (uint32_t)(127 + e) << 23);
                down = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
            }
        }
        if (lane == 0) tile.factor[token] *= up;
        T* to = parts + token * p.wide;
        for (int r = lane; r < p.rankp; r += kLanes) {
            float rest = mine[r] * down;
            for (int q = 0; q < p.parts; ++q) {
                const T v = (T)rest;
                to[q * p.rankp + r] = v;
                rest -= (float)v;
                if (!(fabsf(rest) <= 3e38f)) rest = 0;  // of what is not finite nothing is left
            }
        }
        for (int i = p.parts * p.rankp + lane; i < p.wide; i += kLanes) to[i] = (T)0.0f;
    }
    __syncthreads();
}

enum { kNoBase, kBaseT, kBaseF32 };

// Eight columns of a row of base as they lie there.
template <class T, int kBase>
struct Base {
    u32x4 word[kBase == kBaseF32 ? 2 : 1];
};
// Columns j .. j + 7 of a row of base, and of out; `whole`: they are all
// there.
template <class T, int kBase>
__device__ inline void base_of(const Adapt<T>& p, int64_t row, int64_t j, bool whole, Base<T, kBase>& v) {
    const int64_t at = row * p.base_stride + j;
    if constexpr (kBase == kBaseF32) {
        const float* from = static_cast<const float*>(p.base) + at;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (whole) {
                v.word[h] = word_at<u32x4>(from + h * 4);
            } else {
                v.word[h] = u32x4{};
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (j + h * 4 + r < p.n) v.word[h][r] = __builtin_bit_cast(uint32_t, from[h * 4 + r]);
            }
        }
    } else if constexpr (kBase == kBaseT) {
        const T* from = static_cast<const T*>(p.base) + at;
        v.word[0] = whole ? word_at<u32x4>(from) : __builtin_bit_cast(u32x4, some(from, p.n - j));
    }
}
template <class T, int kBase>
__device__ inline void put(const Adapt<T>& p, int64_t row, int64_t j, f32x4 low, f32x4 high,
                           const Base<T, kBase>& base, bool whole) {
    using x8 = typename Vec<T>::x8;
    float y[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        y[r] = r < 4 ? low[r] : high[r - 4];
        if constexpr (kBase == kBaseF32)
            y[r] += __builtin_bit_cast(float, (uint32_t)base.word[r / 4][r % 4]);
        else if constexpr (kBase == kBaseT)
            y[r] += (float)__builtin_bit_cast(x8, base.word[0])[r];
    }
    const int64_t at = row * p.out_stride + j;
    if (p.out_f32) {
        float* out = static_cast<float*>(p.out) + at;
        if (whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 v = {y[h * 4], y[h * 4 + 1], y[h * 4 + 2], y[h * 4 + 3]};
                __builtin_memcpy(out + h * 4, &v, 16);
            }
            return;
        }
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (j + r < p.n) out[r] = y[r];
    } else {
        T* out = static_cast<T*>(p.out) + at;
        x8 v;
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = (T)y[r];
        if (whole) {
            __builtin_memcpy(out, &v, 16);
            return;
        }
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (j + r < p.n) out[r] = v[r];
    }
}

// Columns first, first + step, .. below end, kC * 16 at a time, of the kTT * 16
// rows of out that a wave has: of each 16, lane l has row l mod 16, of which
// `rows`, `ids`, `ranks` and `factors` are told, and `parts` is h cut, [row][wide]. kFast:
// rankp, if a row's parts are two and stay in registers (0: neither).
//
// Of two products of 16 columns a lane gets four columns each; the rows of B are
// given to them so that these are eight neighbours, a word of out.
template <class T, int kTT, int kC, int kFast, int kBase>
__device__ inline void expand(const Adapt<T>& p, const int (&rows)[kTT], const int (&ids)[kTT],
                              const int (&ranks)[kTT], const float (&factors)[kTT], const T* parts, int64_t first, int64_t step,
                              int64_t end) {
    using x8 = typename Vec<T>::x8;
    const int lane = threadIdx.x % 64, row = lane % 16, part = lane / 16;
    const int held = p.parts * p.rankp, place = row / 4 * 8 + row % 4;
    // what a part's steps read of B; both parts of 16 go into one instruction
    constexpr int kSteps = kFast > 16 ? kFast / 32 : 1, kTimes = kFast > 16 ? 2 : 1;
    x8 hv[kTimes * kSteps][kTT];
    if constexpr (kFast != 0)
#pragma unroll
        for (int s = 0; s < kTimes * kSteps; ++s)
#pragma unroll
            for (int t = 0; t < kTT; ++t)
                hv[s][t] = *reinterpret_cast<const x8*>(parts + (t * 16 + row) * p.wide + s * 32 + part * 8);
    const auto next = [&](int a) {
        int v = INT32_MAX;
#pragma unroll
        for (int t = 0; t < kTT; ++t)
            if (ids[t] > a) v = min(v, ids[t]);
#pragma unroll
        for (int d = 1; d < 16; d *= 2) v = min(v, __shfl_xor(v, d));
        return __builtin_amdgcn_readfirstlane(v);
    };
    const auto rank_in = [&](int a) {
        int r = 0;
#pragma unroll
        for (int t = 0; t < kTT; ++t)
            if (const uint64_t here = __ballot(ids[t] == a))
                r = __builtin_amdgcn_readlane(ranks[t], __builtin_ctzll(here));
        return r;
    };
    // base is asked for a step ahead, behind what is read of B; alike in all
    // lanes, so that no branch comes between the loads
    static_assert(kC % 2 == 0);
    Base<T, kBase> base[kC / 2][kTT], ahead[kC / 2][kTT];
    const auto whole = [&](int64_t n0) { return n0 + kC * 16 <= p.n; };
    const auto ask = [&](int64_t n0) {
        if (kBase == kNoBase || n0 >= end) return;
        if (whole(n0)) {
#pragma unroll
            for (int t = 0; t < kTT; ++t)
#pragma unroll
                for (int c = 0; c < kC / 2; ++c)
                    base_of(p, max(rows[t], 0), n0 + c * 32 + part * 8, true, ahead[c][t]);
        } else {
#pragma unroll
            for (int t = 0; t < kTT; ++t)
#pragma unroll
                for (int c = 0; c < kC / 2; ++c)
                    base_of(p, max(rows[t], 0), n0 + c * 32 + part * 8, false, ahead[c][t]);
        }
    };
    const int a0 = next(-1);
    ask(first);
    for (int64_t n0 = first; n0 < end; n0 += step) {
#pragma unroll
        for (int t = 0; t < kTT; ++t)
#pragma unroll
            for (int c = 0; c < kC / 2; ++c) base[c][t] = ahead[c][t];
        bool asked = false;
        f32x4 total[kC][kTT] = {};
        for (int a = a0; a != INT32_MAX; a = next(a)) {
            const int rank = rank_in(a);
            const T* b[kC];
#pragma unroll
            for (int c = 0; c < kC; ++c)
                b[c] = p.b + a * p.b_stride + min(n0 + c / 2 * 32 + place + c % 2 * 4, (int64_t)p.n - 1) * p.b_row;
            f32x4 acc[kC][kTT] = {};
            const bool words = rank % 8 == 0 && rank > 0;
            if constexpr (kFast != 0) {
                x8 bv[kC][kSteps];
                if (words) {
#pragma unroll
                    for (int c = 0; c < kC; ++c)
#pragma unroll
                        for (int s = 0; s < kSteps; ++s) {
                            const int col = (s * 32 + part * 8) % kFast;
                            bv[c][s] = word_at<x8>(b[c] + (col < rank ? col : 0));
                        }
                } else {
#pragma unroll
                    for (int c = 0; c < kC; ++c)
#pragma unroll
                        for (int s = 0; s < kSteps; ++s) {
                            const int col = (s * 32 + part * 8) % kFast;
                            bv[c][s] = some(b[c] + col, rank - col);
                        }
                }
                if (!asked) ask(n0 + step);
                asked = true;
                if (rank < kFast)
#pragma unroll
                    for (int c = 0; c < kC; ++c)
#pragma unroll
                        for (int s = 0; s < kSteps; ++s)
                            if ((s * 32 + part * 8) % kFast >= rank) bv[c][s] = x8{};
#pragma unroll
                for (int s = 0; s < kTimes * kSteps; ++s)
#pragma unroll
                    for (int c = 0; c < kC; ++c)
#pragma unroll
                        for (int t = 0; t < kTT; ++t)
                            acc[c][t] = mfma16(bv[c][s % kSteps], hv[s][t], acc[c][t]);
            } else {
                int col = part * 8;
                while (col >= p.rankp) col -= p.rankp;
                for (int at = part * 8; at < p.wide; at += 32) {
                    const bool there = at < held && col < rank;
                    x8 bv[kC], h[kTT];
                    if (words) {
#pragma unroll
                        for (int c = 0; c < kC; ++c)
                            bv[c] = word_at<x8>(b[c] + (there ? col : 0));
                    } else {
#pragma unroll
                        for (int c = 0; c < kC; ++c) bv[c] = some(b[c] + col, rank - col);
                    }
#pragma unroll
                    for (int t = 0; t < kTT; ++t)
                        h[t] = *reinterpret_cast<const x8*>(parts + (t * 16 + row) * p.wide + at);
#pragma unroll
                    for (int c = 0; c < kC; ++c)
                        if (!there) bv[c] = x8{};
#pragma unroll
                    for (int c = 0; c < kC; ++c)
#pragma unroll
                        for (int t = 0; t < kTT; ++t) acc[c][t] = mfma16(bv[c], h[t], acc[c][t]);
                    col += 32;
                    while (col >= p.rankp) col -= p.rankp;
                }
                if (!asked) ask(n0 + step);
                asked = true;
            }
            // a row has one adapter; what others have there does not matter
#pragma unroll
            for (int t = 0; t < kTT; ++t)
#pragma unroll
                for (int c = 0; c < kC; ++c)
                    total[c][t] = ids[t] == a ? acc[c][t] * factors[t] : total[c][t];
        }
        if (!asked) ask(n0 + step);
        if (whole(n0)) {
#pragma unroll
            for (int t = 0; t < kTT; ++t)
                if (rows[t] >= 0)
#pragma unroll
                    for (int c = 0; c < kC / 2; ++c)
                        put(p, rows[t], n0 + c * 32 + part * 8, total[c * 2][t], total[c * 2 + 1][t],
                            base[c][t], true);
        } else {
#pragma unroll
            for (int t = 0; t < kTT; ++t)
                if (rows[t] >= 0)
#pragma unroll
                    for (int c = 0; c < kC / 2; ++c)
                        put(p, rows[t], n0 + c * 32 + part * 8, total[c * 2][t], total[c * 2 + 1][t],
                            base[c][t], false);
        }
    }
}

template <bool kBoth, int kR, int kTT, int kWaves, class T>
__host__ __device__ inline int first_lds(const Adapt<T>& p) {
    const int red = kWaves * kR * kTT * 1024, parts = kBoth ? kTT * 16 * p.wide * 2 : 0;
    return red > parts ? red : parts;
}

// h of a tile, cut: in LDS, formed by each of the workgroups that share
// the tile's columns, which follow (kBoth); or in memory, by the last to arrive of
// those that share k.
template <class T, bool kBoth, int kR, int kTT, int kWaves>
__global__ __launch_bounds__(kWaves * 64) void adapt_shrink(Adapt<T> p) {
    constexpr int kTok = kTT * 16, kThreads = kWaves * 64;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Tile<kTok> tile;
    const Share mine = kBoth ? share_of_columns(p.shares) : share_of_k(p.tiles);
    const int64_t first = (int64_t)mine.tile * kTok;  // of the rows in memory
    if constexpr (kTT == 1) {
        if (!gather(p, mine.tile, tile)) {
            if (!kBoth && mine.share == 0 && threadIdx.x < kTok) p.row[first + threadIdx.x] = -1;
            return;
        }
    } else {
        if (!of_many(p, mine.tile, tile)) return;
    }
    // what waves add up, and h cut after it, in one place; h
    float* red = reinterpret_cast<float*>(lds);
    float* h = reinterpret_cast<float*>(lds + first_lds<kBoth, kR, kTT, kWaves>(p));
    const int sums = kTok * p.rankp;
    for (int e = threadIdx.x; e < sums; e += kThreads) h[e] = 0;
    __syncthreads();
    int rank;
    for (int a = next_adapter(tile, -1, rank); a != INT32_MAX; a = next_adapter(tile, a, rank))
        for (int r0 = 0; r0 < p.rankp; r0 += kR * 16)
            shrink<T, kR, kTT, kWaves>(p, tile, a, rank, r0, kBoth ? 0 : mine.share, red,
                                       [&](int token, int r, float v) { h[token * p.rankp + r] = v; });
    if constexpr (kBoth) {
        T* parts = reinterpret_cast<T*>(lds);
        cut<T, kTok, kThreads>(p, tile, h, parts);
        const int row = threadIdx.x % 16;
        int rows[kTT], ids[kTT], ranks[kTT];
        float factors[kTT];
#pragma unroll
        for (int t = 0; t < kTT; ++t) {
            ranks[t] = tile.rank[t * 16 + row];
            rows[t] = tile.row[t * 16 + row];
            ids[t] = tile.id[t * 16 + row];
            factors[t] = tile.factor[t * 16 + row];
        }
        constexpr int kC = kTT == 1 ? 4 : 2;
        const int64_t at = (int64_t)mine.share * p.columns;
        const int64_t from = at + threadIdx.x / 64 * kC * 16, end = min(at + p.columns, (int64_t)p.n);
        constexpr int kStep = kWaves * kC * 16;
        if (!p.base)
            expand<T, kTT, kC, 0, kNoBase>(p, rows, ids, ranks, factors, parts, from, kStep, end);
        else if (p.base_f32)
            expand<T, kTT, kC, 0, kBaseF32>(p, rows, ids, ranks, factors, parts, from, kStep, end);
        else
            expand<T, kTT, kC, 0, kBaseT>(p, rows, ids, ranks, factors, parts, from, kStep, end);
    } else {
        if (p.splits > 1) {
            const Rsrc parts = buffer(p.partial + (int64_t)mine.tile * p.splits * sums,
                                      (int64_t)p.splits * sums * 4);
            for (int e = threadIdx.x * 4; e < sums; e += kThreads * 4)
                leave_part(parts, (mine.share * sums + e) * 4, *reinterpret_cast<f32x4*>(h + e));
            if (!arrive_last(&p.counters[mine.tile], p.splits)) return;
            for (int e = threadIdx.x * 4; e < sums; e += kThreads * 4) {
                f32x4 s = {};
#pragma unroll 8
                for (int y = 0; y < p.splits; ++y) s += take_part(parts, (y * sums + e) * 4);
                *reinterpret_cast<f32x4*>(h + e) = s;
            }
            __syncthreads();
        }
        cut<T, kTok, kThreads>(p, tile, h, p.held + first * p.wide);
        if (threadIdx.x < kTok) {
            if (!p.ordered) {
                p.row[first + threadIdx.x] = tile.row[threadIdx.x];
                p.id[first + threadIdx.x] = tile.id[threadIdx.x];
            }
            p.used[first + threadIdx.x] = tile.rank[threadIdx.x];
            p.factor[first + threadIdx.x] = tile.factor[threadIdx.x];
        }
    }
}

// Columns of a tile from what adapt_shrink left: of a workgroup's waves
// kTok / (kTT * 16) share its rows, the others its columns.
template <class T, int kTok, int kTT, int kC, int kFast, int kBase, int kWaves>
__global__ __launch_bounds__(kWaves * 64) void adapt_expand(Adapt<T> p) {
    constexpr int kSides = kTok / (kTT * 16), kSteps = kWaves / kSides;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = threadIdx.x % 16;
    const Share mine = share_of_columns(p.shares);
    const int64_t first = (int64_t)mine.tile * kTok + wave % kSides * kTT * 16;
    int rows[kTT], ids[kTT], ranks[kTT];
    float factors[kTT];
    bool any = false;
#pragma unroll
    for (int t = 0; t < kTT; ++t) {
        // a tile without rows leaves the others as they were
        rows[t] = p.row[first + t * 16 + row];
        ids[t] = p.id[first + t * 16 + row];
        ranks[t] = p.used[first + t * 16 + row];
        factors[t] = p.factor[first + t * 16 + row];
        any |= rows[t] >= 0;
    }
    if (!__any(any)) return;
    const int64_t at = (int64_t)mine.share * p.columns;
    expand<T, kTT, kC, kFast, kBase>(p, rows, ids, ranks, factors, p.held + first * p.wide,
                                     at + wave / kSides * kC * 16, kSteps * kC * 16,
                                     min(at + p.columns, (int64_t)p.n));
}

template <class T, bool kBoth, int kR, int kTT, int kWaves>
void shrink_launch(const Adapt<T>& p, hipStream_t stream) {
    // at most 56 KB
    const uint32_t lds = first_lds<kBoth, kR, kTT, kWaves>(p) + kTT * 16 * p.rankp * 4;
    adapt_shrink<T, kBoth, kR, kTT, kWaves><<<p.tiles * (kBoth ? p.shares : p.splits), kWaves * 64, lds, stream>>>(p);
}

template <class T, bool kBoth, int kTT, int kWaves>
void shrink_rank(const Adapt<T>& p, hipStream_t stream) {
    if (p.rankp <= 16)
        shrink_launch<T, kBoth, 1, kTT, kWaves>(p, stream);
    else if (p.rankp <= 32)
        shrink_launch<T, kBoth, 2, kTT, kWaves>(p, stream);
    else if (kTT == 1 || p.rankp <= 128)
        shrink_launch<T, kBoth, 4, kTT, kWaves>(p, stream);
    else  // h leaves less room
        shrink_launch<T, kBoth, 2, kTT, kWaves>(p, stream);
}

template <class T, int kTok, int kTT, int kC, int kFast>
void expand_base(const Adapt<T>& p, hipStream_t stream) {
    constexpr int kWaves = 4;
    const uint32_t grid = (uint32_t)p.tiles * p.shares;
    if (!p.base)
        adapt_expand<T, kTok, kTT, kC, kFast, kNoBase, kWaves><<<grid, kWaves * 64, 0, stream>>>(p);
    else if (p.base_f32)
        adapt_expand<T, kTok, kTT, kC, kFast, kBaseF32, kWaves><<<grid, kWaves * 64, 0, stream>>>(p);
    else
        adapt_expand<T, kTok, kTT, kC, kFast, kBaseT, kWaves><<<grid, kWaves * 64, 0, stream>>>(p);
}

// Columns a workgroup and the workgroups of a tile: enough to fill the card, if
// `tiles` tiles have rows.
template <class T>
void share_columns(Adapt<T>& p, int columns, int64_t tiles, int64_t wanted) {
    const int64_t shares = std::min(groups(p.n, columns), std::max<int64_t>(1, wanted / tiles));
    p.columns = (int32_t)(groups(groups(p.n, shares), columns) * columns);
    p.shares = (int32_t)groups(p.n, p.columns);
}

template <class T, int kTok, int kTT, int kC>
void expand_launch(Adapt<T> p, int64_t tiles, hipStream_t stream) {
    share_columns(p, 4 / (kTok / (kTT * 16)) * kC * 16, tiles, 4096);
    // Parts of h in registers, or read again for every 64 columns. 250 x 14336 x 4096
    // with 32 adapters takes 18.3 us with rank 8, 18.5 with 16, 22.4 (24), 22.7 (32),
    // 28.4 (48), 31.8 (64), 63.0 (128); 4099 x 4096 x 14336 with 8 adapters 87, 86,
    // 98, 88, 112, 108, 226; with a result of 32 bits, three parts, 118 with rank 16
    // and 196 with 64. Rank 128 would take 64 registers a lane for its parts alone.
    const int fast = p.parts == 2 ? p.rankp : 0;
    if (fast == 16) return expand_base<T, kTok, kTT, kC, 16>(p, stream);
    if (fast == 32) return expand_base<T, kTok, kTT, kC, 32>(p, stream);
    if (fast == 64) return expand_base<T, kTok, kTT, kC, 64>(p, stream);
    expand_base<T, kTok, kTT, kC, 0>(p, stream);
}

// Floats of `work` that a tile takes beside its shares of h.
template <class T>
uint64_t tile_floats(const Adapt<T>& p, int rows) {
    return rows * (p.wide / 2 + 4);
}

// Rows [0, p.m) of a call; floats: the room in `work`.
template <class T, int kTT, int kWaves>
void tiles_launch(Adapt<T> p, char* work, uint64_t floats, hipStream_t stream) {
    constexpr int kTok = kTT * 16;
    int64_t tiles = groups(p.m, kTok);  // at least
    int64_t grid = tiles;
    const bool counted = p.count < kCounted;
    if (kTT == 1 || counted) {
        grid = counted ? std::min<int64_t>(p.m, p.m / kTok + p.count + 1) : p.m;
        tiles = std::min<int64_t>(grid, tiles + p.count);
    }
    p.tiles = (int32_t)grid;
    const uint64_t sums = (uint64_t)kTok * p.rankp, each = tile_floats(p, kTok);
    // One kernel, without room for what the first leaves, or where h is formed again
    // by every workgroup of a tile's columns in one round of loads: 1 x 512 x 1024
    // 7.2 us against 8.3 in two (a call 9.6 against 12.0), 24 x 1024 x 1024 8.0
    // against 10.5, 200 x 1024 x 8192 13.5 against 13.5 of rank 16; of rank 64
    // 24 x 1024 x 8192 takes 23.1 against 17.5.
    const bool short_sums = kTT == 1 && p.rankp <= 16 && p.k <= kUnit * 4 * kWaves;
    if (floats < grid * each || short_sums) {
        if (kTT > 1) p.tiles = (int32_t)(tiles = groups(p.m, kTok));  // as they come
        share_columns(p, kWaves * (kTT == 1 ? 4 : 2) * 16, tiles, 1024);
        p.splits = 1;
        return shrink_rank<T, true, kTT, kWaves>(p, stream);
    }
    // workgroups that share a tile's k: to fill the card, each wave left with
    // two rounds of loads or more
    const int64_t room = (floats - grid * each) / (grid * sums);
    p.splits = (int32_t)std::max<int64_t>(1, std::min({512 / tiles, groups(p.k, kUnit) / (2 * kWaves), room}));
    if (grid > (int64_t)kWorkCounters) p.splits = 1;
    p.counters = reinterpret_cast<uint32_t*>(work);
    p.held = reinterpret_cast<T*>(work + kWorkHead);
    p.factor = reinterpret_cast<float*>(p.held + grid * kTok * p.wide);
    p.row = reinterpret_cast<int32_t*>(p.factor + grid * kTok);
    p.id = p.row + grid * kTok;
    p.used = p.id + grid * kTok;
    p.partial = reinterpret_cast<float*>(p.used + grid * kTok);
    p.ordered = kTT > 1 && counted;
    if constexpr (kTT > 1) {
        if (p.ordered) adapt_order<T, kTok><<<1, kOrderThreads, 0, stream>>>(p);
    }
    shrink_rank<T, false, kTT, kWaves>(p, stream);
    expand_launch<T, kTok, kTT == 1 ? 1 : 2, 4>(p, tiles, stream);
}

template <class T>
int run(const ii_adapt_args& a, hipStream_t stream) {
    Adapt<T> p = {};
    p.a = static_cast<const T*>(a.a);
    p.b = static_cast<const T*>(a.b);
    p.scales = a.scales;
    p.ranks = a.ranks;
    p.x_stride = a.m > 1 ? a.x_stride : 0;
    p.a_stride = a.count > 1 ? a.a_stride : 0;
    p.a_row = a.rank > 1 ? a.a_row_stride : 0;
    p.b_stride = a.count > 1 ? a.b_stride : 0;
    p.b_row = a.n > 1 ? a.b_row_stride : 0;
    p.base_stride = a.m > 1 ? a.base_stride : 0;
    p.out_stride = a.m > 1 ? a.out_stride : 0;
    p.n = (int32_t)a.n;
    p.k = (int32_t)a.k;
    p.rank = a.rank;
    p.count = (int32_t)a.count;
    p.rankp = (int32_t)groups(a.rank, 8) * 8;
    p.out_f32 = a.out_dtype == II_F32;
    p.base_f32 = a.base_dtype == II_F32;
    p.parts = p.out_f32 ? 3 : 2;
    p.wide = (int32_t)groups(p.parts * p.rankp, 32) * 32;
    uint64_t floats = 0;
    if (a.work_bytes > kWorkHead)
        floats = (std::min<uint64_t>(a.work_bytes, II_WORK_BYTES) - kWorkHead) / 4;
    const int64_t spare = a.count < kCounted ? a.count + 1 : 0;  // tiles that are not full
    const bool room = floats >= (uint64_t)(spare + 1) * tile_floats(p, 32);
    // (of ranks above 128 h and its parts of 32 rows pass 64 KB of LDS)
    const bool many = a.m > kGathered && (a.rank <= 128 || room);
    // rows that are gathered, or whose tiles there is room for, at once
    // (a dispatch counts its work-items in 32 bits)
    int64_t rows = std::min<int64_t>(a.m, many ? 1 << 20 : kGathered);
    if (many && room)
        rows = std::min<int64_t>(rows, (floats / tile_floats(p, 32) - spare) * 32);
    for (int64_t i = 0; i < a.m; i += rows) {
        p.m = (int32_t)std::min(rows, a.m - i);
        p.x = static_cast<const T*>(a.x) + i * p.x_stride;
        p.adapters = a.adapters + i;
        const auto at = [&](const void* from, int64_t stride, bool f32) {
            return from ? static_cast<const char*>(from) + i * stride * (f32 ? 4 : 2) : nullptr;
        };
        p.base = at(a.base, p.base_stride, p.base_f32);
        p.out = const_cast<char*>(at(a.out, p.out_stride, p.out_f32));
        if (many)
            tiles_launch<T, 2, 4>(p, static_cast<char*>(a.work), floats, stream);
        else
            tiles_launch<T, 1, 4>(p, static_cast<char*>(a.work), floats, stream);
    }
    return launched("ii_adapt");
}

int check(const ii_adapt_args& a) {
    const char* fn = "ii_adapt";
    constexpr int64_t most = INT32_MAX;
    if (!half_type(a.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, a.dtype);
    for (const int32_t t : {a.out_dtype, a.base_dtype})
        if (t != a.dtype && t != II_F32) return fail(II_EINVAL, "%s: out or base of type %d", fn, t);
    if (a.rank < 1 || a.rank > kMaxRank) return fail(II_EINVAL, "%s: rank %d", fn, a.rank);
    if (a.m < 0 || a.n < 0 || a.k < 0 || a.count < 0 || a.m > most || a.n > most || a.k > most ||
        a.count > most)
        return fail(II_EINVAL, "%s: sizes %lld, %lld, %lld, %lld adapters", fn, (long long)a.m,
                    (long long)a.n, (long long)a.k, (long long)a.count);
    if (a.x_stride < 0 || a.base_stride < 0) return fail(II_EINVAL, "%s: a stride is negative", fn);
    if (a.m > 1 && a.out_stride < a.n)
        return fail(II_EINVAL, "%s: rows of out meet (stride %lld, %lld columns)", fn,
                    (long long)a.out_stride, (long long)a.n);
    if (!a.m || !a.n) return II_OK;
    const uint64_t m = a.m, n = a.n, k = a.k, size = 2;
    const uint64_t osize = a.out_dtype == II_F32 ? 4 : 2, bsize = a.base_dtype == II_F32 ? 4 : 2;
    Rows out, scratch, r;
    uint64_t stride;
    if (__builtin_mul_overflow((uint64_t)(m > 1 ? a.out_stride : 0), osize, &stride))
        return fail(II_EOVERFLOW, "%s: the stride of out", fn);
    int rc = check_rows(fn, "out", a.out, m, n * osize, stride, osize, &out);
    if (rc || (rc = check_work(fn, a.work, a.work_bytes, &scratch)) ||
        (rc = check_apart(fn, "work", out, scratch)))
        return rc;
    // [count][rows][width] of A and of B as one range
    const auto span = [&](const char* what, const void* p, int64_t rows, int64_t width, int64_t stride,
                          int64_t row_stride) -> int {
        int64_t s, rs;
        if (__builtin_mul_overflow(stride, (int64_t)size, &s) ||
            __builtin_mul_overflow(row_stride, (int64_t)size, &rs))
            return fail(II_EOVERFLOW, "%s: the strides of %s", fn, what);
        if (!a.count || !rows || !width) return II_OK;
        const Axis axes[2] = {{a.count, s}, {rows, rs}};
        uint64_t bytes;
        if (const int rc = check_span(fn, what, axes, 2, width * size, false, &bytes)) return rc;
        if (const int rc = check_rows(fn, what, p, 1, bytes, 0, size, &r)) return rc;
        if (const int rc = check_apart(fn, what, scratch, r)) return rc;
        return check_apart(fn, what, out, r);
    };
    if ((rc = span("a", a.a, a.rank, a.k, a.a_stride, a.a_row_stride)) ||
        (rc = span("b", a.b, a.n, a.rank, a.b_stride, a.b_row_stride)))
        return rc;
    const struct {
        const char* what;
        const void* p;
        uint64_t rows, width;
        int64_t stride;
        uint64_t size;
        bool need, in_place;
    } ins[] = {{"x", a.x, m, k, a.x_stride, 2, true, false},
               {"adapters", a.adapters, 1, m, 0, 4, true, false},
               {"scales", a.scales, 1, (uint64_t)a.count, 0, 4, false, false},
               {"ranks", a.ranks, 1, (uint64_t)a.count, 0, 4, false, false},
               // each element of base is read by the lane that then writes it
               {"base", a.base, m, n, a.base_stride, bsize, false,
                a.base == a.out && osize == bsize && (m == 1 || a.base_stride == a.out_stride)}};
    for (const auto& in : ins) {
        if (!in.p && !in.need) continue;
        if (__builtin_mul_overflow((uint64_t)(in.rows > 1 ? in.stride : 0), in.size, &stride))
            return fail(II_EOVERFLOW, "%s: the stride of %s", fn, in.what);
        rc = check_rows(fn, in.what, in.p, in.rows, in.width * in.size, stride, in.size, &r);
        if (rc || (rc = check_apart(fn, in.what, scratch, r))) return rc;
        if (!in.in_place && (rc = check_apart(fn, in.what, out, r))) return rc;
    }
    return II_OK;
}

}  // namespace
}  // namespace ii

extern "C" int ii_adapt(const ii_adapt_args* a, hipStream_t stream) {
    if (!a) return ii::fail(II_EINVAL, "ii_adapt: args is NULL");
    {
        const ii::Checks checks;
        if (const int rc = ii::check(*a)) return rc;
    }
    if (!a->m || !a->n) return II_OK;
    return a->dtype == II_BF16 ? ii::run<__bf16>(*a, stream) : ii::run<_Float16>(*a, stream);
}
