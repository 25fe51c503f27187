// ii_adapt: low-rank adapters of many requests beside a shared projection,
// out[i] = base[i] + s_a B_a (A_a x[i]), a the adapter of row i.
//
// Rows of one adapter share what is read of it, so rows are taken in tiles of
// one adapter. A few rows, in any order, are gathered: the workgroup of a row
// looks whether the row is the first, the 17th, .. of its adapter, takes it and
// the next 15 if so, and ends if not. Of many rows, which come in runs, a
// workgroup takes 64 neighbours, with a pass for each adapter among them.
//
// h = A x is a sum over k that the waves of a workgroup, and workgroups, share;
// it is short, and is kept in 32 bits (in `work`, or LDS). For the product with
// B, whose matrix instruction takes 16 bits, a row of h is cut into two or three
// parts of T, the second what the first's rounding left out: 16 bits of bf16 and
// 22 of f16 in two parts, more than a result of 16 bits shows, and all 24 in
// three, for a result of 32. Parts lie behind one another as one longer sum.
// f16 has little range: rows are brought to its middle by a power of two first.
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

constexpr int kMaxRank = 256;
constexpr int kGathered = 1024;  // rows that are gathered
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
    int32_t columns;      // of out, a workgroup
    int32_t splits;       // workgroups that share k
    bool out_f32, base_f32, words, b_words, quads;
    float* h;             // [splits][m][rankp]
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

// A tile's rows and their adapters; rows past `count` have none.
template <int kTok>
struct Tile {
    int row[kTok], id[kTok];
    float factor[kTok], shrunk[kTok];  // of a result, of h before it is cut
    int count;
};

// The tile that begins with row b, false if none does. Called by all threads.
template <class T, int kTok>
__device__ inline bool gather(const Adapt<T>& p, int b, Tile<kTok>& tile) {
    const int lane = threadIdx.x % 64;
    const int mine = adapter_of(p, b);
    int id[kGathered / 64];
#pragma unroll
    for (int i = 0; i < kGathered / 64; ++i) {
        const int j = i * 64 + lane;
        id[i] = j < p.m ? adapter_of(p, j) : -2;
    }
    int before = 0, found = 0;
#pragma unroll
    for (int i = 0; i < kGathered / 64; ++i) {
        const uint64_t same = __ballot(id[i] == mine);
        const int past = min(max(b - i * 64, 0), 64);  // of this word, before b
        const uint64_t low = past == 64 ? ~0ull : (1ull << past) - 1;
        before += __popcll(same & low);
        const uint64_t rest = same & ~low;
        const int place = found + __popcll(rest & ((1ull << lane) - 1));
        if (threadIdx.x < 64 && rest >> lane & 1 && place < kTok) {
            tile.row[place] = i * 64 + lane;
            tile.id[place] = mine;
        }
        found += __popcll(rest);
    }
    if (before % kTok) return false;
    if (threadIdx.x < kTok && (int)threadIdx.x >= found) {
        tile.row[threadIdx.x] = b;
        tile.id[threadIdx.x] = -1;
    }
    if (threadIdx.x == 0) tile.count = min(found, kTok);
    __syncthreads();
    return true;
}

// Rows b kTok .. as they come.
template <class T, int kTok>
__device__ inline void neighbours(const Adapt<T>& p, int b, Tile<kTok>& tile) {
    const int64_t first = (int64_t)b * kTok;
    if (threadIdx.x < kTok) {
        const int64_t i = min(first + threadIdx.x, (int64_t)p.m - 1);
        tile.row[threadIdx.x] = (int)i;
        tile.id[threadIdx.x] = first + threadIdx.x < p.m ? adapter_of(p, i) : -1;
    }
    if (threadIdx.x == 0) tile.count = (int)min((int64_t)kTok, p.m - first);
    __syncthreads();
}

// The least adapter of the tile above a, or INT_MAX.
template <int kTok>
__device__ inline int next_adapter(const Tile<kTok>& tile, int a) {
    static_assert(kTok <= 64);
    const int id = tile.id[threadIdx.x % kTok];
    int v = id > a ? id : INT32_MAX;
#pragma unroll
    for (int d = 1; d < kTok; d *= 2) v = min(v, __shfl_xor(v, d));
    return __builtin_amdgcn_readfirstlane(v);
}

// Elements of a row from `from` on, of which `left` are there, others zero.
template <class T>
__device__ inline typename Vec<T>::x8 some(const T* from, int64_t left, bool words) {
    typename Vec<T>::x8 v = {};
    if (words && left >= 8) return *reinterpret_cast<const typename Vec<T>::x8*>(from);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) v[j] = from[j];
    return v;
}

// Rows r0 .. r0 + kR * 16 of h of the tile's rows whose adapter is a, this
// workgroup's share of k, given to keep(token, rank, value).
template <class T, int kR, int kTT, int kWaves, class Keep>
__device__ inline void shrink(const Adapt<T>& p, const Tile<kTT * 16>& tile, int a, int r0, int split,
                              float* red, Keep&& keep) {
    using x8 = typename Vec<T>::x8;
    constexpr int kSums = kR * kTT * 256;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, part = lane / 16;
    const int rank = rank_of(p, a);
    const T *ap[kR], *xp[kTT];
#pragma unroll
    for (int r = 0; r < kR; ++r)  // rows past the rank are left out below
        ap[r] = p.a + a * p.a_stride + min(r0 + r * 16 + row, max(rank - 1, 0)) * p.a_row + part * 8;
#pragma unroll
    for (int t = 0; t < kTT; ++t) xp[t] = p.x + tile.row[t * 16 + row] * p.x_stride + part * 8;
    f32x4 acc[kR][kTT] = {};
    const int units = (int)groups(p.k, kUnit), whole = p.words ? p.k / kUnit : 0;
    const int step = kWaves * p.splits;
    int u = split * kWaves + wave;
    constexpr int kAhead = kTT > 1 ? 2 : 4;
    const auto take = [&](int u, x8(&av)[2][kR], x8(&xv)[2][kTT]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t k = (int64_t)u * kUnit + h * 32;
#pragma unroll
            for (int r = 0; r < kR; ++r) av[h][r] = *reinterpret_cast<const x8*>(ap[r] + k);
#pragma unroll
            for (int t = 0; t < kTT; ++t) xv[h][t] = *reinterpret_cast<const x8*>(xp[t] + k);
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
        for (; u + (kAhead - 1) * step < whole; u += kAhead * step) {
            x8 av[kAhead][2][kR], xv[kAhead][2][kTT];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) take(u + i * step, av[i], xv[i]);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) multiply(av[i], xv[i]);
        }
        for (; u < units; u += step) {
            x8 av[2][kR], xv[2][kTT];
            if (u < whole) {
                take(u, av, xv);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t k = (int64_t)u * kUnit + h * 32, left = p.k - k - part * 8;
#pragma unroll
                    for (int r = 0; r < kR; ++r) av[h][r] = some(ap[r] + k, left, p.words);
#pragma unroll
                    for (int t = 0; t < kTT; ++t) xv[h][t] = some(xp[t] + k, left, p.words);
                }
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
    if (threadIdx.x < kTok * kLanes) {
        const int token = threadIdx.x / kLanes, id = tile.id[token];
        float up = 1, down = 1;
        if constexpr (std::is_same_v<T, _Float16>) {
            float most = 0;
            for (int r = threadIdx.x % kLanes; r < p.rankp; r += kLanes)
                most = fmaxf(most, fabsf(h[token * p.rankp + r]));
#pragma unroll
            for (int d = 1; d < kLanes; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
            // the largest to 2^12 .. 2^13
            const int e = min(max((int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127 - 12, -100), 100);
            if (most > 0) {
                up = __builtin_bit_cast(float, (uint32_t)(127 + e) << 23);
                down = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
            }
        }
        if (threadIdx.x % kLanes == 0) {
            tile.shrunk[token] = down;
            tile.factor[token] = id < 0 ? 0.0f : up * (p.scales ? p.scales[id] : 1.0f);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kTok * p.wide; e += kThreads) {
        const int token = e / p.wide, i = e % p.wide, part = i / p.rankp;
        float rest = part < p.parts ? h[token * p.rankp + i % p.rankp] * tile.shrunk[token] : 0.0f;
        T v = (T)rest;
        for (int q = 0; q < part; ++q) {
            rest -= (float)v;
            if (!(fabsf(rest) <= 3e38f)) rest = 0;  // of what is not finite nothing is left
            v = (T)rest;
        }
        parts[e] = v;
    }
    __syncthreads();
}

template <class T>
__device__ inline void put(const Adapt<T>& p, int64_t row, int64_t j, f32x4 y) {
    using x4 = typename Vec<T>::x4;
    if (p.quads && j + 4 <= p.n) {
        if (p.base && p.base_f32) {
            y += *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.base) + row * p.base_stride + j);
        } else if (p.base) {
            const x4 v = *reinterpret_cast<const x4*>(static_cast<const T*>(p.base) + row * p.base_stride + j);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] += (float)v[r];
        }
        if (p.out_f32) {
            *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + row * p.out_stride + j) = y;
        } else {
            x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = (T)y[r];
            *reinterpret_cast<x4*>(static_cast<T*>(p.out) + row * p.out_stride + j) = v;
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (j + r >= p.n) break;
        float v = y[r];
        if (p.base)
            v += p.base_f32 ? static_cast<const float*>(p.base)[row * p.base_stride + j + r]
                            : (float)static_cast<const T*>(p.base)[row * p.base_stride + j + r];
        if (p.out_f32)
            static_cast<float*>(p.out)[row * p.out_stride + j + r] = v;
        else
            static_cast<T*>(p.out)[row * p.out_stride + j + r] = (T)v;
    }
}

// Columns first .. end of the tile's rows of out, kC * 16 at a time a wave.
template <class T, int kTT, int kC, int kWaves>
__device__ inline void expand(const Adapt<T>& p, const Tile<kTT * 16>& tile, const T* parts, int64_t first,
                              int64_t end) {
    using x8 = typename Vec<T>::x8;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, part = lane / 16;
    const int steps = p.wide / 32, held = p.parts * p.rankp;
    for (int64_t n0 = first + wave * kC * 16; n0 < end; n0 += kWaves * kC * 16) {
        f32x4 total[kC][kTT] = {};
        for (int a = next_adapter(tile, -1); a != INT32_MAX; a = next_adapter(tile, a)) {
            const int rank = rank_of(p, a);
            const T* b[kC];
#pragma unroll
            for (int c = 0; c < kC; ++c)
                b[c] = p.b + a * p.b_stride + min(n0 + c * 16 + row, (int64_t)p.n - 1) * p.b_row;
            f32x4 acc[kC][kTT] = {};
            int col = part * 8;
            while (col >= p.rankp) col -= p.rankp;
            for (int s = 0; s < steps; ++s) {
                const int at = s * 32 + part * 8;
                x8 bv[kC], hv[kTT];
#pragma unroll
                for (int c = 0; c < kC; ++c)
                    bv[c] = some(b[c] + col, at < held ? rank - col : 0, p.b_words);
#pragma unroll
                for (int t = 0; t < kTT; ++t)
                    hv[t] = *reinterpret_cast<const x8*>(parts + (t * 16 + row) * p.wide + at);
#pragma unroll
                for (int c = 0; c < kC; ++c)
#pragma unroll
                    for (int t = 0; t < kTT; ++t) acc[c][t] = mfma16(bv[c], hv[t], acc[c][t]);
                col += 32;
                while (col >= p.rankp) col -= p.rankp;
            }
            // a row has one adapter; what others have there does not matter
#pragma unroll
            for (int t = 0; t < kTT; ++t)
                if (tile.id[t * 16 + row] == a)
#pragma unroll
                    for (int c = 0; c < kC; ++c) total[c][t] = acc[c][t] * tile.factor[t * 16 + row];
        }
#pragma unroll
        for (int t = 0; t < kTT; ++t)
            if (t * 16 + row < tile.count)
#pragma unroll
                for (int c = 0; c < kC; ++c)
                    put(p, tile.row[t * 16 + row], n0 + c * 16 + part * 4, total[c][t]);
    }
}

enum { kBoth, kShrink, kExpand };

// kBoth: h in LDS, formed by each of the workgroups that share a tile's columns.
// kShrink: a share of k of h, into memory. kExpand: the rest.
template <class T, int kStage, int kR, int kTT, int kWaves>
__global__ __launch_bounds__(kWaves * 64) void adapt_tiles(Adapt<T> p) {
    constexpr int kTok = kTT * 16, kThreads = kWaves * 64;
    constexpr int kRed = kStage == kExpand ? 0 : kWaves * kR * kTT * 256;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Tile<kTok> tile;
    if constexpr (kTT == 1) {
        if (!gather(p, blockIdx.x, tile)) return;
    } else {
        neighbours(p, blockIdx.x, tile);
    }
    float* red = reinterpret_cast<float*>(lds);
    float* h = red + kRed;
    if constexpr (kStage != kExpand) {
        if constexpr (kStage == kBoth)
            for (int e = threadIdx.x; e < kTok * p.rankp; e += kThreads) h[e] = 0;
        __syncthreads();
        for (int a = next_adapter(tile, -1); a != INT32_MAX; a = next_adapter(tile, a))
            for (int r0 = 0; r0 < p.rankp; r0 += kR * 16)
                shrink<T, kR, kTT, kWaves>(
                    p, tile, a, r0, kStage == kBoth ? 0 : blockIdx.y, red, [&](int token, int r, float v) {
                        if (kStage == kBoth)
                            h[token * p.rankp + r] = v;
                        else
                            p.h[((int64_t)blockIdx.y * p.m + tile.row[token]) * p.rankp + r] = v;
                    });
    } else {
        for (int e = threadIdx.x; e < kTok * p.rankp; e += kThreads) {
            const int token = e / p.rankp, r = e % p.rankp;
            float v = 0;
            if (tile.id[token] >= 0)
                for (int s = 0; s < p.splits; ++s)
                    v += p.h[((int64_t)s * p.m + tile.row[token]) * p.rankp + r];
            h[e] = v;
        }
        __syncthreads();
    }
    if constexpr (kStage != kShrink) {
        T* parts = reinterpret_cast<T*>(h + kTok * p.rankp);
        cut<T, kTok, kThreads>(p, tile, h, parts);
        const int64_t first = (int64_t)blockIdx.y * p.columns;
        expand<T, kTT, kTT == 1 ? 4 : 2, kWaves>(p, tile, parts, first, min(first + p.columns, (int64_t)p.n));
    }
}

template <class T, int kStage, int kR, int kTT, int kWaves>
void stage_launch(Adapt<T> p, uint32_t tiles, uint32_t shares, hipStream_t stream) {
    constexpr int kTok = kTT * 16;
    uint32_t lds = kStage == kExpand ? 0 : kWaves * kR * kTT * 1024;
    if (kStage != kShrink) lds += kTok * (p.rankp * 4 + p.wide * 2);
    // more than 64 KB has to be asked for
    static const hipError_t ready = hipFuncSetAttribute(
        reinterpret_cast<const void*>(&adapt_tiles<T, kStage, kR, kTT, kWaves>),
        hipFuncAttributeMaxDynamicSharedMemorySize, 150 * 1024);
    (void)ready;
    adapt_tiles<T, kStage, kR, kTT, kWaves><<<dim3(tiles, shares), kWaves * 64, lds, stream>>>(p);
}

template <class T, int kStage, int kTT, int kWaves>
void rank_launch(const Adapt<T>& p, uint32_t tiles, uint32_t shares, hipStream_t stream) {
    if (kStage == kExpand || p.rankp <= 16)
        stage_launch<T, kStage, 1, kTT, kWaves>(p, tiles, shares, stream);
    else if (p.rankp <= 32)
        stage_launch<T, kStage, 2, kTT, kWaves>(p, tiles, shares, stream);
    else
        stage_launch<T, kStage, 4, kTT, kWaves>(p, tiles, shares, stream);
}

// Rows [0, p.m) of a call, in tiles of kTT * 16; floats: the room for h.
template <class T, int kTT, int kWaves>
void tiles_launch(Adapt<T> p, uint64_t floats, hipStream_t stream) {
    constexpr int kTok = kTT * 16;
    const uint32_t grid = (uint32_t)(kTT == 1 ? p.m : groups(p.m, kTok));  // some end at once
    const int64_t tiles = groups(p.m, kTok);
    // columns a workgroup: enough workgroups to fill the card
    constexpr int kCols = kWaves * (kTT == 1 ? 4 : 2) * 16;
    const int64_t shares = std::min(groups(p.n, kCols), std::max<int64_t>(1, 1024 / tiles));
    p.columns = (int32_t)(groups(groups(p.n, shares), kCols) * kCols);
    const uint32_t by = (uint32_t)groups(p.n, p.columns);
    const int64_t units = groups(p.k, kUnit);
    p.splits = (int32_t)std::max<int64_t>(
        1, std::min({512 / tiles, units / (2 * kWaves), (int64_t)(floats / ((uint64_t)p.m * p.rankp))}));
    if (floats < (uint64_t)p.m * p.rankp) {
        p.splits = 1;
        rank_launch<T, kBoth, kTT, kWaves>(p, grid, by, stream);
    } else {
        rank_launch<T, kShrink, kTT, kWaves>(p, grid, p.splits, stream);
        rank_launch<T, kExpand, kTT, kWaves>(p, grid, by, stream);
    }
}

template <class T>
int run(const ii_adapt_args& a, hipStream_t stream) {
    Adapt<T> p = {};
    const bool many = a.m > kGathered && a.rank <= 128;
    const auto words = [](const void* at, int64_t s) {
        return reinterpret_cast<uintptr_t>(at) % 16 == 0 && s % 8 == 0;
    };
    const auto quad = [](const void* at, int64_t s, int size) {
        return !at || (reinterpret_cast<uintptr_t>(at) % (4 * size) == 0 && s % 4 == 0);
    };
    p.a = static_cast<const T*>(a.a);
    p.b = static_cast<const T*>(a.b);
    p.scales = a.scales;
    p.ranks = a.ranks;
    // strides of axes of one place say nothing of how they can be read
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
    p.words = a.k % 8 == 0 && words(a.x, p.x_stride) && words(a.a, p.a_stride) && words(a.a, p.a_row);
    p.b_words = words(a.b, p.b_stride) && words(a.b, p.b_row);
    p.quads = quad(a.out, p.out_stride, p.out_f32 ? 4 : 2) && quad(a.base, p.base_stride, p.base_f32 ? 4 : 2);
    uint64_t floats = 0;
    if (a.work_bytes > kWorkHead) {
        p.h = reinterpret_cast<float*>(static_cast<char*>(a.work) + kWorkHead);
        floats = (std::min<uint64_t>(a.work_bytes, II_WORK_BYTES) - kWorkHead) / 4;
    }
    // rows that are gathered, or whose h there is room for, at once
    int64_t rows = many ? a.m : std::min<int64_t>(a.m, kGathered);
    if (many && floats >= (uint64_t)64 * p.rankp)
        rows = std::min<int64_t>(rows, floats / p.rankp / 64 * 64);
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
            tiles_launch<T, 4, 4>(p, floats, stream);
        else
            tiles_launch<T, 1, 8>(p, floats, stream);
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
        bool need;
    } ins[] = {{"x", a.x, m, k, a.x_stride, 2, true},
               {"adapters", a.adapters, 1, m, 0, 4, true},
               {"scales", a.scales, 1, (uint64_t)a.count, 0, 4, false},
               {"ranks", a.ranks, 1, (uint64_t)a.count, 0, 4, false},
               {"base", a.base, m, n, a.base_stride, bsize, false}};
    for (const auto& in : ins) {
        if (!in.p && !in.need) continue;
        if (__builtin_mul_overflow((uint64_t)(in.rows > 1 ? in.stride : 0), in.size, &stride))
            return fail(II_EOVERFLOW, "%s: the stride of %s", fn, in.what);
        rc = check_rows(fn, in.what, in.p, in.rows, in.width * in.size, stride, in.size, &r);
        if (rc || (rc = check_apart(fn, in.what, scratch, r))) return rc;
        // each element of base is read by the lane that then writes it
        if (in.p == a.base && in.p == a.out && osize == bsize && (m == 1 || a.base_stride == a.out_stride))
            continue;
        if ((rc = check_apart(fn, in.what, out, r))) return rc;
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
