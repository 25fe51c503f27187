// ii_linear: products with weight matrices, and their epilogue.
#include <algorithm>

#include "ops.h"
#include "ops_device.h"

namespace ii {
namespace {

template <class T>
struct Linear {
    const T *x, *w, *w2, *bias, *bias2, *residual;
    void* out;
    int64_t x_stride, w_stride, w2_stride, residual_stride, out_stride;
    int32_t m, n, k, act;
    bool out_f32;
};

__device__ inline float activate(float y, int act) {
    switch (act) {
    case II_ACT_RELU: return y < 0 ? 0.0f : y;  // NaN stays
    case II_ACT_SILU: return y / (1.0f + expf(-y));
    case II_ACT_GELU: return 0.5f * y * (1.0f + erff(y * 0.70710678118654752f));
    }
    return y;
}

template <class T, bool kGated>
__device__ inline void put(const Linear<T>& p, int64_t i, int64_t j, float y, float z) {
    if (p.bias) y += (float)p.bias[j];
    y = activate(y, p.act);
    if (kGated) {
        if (p.bias2) z += (float)p.bias2[j];
        y *= z;
    }
    if (p.residual) y += (float)p.residual[i * p.residual_stride + j];
    if (p.out_f32)
        static_cast<float*>(p.out)[i * p.out_stride + j] = y;
    else
        static_cast<T*>(p.out)[i * p.out_stride + j] = (T)y;
}

// 64 tokens by 64 weight rows a workgroup of four waves, 32 elements of k at
// a time through LDS, every element loaded by itself: rows at any address.
constexpr int kElemTile = 64, kElemK = 32, kElemPad = 8;

template <class T>
__device__ inline void stage_elements(T (*to)[kElemK + kElemPad], const T* from, int64_t stride,
                                      int64_t row0, int64_t rows, int64_t k0, int64_t k) {
    const int t = threadIdx.x, r = t / 4, c = t % 4 * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        T v = (T)0.0f;
        if (row0 + r < rows && k0 + c + j < k) v = from[(row0 + r) * stride + k0 + c + j];
        to[r][c + j] = v;
    }
}

template <class T, bool kGated>
__global__ __launch_bounds__(256) void linear_elements(Linear<T> p) {
    using x8 = typename Vec<T>::x8;
    __shared__ T xs[kElemTile][kElemK + kElemPad];
    __shared__ T ws[kGated ? 2 : 1][kElemTile][kElemK + kElemPad];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, part = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * kElemTile, m0 = (int64_t)blockIdx.y * kElemTile;
    f32x4 acc[kGated ? 2 : 1][4] = {};
    for (int64_t k0 = 0; k0 < p.k; k0 += kElemK) {
        stage_elements(xs, p.x, p.x_stride, m0, p.m, k0, p.k);
        stage_elements(ws[0], p.w, p.w_stride, n0, p.n, k0, p.k);
        if (kGated) stage_elements(ws[kGated], p.w2, p.w2_stride, n0, p.n, k0, p.k);
        __syncthreads();
#pragma unroll
        for (int g = 0; g <= (kGated ? 1 : 0); ++g) {
            const x8 a = *reinterpret_cast<const x8*>(&ws[g][wave * 16 + row][part * 8]);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                acc[g][t] = mfma16(a, *reinterpret_cast<const x8*>(&xs[t * 16 + row][part * 8]),
                                   acc[g][t]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t i = m0 + t * 16 + row, j = n0 + wave * 16 + part * 4 + r;
            if (i < p.m && j < p.n) put<T, kGated>(p, i, j, acc[0][t][r], acc[kGated][t][r]);
        }
}

// Few tokens: the weights are read once, straight into the matrix
// instructions' registers, by as many waves as it takes to keep the memory
// busy. A workgroup owns kRows * 16 weight rows (with a gate: 16 of w, 16 of
// w2); its kWaves waves take units of 64 elements of k (a 128-byte line of
// each row) in turn, gridDim.y workgroups share a long k. Waves join their
// sums in LDS in the order of the waves; workgroups leave theirs in `work`,
// and the last to arrive adds them in the order of their places.
constexpr int kUnit = 64;  // elements of k a wave takes at once

template <class T, bool kGated, int kRows, int kTokens, int kWaves, int kAhead>
__global__ __launch_bounds__(kWaves * 64) void linear_stream(Linear<T> p, uint32_t* counters,
                                                             float* partial) {
    using x8 = typename Vec<T>::x8;
    constexpr int kSets = kGated ? 2 : 1, kMine = kRows * 16 / kSets;  // rows of each matrix
    constexpr int kSums = kRows * kTokens * 256;
    __shared__ float red[kWaves * kSums];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, part = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * kMine;
    const int units = (p.k + kUnit - 1) / kUnit, whole = p.k / kUnit;

    const T* wp[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int64_t j = min(n0 + (kGated ? 0 : r * 16) + row, (int64_t)p.n - 1);
        wp[r] = (kGated && r ? p.w2 + j * p.w2_stride : p.w + j * p.w_stride) + part * 8;
    }
    const T* xp[kTokens];
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
        xp[t] = p.x + (int64_t)min(t * 16 + row, p.m - 1) * p.x_stride + part * 8;

    f32x4 acc[kRows][kTokens] = {};
    auto load = [&](const T* from, int u, int h) {
        const int64_t k = (int64_t)u * kUnit + h * 32;
        return *reinterpret_cast<const x8*>(from + k);
    };
    const int step = kWaves * gridDim.y;
    int u = blockIdx.y * kWaves + wave;
    for (; u + (kAhead - 1) * step < whole; u += kAhead * step) {
        x8 a[kAhead][2][kRows], b[kAhead][2][kTokens];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) a[i][h][r] = load(wp[r], u + i * step, h);
#pragma unroll
                for (int t = 0; t < kTokens; ++t) b[i][h][t] = load(xp[t], u + i * step, h);
            }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < kRows; ++r)
#pragma unroll
                    for (int t = 0; t < kTokens; ++t)
                        acc[r][t] = mfma16(a[i][h][r], b[i][h][t], acc[r][t]);
    }
    for (; u < units; u += step)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool in = (int64_t)u * kUnit + h * 32 + part * 8 < p.k;  // k is whole words
            x8 a[kRows] = {}, b[kTokens] = {};
            if (in) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) a[r] = load(wp[r], u, h);
#pragma unroll
                for (int t = 0; t < kTokens; ++t) b[t] = load(xp[t], u, h);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int t = 0; t < kTokens; ++t) acc[r][t] = mfma16(a[r], b[t], acc[r][t]);
        }

    // red[wave][r][t][token][weight row]
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int t = 0; t < kTokens; ++t)
            *reinterpret_cast<f32x4*>(&red[wave * kSums + ((r * kTokens + t) * 16 + row) * 16 +
                                           part * 4]) = acc[r][t];
    __syncthreads();
    // every thread joins the same places below, so the sums stay in red[0..]
    for (int e = threadIdx.x; e < kSums; e += kWaves * 64) {
        float s = red[e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += red[w * kSums + e];
        red[e] = s;
    }
    if (gridDim.y > 1) {
        float* mine = partial + ((int64_t)blockIdx.x * gridDim.y + blockIdx.y) * kSums;
        for (int e = threadIdx.x; e < kSums; e += kWaves * 64) leave_part(&mine[e], red[e]);
        if (!arrive_last(&counters[blockIdx.x], gridDim.y)) return;
        const float* all = partial + (int64_t)blockIdx.x * gridDim.y * kSums;
        for (int e = threadIdx.x; e < kSums; e += kWaves * 64) {
            float s = 0;
            for (uint32_t y = 0; y < gridDim.y; ++y) s += take_part(&all[(int64_t)y * kSums + e]);
            red[e] = s;
        }
    }
    // with a gate a thread's y and z lie kSums / 2 apart: another thread's sums
    if (kGated) __syncthreads();
    for (int e = threadIdx.x; e < kSums / kSets; e += kWaves * 64) {
        const int r = e / (kTokens * 256), i = e / 16 % (kTokens * 16);
        const int64_t j = n0 + r * 16 + e % 16;
        if (i < p.m && j < p.n)
            put<T, kGated>(p, i, j, red[e], kGated ? red[e + kSums / 2] : 0.0f);
    }
}

// Some tokens: as above, but rows of x go through LDS, where the kRowWaves
// waves of a k group share them; each wave owns 16 weight rows (with a gate 16
// of w and 16 of w2), kKGroups groups of waves and gridDim.y workgroups share
// k. Weights are requested two chunks ahead of their use, x one.
constexpr int kChunkPad = 8;         // LDS rows 16 bytes apart in banks

// elements of k a group takes at once
constexpr int shared_chunk(bool gated) { return gated ? 64 : 128; }

template <class T, bool kGated, int kTokens, int kRowWaves, int kKGroups>
__global__ __launch_bounds__(kRowWaves * kKGroups * 64) void linear_shared(Linear<T> p,
                                                                           uint32_t* counters,
                                                                           float* partial) {
    using x8 = typename Vec<T>::x8;
    constexpr int kRows = kGated ? 2 : 1, kRing = 3;
    constexpr int kChunk = shared_chunk(kGated), kSteps = kChunk / 32;
    constexpr int kGroup = kRowWaves * 64, kThreads = kGroup * kKGroups;
    constexpr int kXAll = kTokens * 16 * (kChunk / 8), kXWords = (kXAll + kGroup - 1) / kGroup;
    static_assert(kXAll % kGroup == 0 || kXWords == 1);
    constexpr int kSums = kRows * kTokens * 256;  // of a wave
    constexpr int kXs = kTokens * 16 * (kChunk + kChunkPad);
    constexpr int kBytes = std::max(2 * kKGroups * kXs * 2, kRowWaves * kKGroups * kSums * 4);
    __shared__ __attribute__((aligned(16))) char lds[kBytes];
    T(*xs)[kKGroups][kXs] = reinterpret_cast<T(*)[kKGroups][kXs]>(lds);
    float* red = reinterpret_cast<float*>(lds);

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, part = lane / 16;
    const int rw = wave % kRowWaves, kg = wave / kRowWaves, in_group = threadIdx.x % kGroup;
    const int64_t n0 = (int64_t)blockIdx.x * (kRowWaves * 16) + rw * 16;
    const int chunks = (p.k + kChunk - 1) / kChunk;
    const int step = kKGroups * gridDim.y, c0 = blockIdx.y * kKGroups + kg;
    const int rounds = (chunks + step - 1) / step;  // alike in every wave

    const int64_t wj = min(n0 + row, (int64_t)p.n - 1);
    const T* wp[kRows];
    wp[0] = p.w + wj * p.w_stride + part * 8;
    if (kGated) wp[kRows - 1] = p.w2 + wj * p.w2_stride + part * 8;
    const int xrow = in_group / (kChunk / 8), xword = in_group % (kChunk / 8);
    constexpr int kXRows = kGroup / (kChunk / 8);  // rows a pass of the group covers
    const T* xp[kXWords];
#pragma unroll
    for (int i = 0; i < kXWords; ++i)
        xp[i] = p.x + (int64_t)min(xrow + i * kXRows, p.m - 1) * p.x_stride + xword * 8;

    x8 a[kRing][kRows][kSteps], xr[kXWords];
    f32x4 acc[kRows][kTokens] = {};
    auto fetch_w = [&](int round, x8(&to)[kRows][kSteps]) {
        const int64_t k = (int64_t)(c0 + round * step) * kChunk;
        if (k + kChunk <= p.k) {
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
                    to[r][s] = *reinterpret_cast<const x8*>(wp[r] + k + s * 32);
        } else {
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    to[r][s] = x8{};
                    if (k + s * 32 + part * 8 < p.k)
                        to[r][s] = *reinterpret_cast<const x8*>(wp[r] + k + s * 32);
                }
        }
    };
    auto fetch_x = [&](int round) {
        const int64_t k = (int64_t)(c0 + round * step) * kChunk;
#pragma unroll
        for (int i = 0; i < kXWords; ++i) {
            xr[i] = x8{};
            if (in_group < kXAll && k + xword * 8 < p.k) xr[i] = *reinterpret_cast<const x8*>(xp[i] + k);
        }
    };
    auto keep_x = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kXWords; ++i)
            if (in_group < kXAll) *reinterpret_cast<x8*>(
                &xs[buf][kg][(xrow + i * kXRows) * (kChunk + kChunkPad) + xword * 8]) = xr[i];
    };

    fetch_x(0);
    fetch_w(0, a[0]);
    if (rounds > 1) fetch_w(1, a[1]);
    keep_x(0);
    __syncthreads();
    for (int base = 0; base < rounds; base += kRing * 2) {
#pragma unroll
        for (int i = 0; i < kRing * 2; ++i) {
            const int round = base + i;
            if (round < rounds) {
                if (round + 1 < rounds) fetch_x(round + 1);
                if (round + 2 < rounds) fetch_w(round + 2, a[(i + 2) % kRing]);
                const T* x = &xs[i % 2][kg][row * (kChunk + kChunkPad) + part * 8];
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
#pragma unroll
                    for (int t = 0; t < kTokens; ++t) {
                        const x8 b = *reinterpret_cast<const x8*>(
                            x + t * 16 * (kChunk + kChunkPad) + s * 32);
#pragma unroll
                        for (int r = 0; r < kRows; ++r)
                            acc[r][t] = mfma16(a[i % kRing][r][s], b, acc[r][t]);
                    }
                if (round + 1 < rounds) keep_x((i + 1) % 2);
                __syncthreads();
            }
        }
    }

    // red[k group][row wave][r][t][token][weight row]
    constexpr int kAll = kRowWaves * kSums;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int t = 0; t < kTokens; ++t)
            *reinterpret_cast<f32x4*>(
                &red[wave * kSums + ((r * kTokens + t) * 16 + row) * 16 + part * 4]) = acc[r][t];
    __syncthreads();
    if (kKGroups > 1)
        for (int e = threadIdx.x; e < kAll; e += kThreads) {
            float s = red[e];
#pragma unroll
            for (int g = 1; g < kKGroups; ++g) s += red[g * kAll + e];
            red[e] = s;
        }
    if (gridDim.y > 1) {
        float* mine = partial + ((int64_t)blockIdx.x * gridDim.y + blockIdx.y) * kAll;
        for (int e = threadIdx.x; e < kAll; e += kThreads) leave_part(&mine[e], red[e]);
        if (!arrive_last(&counters[blockIdx.x], gridDim.y)) return;
        const float* all = partial + (int64_t)blockIdx.x * gridDim.y * kAll;
        for (int e = threadIdx.x; e < kAll; e += kThreads) {
            float s = 0;
            for (uint32_t y = 0; y < gridDim.y; ++y) s += take_part(&all[(int64_t)y * kAll + e]);
            red[e] = s;
        }
    }
    __syncthreads();
    // lanes along a token's columns
    constexpr int kCols = kRowWaves * 16, kOut = kCols * kTokens * 16;
    for (int e = threadIdx.x; e < kOut; e += kThreads) {
        const int i = e / kCols, c = e % kCols;
        const int64_t j = (int64_t)blockIdx.x * kCols + c;
        const int at = c / 16 * kSums + (i / 16 * 16 + i % 16) * 16 + c % 16;
        if (i < p.m && j < p.n)
            put<T, kGated>(p, i, j, red[at], kGated ? red[at + kSums / 2] : 0.0f);
    }
}

// Many tokens: 256 tokens by 256 weight rows (with a gate 128 of w and 128 of
// w2, in turn by 16) a workgroup of eight waves, each 128 tokens by 64 rows.
// Both operands go from memory straight into LDS, 64 elements of k at a time,
// the next ones while these are multiplied. An LDS row is 128 bytes, its
// 16-byte words exchanged by the row's last three bits, so that the eight
// lanes of one LDS cycle, a row each, meet all banks.
constexpr int kTile = 256, kTileK = 64, kTileWaves = 8;

using Rsrc = __amdgpu_buffer_rsrc_t;

__device__ inline Rsrc rows_rsrc(const void* base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0,
                                             (int)(uint32_t)min(bytes, (int64_t)0xffffffffll),
                                             0x00020000);
}

template <class T, bool kGated>
__global__ __launch_bounds__(kTileWaves * 64) void linear_tile(Linear<T> p, int tiles_m,
                                                               int tiles_n) {
    using x8 = typename Vec<T>::x8;
    __shared__ __attribute__((aligned(1024))) T ws0[kTile * kTileK];
    __shared__ __attribute__((aligned(1024))) T ws1[kTile * kTileK];
    __shared__ __attribute__((aligned(1024))) T xs0[kTile * kTileK];
    __shared__ __attribute__((aligned(1024))) T xs1[kTile * kTileK];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int row = lane % 16, part = lane / 16;

    // workgroups go to the 8 XCDs in turn: each XCD gets a run of tiles, in
    // bands of 4 tiles of tokens, so that the tiles its L2 serves at one time
    // share rows
    const int total = tiles_m * tiles_n, xcd = blockIdx.x % 8, place = blockIdx.x / 8;
    const int tile = xcd * (total / 8) + min(xcd, total % 8) + place;
    constexpr int kBand = 4;
    const int band = tile / (kBand * tiles_n), in_band = tile % (kBand * tiles_n);
    const int high = min(kBand, tiles_m - band * kBand);
    const int tm = band * kBand + in_band % high, tn = in_band / high;

    constexpr int kCols = kGated ? kTile / 2 : kTile;  // columns of out
    const int64_t m0 = (int64_t)tm * kTile, n0 = (int64_t)tn * kCols;

    // what this wave brings: 32 rows of each operand, 8 rows an instruction
    const int64_t n_end = p.n - 1 - n0, m_end = p.m - 1 - m0;
    const Rsrc wr = rows_rsrc(p.w + n0 * p.w_stride, (n_end * p.w_stride + p.k) * 2);
    const Rsrc w2r = kGated ? rows_rsrc(p.w2 + n0 * p.w2_stride, (n_end * p.w2_stride + p.k) * 2) : wr;
    const Rsrc xr = rows_rsrc(p.x + m0 * p.x_stride, (m_end * p.x_stride + p.k) * 2);
    int woff[4], xoff[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = wave * 32 + i * 8 + lane / 8, word = (lane % 8) ^ (r % 8);
        const int64_t c = kGated ? r / 32 * 16 + r % 16 : r;
        const int64_t stride = kGated && i >= 2 ? p.w2_stride : p.w_stride;
        woff[i] = (int)((min(c, n_end) * stride + word * 8) * 2);
        xoff[i] = (int)((min((int64_t)r, m_end) * p.x_stride + word * 8) * 2);
    }
    auto bring = [&](int k, T* ws, T* xs) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                kGated && i >= 2 ? w2r : wr,
                (__attribute__((address_space(3))) void*)(ws + (wave * 32 + i * 8) * kTileK), 16,
                woff[i], k * 2, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                xr, (__attribute__((address_space(3))) void*)(xs + (wave * 32 + i * 8) * kTileK), 16,
                xoff[i], k * 2, 0, 0);
        }
    };
    const int wn = wave % 4 * 64, wm = wave / 4 * 128;
    f32x4 acc[4][8] = {};
    auto multiply = [&](const T* ws, const T* xs) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            x8 a[4], b[8];
            const int word = ((s * 4 + part) ^ (row % 8)) * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[i] = *reinterpret_cast<const x8*>(ws + (wn + i * 16 + row) * kTileK + word);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                b[j] = *reinterpret_cast<const x8*>(xs + (wm + j * 16 + row) * kTileK + word);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] = mfma16(a[i], b[j], acc[i][j]);
        }
    };
    const int steps = p.k / kTileK;
    if (steps > 0) bring(0, ws0, xs0);
    for (int t = 0; t < steps; t += 2) {
        __syncthreads();
        if (t + 1 < steps) bring((t + 1) * kTileK, ws1, xs1);
        multiply(ws0, xs0);
        if (t + 1 < steps) {
            __syncthreads();
            if (t + 2 < steps) bring((t + 2) * kTileK, ws0, xs0);
            multiply(ws1, xs1);
        }
    }
    if (p.k % kTileK) {  // the rest of k: words past it are zero
        __syncthreads();
        const int k0 = steps * kTileK;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = wave * 32 + i * 8 + lane / 8, word = (lane % 8) ^ (r % 8);
            const bool in = k0 + word * 8 < p.k;
            const char* w = reinterpret_cast<const char*>(kGated && i >= 2 ? p.w2 + n0 * p.w2_stride
                                                                           : p.w + n0 * p.w_stride);
            const char* x = reinterpret_cast<const char*>(p.x + m0 * p.x_stride);
            x8 a = {}, b = {};
            if (in) {
                a = *reinterpret_cast<const x8*>(w + (uint32_t)woff[i] + (int64_t)k0 * 2);
                b = *reinterpret_cast<const x8*>(x + (uint32_t)xoff[i] + (int64_t)k0 * 2);
            }
            *reinterpret_cast<x8*>(ws0 + r * kTileK + lane % 8 * 8) = a;
            *reinterpret_cast<x8*>(xs0 + r * kTileK + lane % 8 * 8) = b;
        }
        __syncthreads();
        multiply(ws0, xs0);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; i += kGated ? 2 : 1)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t at = m0 + wm + j * 16 + row;
                const int64_t c = n0 + (kGated ? (wn + i * 16) / 2 : wn + i * 16) + part * 4 + r;
                if (at < p.m && c < p.n)
                    put<T, kGated>(p, at, c, acc[i][j][r], acc[kGated ? i + 1 : i][j][r]);
            }
}

struct Work {
    uint32_t* counters = nullptr;
    float* partial = nullptr;
    uint64_t floats = 0;
};

template <class T, bool kGated, int kRows, int kTokens, int kWaves, int kAhead>
void stream_launch(const Linear<T>& p, const Work& work, hipStream_t stream) {
    constexpr int kMine = kRows * 16 / (kGated ? 2 : 1);
    constexpr uint64_t kSums = kRows * kTokens * 256;
    const uint32_t tiles = (p.n + kMine - 1) / kMine;
    const int units = (p.k + kUnit - 1) / kUnit;
    // workgroups that share a tile's k: to fill the compute units, each wave
    // left with two rounds of loads or more
    uint32_t split = 1;
    if (work.partial && tiles <= kWorkCounters && tiles < 256)
        split = std::min<uint32_t>(std::max(1, units / (kWaves * kAhead * 2)), 512 / tiles);
    while (split > 1 && tiles * split * kSums > work.floats) --split;
    linear_stream<T, kGated, kRows, kTokens, kWaves, kAhead>
        <<<dim3(tiles, split), kWaves * 64, 0, stream>>>(p, work.counters, work.partial);
}

template <class T, bool kGated, int kRows, int kTokens, int kAhead>
void stream_waves(const Linear<T>& p, const Work& work, hipStream_t stream) {
    const int64_t tiles = (p.n + 15) / 16, units = (p.k + kUnit - 1) / kUnit;
    if (tiles <= 512 && units >= 32)
        stream_launch<T, kGated, kRows, kTokens, kTokens < 4 ? 16 : 8, kAhead>(p, work, stream);
    else if (tiles <= 2048 && units >= 16)
        stream_launch<T, kGated, kRows, kTokens, 8, kAhead>(p, work, stream);
    else
        stream_launch<T, kGated, kRows, kTokens, 4, kAhead>(p, work, stream);
}

template <class T, bool kGated, int kTokens, int kRowWaves, int kKGroups>
void shared_launch(const Linear<T>& p, const Work& work, hipStream_t stream) {
    constexpr int kCols = kRowWaves * 16;
    constexpr uint64_t kAll = (uint64_t)kCols * kTokens * 16 * (kGated ? 2 : 1);
    const uint32_t tiles = (p.n + kCols - 1) / kCols;
    const uint32_t chunks = (p.k + shared_chunk(kGated) - 1) / shared_chunk(kGated);
    // as many workgroups as compute units, each wave with a chunk or more
    uint32_t split = 1;
    if (work.partial && tiles < 256)
        split = std::max(1u, std::min(256 / tiles, (chunks + kKGroups - 1) / kKGroups));
    while (split > 1 && tiles * split * kAll > work.floats) --split;
    linear_shared<T, kGated, kTokens, kRowWaves, kKGroups>
        <<<dim3(tiles, split), kRowWaves * kKGroups * 64, 0, stream>>>(p, work.counters,
                                                                       work.partial);
}

// A workgroup a compute unit with all the waves it takes, or two of half as
// many where there are rows enough. Measured at 24 x 4096 x 14336 (256
// workgroups in all): 16 waves by 32 rows 30.7 us, by 64 rows 31.4, 8 waves by
// 32 rows and twice the workgroups 34.5; at 8 x 128256 x 4096: 8 waves by 64
// rows 191 us, 16 waves 215, 4 waves 202; with a gate at 24 x 14336 x 4096: 8
// waves by 32 rows 52.6 us, by 64 rows 58.8, 16 waves by 64 rows 57.0.
template <class T, bool kGated, int kTokens>
void shared_groups(const Linear<T>& p, const Work& work, hipStream_t stream) {
    if constexpr (kTokens <= 2) {
        if ((p.n + 31) / 32 <= 256)
            return shared_launch<T, kGated, kTokens, 2, 8>(p, work, stream);
    }
    if constexpr (kTokens <= 4) {
        if ((p.n + 63) / 64 <= (kGated ? 128 : 256))
            return shared_launch<T, kGated, kTokens, 4, 4>(p, work, stream);
    }
    if constexpr (kGated && kTokens <= 2)
        shared_launch<T, kGated, kTokens, 2, 4>(p, work, stream);
    else
        shared_launch<T, kGated, kTokens, 4, 2>(p, work, stream);
}

// Whether rows can be read in 16-byte words.
bool words(const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0;
}

template <class T, bool kGated>
void launch(const Linear<T>& p, const Work& work, hipStream_t stream) {
    const bool wide = p.k > 0 && p.k % 8 == 0 && words(p.x, p.x_stride) && words(p.w, p.w_stride) &&
                      (!p.w2 || words(p.w2, p.w2_stride));
    // rows of x that the waves' own loads find in the caches: 1 x 4096 x 14336
    // 25.0 us against 28.1 through LDS, 1 x 128256 x 4096 177 against 186; from
    // 8 tokens on it is 29.2 against 27.4, 212 against 191
    if (wide && p.m <= 4) return stream_waves<T, kGated, kGated ? 2 : 1, 1, 4>(p, work, stream);
    if (wide && p.m <= 16) return shared_groups<T, kGated, 1>(p, work, stream);
    if (wide && p.m <= 32) return shared_groups<T, kGated, 2>(p, work, stream);
    if (wide && p.m <= 64) return shared_groups<T, kGated, 4>(p, work, stream);
    if (wide && p.m <= 128) return shared_groups<T, kGated, 8>(p, work, stream);
    // a tile's rows are addressed in 32 bits
    const bool near = std::max({p.x_stride, p.w_stride, p.w2_stride}) < (1 << 21);
    if (wide && near) {
        const int cols = kGated ? kTile / 2 : kTile;
        const int tm = (p.m + kTile - 1) / kTile, tn = (p.n + cols - 1) / cols;
        linear_tile<T, kGated><<<tm * tn, kTileWaves * 64, 0, stream>>>(p, tm, tn);
        return;
    }
    const dim3 grid((p.n + kElemTile - 1) / kElemTile, (p.m + kElemTile - 1) / kElemTile);
    linear_elements<T, kGated><<<grid, 256, 0, stream>>>(p);
}

template <class T>
int run(const ii_linear_args& a, hipStream_t stream) {
    Linear<T> p;
    p.x = static_cast<const T*>(a.x);
    p.w = static_cast<const T*>(a.w);
    p.w2 = static_cast<const T*>(a.w2);
    p.bias = static_cast<const T*>(a.bias);
    p.bias2 = static_cast<const T*>(a.bias2);
    p.residual = static_cast<const T*>(a.residual);
    p.out = a.out;
    p.x_stride = a.x_stride;
    p.w_stride = a.w_stride;
    p.w2_stride = a.w2_stride;
    p.residual_stride = a.residual_stride;
    p.out_stride = a.out_stride;
    p.m = (int32_t)a.m;
    p.n = (int32_t)a.n;
    p.k = (int32_t)a.k;
    p.act = a.act;
    p.out_f32 = a.out_dtype == II_F32;
    Work work;
    if (a.work_bytes > kWorkHead) {
        work.counters = static_cast<uint32_t*>(a.work);
        work.partial = reinterpret_cast<float*>(static_cast<char*>(a.work) + kWorkHead);
        work.floats = (a.work_bytes - kWorkHead) / 4;
    }
    if (p.w2)
        launch<T, true>(p, work, stream);
    else
        launch<T, false>(p, work, stream);
    return launched("ii_linear");
}

int check(const ii_linear_args& a) {
    const char* fn = "ii_linear";
    constexpr int64_t most = INT32_MAX;
    if (!half_type(a.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, a.dtype);
    if (a.out_dtype != a.dtype && a.out_dtype != II_F32)
        return fail(II_EINVAL, "%s: out_dtype %d", fn, a.out_dtype);
    if (a.act < II_ACT_NONE || a.act > II_ACT_GELU)
        return fail(II_EINVAL, "%s: act %d", fn, a.act);
    if (a.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, a.reserved);
    if (a.m < 0 || a.n < 0 || a.k < 0 || a.m > most || a.n > most || a.k > most)
        return fail(II_EINVAL, "%s: sizes %lld, %lld, %lld", fn, (long long)a.m, (long long)a.n,
                    (long long)a.k);
    if (a.bias2 && !a.w2) return fail(II_EINVAL, "%s: bias2 without w2", fn);
    if (a.x_stride < 0 || a.w_stride < 0 || a.w2_stride < 0 || a.residual_stride < 0)
        return fail(II_EINVAL, "%s: a stride is negative", fn);
    if (a.m > 1 && a.out_stride < a.n)
        return fail(II_EINVAL, "%s: rows of out meet (stride %lld, %lld columns)", fn,
                    (long long)a.out_stride, (long long)a.n);
    if (!a.m || !a.n) return II_OK;
    const uint64_t m = a.m, n = a.n, k = a.k, size = 2, osize = a.out_dtype == II_F32 ? 4 : 2;
    Rows out, r;
    int rc = check_rows(fn, "out", a.out, m, n * osize, (m > 1 ? a.out_stride : 0) * osize, osize,
                        &out);
    if (rc) return rc;
    const struct {
        const char* what;
        const void* p;
        uint64_t rows, width, stride;
        bool need;
    } ins[] = {{"x", a.x, m, k, (uint64_t)a.x_stride, true},
               {"w", a.w, n, k, (uint64_t)a.w_stride, true},
               {"w2", a.w2, n, k, (uint64_t)a.w2_stride, false},
               {"bias", a.bias, 1, n, 0, false},
               {"bias2", a.bias2, 1, n, 0, false},
               {"residual", a.residual, m, n, (uint64_t)a.residual_stride, false}};
    for (const auto& in : ins) {
        if (!in.p && !in.need) continue;
        uint64_t stride;
        if (__builtin_mul_overflow(in.rows > 1 ? in.stride : 0, size, &stride))
            return fail(II_EOVERFLOW, "%s: the stride of %s", fn, in.what);
        rc = check_rows(fn, in.what, in.p, in.rows, in.width * size, stride, size, &r);
        if (rc) return rc;
        if (in.p == a.residual && in.p == a.out && a.out_dtype == a.dtype &&
            (m == 1 || a.residual_stride == a.out_stride) && in.rows == m && in.width == n)
            continue;  // each element is read by the lane that then writes it
        rc = check_apart(fn, in.what, out, r);
        if (rc) return rc;
    }
    return check_work(fn, a.work, a.work_bytes);
}

}  // namespace
}  // namespace ii

extern "C" int ii_linear(const ii_linear_args* a, hipStream_t stream) {
    if (!a) return ii::fail(II_EINVAL, "ii_linear: args is NULL");
    if (const int rc = ii::check(*a)) return rc;
    if (!a->m || !a->n) return II_OK;
    return a->dtype == II_BF16 ? ii::run<__bf16>(*a, stream) : ii::run<_Float16>(*a, stream);
}
