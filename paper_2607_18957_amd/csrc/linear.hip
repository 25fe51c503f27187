// ii_linear: products with weight matrices, and their epilogue.
#include <algorithm>
#include <type_traits>

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
    bool quads;  // four columns of out, biases and residual at a time
};

// y / (1 + exp(-y)). The product of -y and log2(e) is kept in two floats (double-
// length arithmetic), so that the exponential is right to some units in the last
// place however negative y is. Below -64 both sides of the quotient are taken
// 2^-64 times: 1 + exp(-y) passes float's range at -88 and its reciprocal leaves
// the normal range at -87, where the quotient is normal down to -92. The
// reciprocal is the hardware's (1 unit): the division took 5% of a large gated
// product's time.
__device__ inline float silu(float y) {
#pragma clang fp contract(off)  // t is the rounded product everywhere
    constexpr float kHigh = -1.44269504f, kLow = -1.92596299e-8f;  // -log2(e)
    // at -200 the quotient is 0 already
    const float x = __builtin_amdgcn_fmed3f(y, -200.0f, 200.0f);
    const float t = x * kHigh, rest = fmaf(x, kLow, fmaf(x, kHigh, -t));
    const bool low = x < -64.0f;
    const float s = low ? 0x1p-64f : 1.0f;
    const float e = __builtin_amdgcn_exp2f(t - (low ? 64.0f : 0.0f)) * fmaf(rest, 0.693147181f, 1.0f);
    return y * s * __builtin_amdgcn_rcpf(s + e);
}

__device__ inline float activate(float y, int act) {
    switch (act) {
    case II_ACT_RELU: return y < 0 ? 0.0f : y;  // NaN stays
    case II_ACT_SILU: return silu(y);
    // 1 + erf(x) = erfc(-x), which does not cancel where y is negative
    case II_ACT_GELU: return 0.5f * y * erfcf(y * -0.70710678118654752f);
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

// Columns j .. j + 3 of row i, j a multiple of 4.
template <class T, bool kGated>
__device__ inline void put4(const Linear<T>& p, int64_t i, int64_t j, f32x4 y, f32x4 z) {
    using x4 = typename Vec<T>::x4;
    if (!p.quads || j + 4 > p.n) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (j + r < p.n) put<T, kGated>(p, i, j + r, y[r], z[r]);
        return;
    }
    const auto add = [](f32x4& to, const T* from) {
        const x4 v = *reinterpret_cast<const x4*>(from);
#pragma unroll
        for (int r = 0; r < 4; ++r) to[r] += (float)v[r];
    };
    if (p.bias) add(y, p.bias + j);
    if (p.act != II_ACT_NONE)
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = activate(y[r], p.act);
    if (kGated) {
        if (p.bias2) add(z, p.bias2 + j);
        y *= z;
    }
    if (p.residual) add(y, p.residual + i * p.residual_stride + j);
    if (p.out_f32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + i * p.out_stride + j) = y;
    } else {
        x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = (T)y[r];
        *reinterpret_cast<x4*>(static_cast<T*>(p.out) + i * p.out_stride + j) = v;
    }
}

// The sums of the gridDim.y workgroups of a tile, kSums of each in red, joined
// in red of the last of them; false in the others.
template <int kSums, int kThreads>
__device__ inline bool join(float* red, uint32_t* counters, float* partial) {
    const Rsrc parts = buffer(partial + (int64_t)blockIdx.x * gridDim.y * kSums,
                              (int64_t)gridDim.y * kSums * 4);
    __syncthreads();
    for (int e = threadIdx.x * 4; e < kSums; e += kThreads * 4)
        leave_part(parts, (blockIdx.y * kSums + e) * 4, *reinterpret_cast<f32x4*>(&red[e]));
    if (!arrive_last(&counters[blockIdx.x], gridDim.y)) return false;
    for (int e = threadIdx.x * 4; e < kSums; e += kThreads * 4) {
        f32x4 s = {};
#pragma unroll 4
        for (uint32_t y = 0; y < gridDim.y; ++y) s += take_part(parts, (y * kSums + e) * 4);
        *reinterpret_cast<f32x4*>(&red[e]) = s;
    }
    return true;
}

// Few tokens: the weights are read once, straight into the matrix
// instructions' registers, by as many waves as it takes to keep the memory
// busy. A workgroup owns kRows * 16 weight rows (with a gate: 16 of w, 16 of
// w2); its kWaves waves take units of 64 elements of k (a 128-byte line of
// each row) in turn, gridDim.y workgroups share a long k. Waves join their
// sums in LDS in the order of the waves; workgroups leave theirs in `work`,
// and the last to arrive adds them in the order of their places.
// Bound by memory: 1 x 14336 x 4096 24.2 us, 4.9 TB/s.
constexpr int kUnit = 64;  // elements of k a wave takes at once

template <class T, bool kGated, int kRows, int kTokens, int kWaves, int kAhead>
__global__ __launch_bounds__(kWaves * 64) void linear_stream(Linear<T> p, uint32_t* counters,
                                                             float* partial) {
    using x8 = typename Vec<T>::x8;
    constexpr int kSets = kGated ? 2 : 1, kMine = kRows * 16 / kSets;  // rows of each matrix
    constexpr int kSums = kRows * kTokens * 256;
    __shared__ __attribute__((aligned(16))) float red[kWaves * kSums];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16, part = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * kMine;
    const int units = (int)groups(p.k, kUnit), whole = p.k / kUnit;

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
    if (gridDim.y > 1 && !join<kSums, kWaves * 64>(red, counters, partial)) return;
    __syncthreads();
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
// k. Weights are requested two chunks ahead of their use, x one. Bound by
// memory: 24 x 4096 x 14336 with a residual 31 us, 3.8 TB/s.
constexpr int kRowWaves = 2, kKGroups = 8;
constexpr int kChunkPad = 8;         // LDS rows 16 bytes apart in banks

// elements of k a group takes at once
constexpr int shared_chunk(bool gated) { return gated ? 64 : 128; }

template <class T, bool kGated, int kTokens>
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
    const int chunks = (int)groups(p.k, kChunk);
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
    if (gridDim.y > 1 && !join<kAll, kThreads>(red, counters, partial)) return;
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

// Many tokens: kTile tokens by kTile weight rows (with a gate half of them of
// w2, in turn by 16) a workgroup of eight waves, each kTile / 2 tokens by
// kTile / 4 rows. Both operands go from memory straight into LDS, 64 elements
// of k at a time, the next ones while these are multiplied. An LDS row is 128
// bytes, its 16-byte words exchanged by the row's last three bits, so that the
// eight lanes of one LDS cycle, a row each, meet all banks. A workgroup goes
// on to its next tile's first words before it writes a tile. Few tiles share k
// among gridDim.y workgroups, which leave their sums in `partial`.
//
// Bound by the matrix instructions, which the barriers between the stages keep
// from being fed without a pause: 4099 x 14336 x 4096 with a gate 822 us, 1171
// TFLOP/s, matrix units busy in 58% of the cycles. 256 x 256 takes every
// register, and 6 to 8 more in scratch.
constexpr int kTileK = 64, kTileWaves = 8;

// 16 bytes a lane from r at offset + step into LDS, the wave's 1024 in a row.
__device__ inline void load_lds16(Rsrc r, void* lds, int offset, int step) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16,
                                             offset, step, 0, 0);
}

// One LDS buffer of a stage; each is a variable of its own, so that the
// compiler can tell reads of one from loads into another.
template <class T, int kStage, int kOperand, int kRows>
__device__ inline T* stage_rows() {
    __shared__ __attribute__((aligned(1024))) T rows[kRows * kTileK];
    return rows;
}

template <int kValue>
struct Int {
    static constexpr int value = kValue;
};
// f(Int<0>), f(Int<1>), .. f(Int<kN - 1>)
template <int kN, int kI = 0, class F>
__device__ inline void each_of(F&& f) {
    if constexpr (kI < kN) {
        f(Int<kI>{});
        each_of<kN, kI + 1>(f);
    }
}

// All but kYounger of this wave's last memory instructions done, its LDS reads
// too; then every wave of the workgroup.
template <int kYounger>
__device__ inline void meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kYounger) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <class T, bool kGated, int kM, int kN, int kStages, bool kDirect>
__global__ __launch_bounds__(kTileWaves * 64, kM * kN == 256 * 256 ? 2 : 4) void linear_tile(
    Linear<T> p, int tiles_m, int tiles_n, uint32_t* counters, float* partial) {
    using x8 = typename Vec<T>::x8;
    // instructions of a wave that bring an operand, 8 rows each
    constexpr int kBringW = kN / 64, kBringX = kM / 64;
    constexpr int kA = kN / 64, kB = kM / 32;  // a wave's fragments of 16 rows
    static_assert(!kGated || kA % 2 == 0);
    constexpr int kCols = kGated ? kN / 2 : kN;  // columns of out
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int row = lane % 16, part = lane / 16;
    const int wn = wave % 4 * (kN / 4), wm = wave / 4 * (kM / 2);

    // Workgroups go to the 8 XCDs in turn: each XCD gets a run of tiles, in
    // bands of 4 tiles of tokens, so that the tiles its L2 serves at one time
    // share rows.
    constexpr int kBand = 4;
    const int total = tiles_m * tiles_n, xcd = blockIdx.x % 8;
    const int begin = xcd * (total / 8) + min(xcd, total % 8);
    const int end = begin + total / 8 + (xcd < total % 8);
    const int stride = (gridDim.x - xcd + 7) / 8;  // workgroups of this XCD
    int tile = begin + blockIdx.x / 8;
    if (tile >= end) return;

    // this workgroup's part of k, in steps; the last part has the rest
    const int steps_all = p.k / kTileK, each = (steps_all + gridDim.y - 1) / gridDim.y;
    const int step0 = min((int)blockIdx.y * each, steps_all);
    const int steps = min(each, steps_all - step0);
    const int64_t k0 = (int64_t)step0 * kTileK;
    const bool rest = p.k % kTileK && blockIdx.y == gridDim.y - 1;

    // what this wave brings of a tile: an eighth of the rows of each operand
    int64_t m0, n0;
    const T *wbase, *xbase;
    Rsrc wr, xr;
    using Offset = std::conditional_t<kDirect, int, int64_t>;
    Offset woff[kBringW], xoff[kBringX];
    // with a gate, a tile's weight rows are 16 by 16 of w and of w2
    auto mat = [&](int i) { return kGated && (wave * (kN / 8) + i * 8) / 16 % 2; };
    const T* w2base = nullptr;
    Rsrc w2r;
    auto place = [&]() {
        const int band = tile / (kBand * tiles_n), in_band = tile % (kBand * tiles_n);
        const int high = min(kBand, tiles_m - band * kBand);
        m0 = (int64_t)(band * kBand + in_band % high) * kM;
        n0 = (int64_t)(in_band / high) * kCols;
        const int64_t n_end = p.n - 1 - n0, m_end = p.m - 1 - m0, k = p.k - k0;
        wbase = p.w + n0 * p.w_stride + k0;
        xbase = p.x + m0 * p.x_stride + k0;
        wr = buffer(wbase, (n_end * p.w_stride + k) * 2);
        xr = buffer(xbase, (m_end * p.x_stride + k) * 2);
        if (kGated) {
            w2base = p.w2 + n0 * p.w2_stride + k0;
            w2r = buffer(w2base, (n_end * p.w2_stride + k) * 2);
        }
#pragma unroll
        for (int i = 0; i < kBringW; ++i) {
            const int r = wave * (kN / 8) + i * 8 + lane / 8, word = (lane % 8) ^ (r % 8);
            const int64_t c = kGated ? r / 32 * 16 + r % 16 : r;
            const int64_t s = mat(i) ? p.w2_stride : p.w_stride;
            woff[i] = (Offset)((min(c, n_end) * s + word * 8) * 2);
        }
#pragma unroll
        for (int i = 0; i < kBringX; ++i) {
            const int r = wave * (kM / 8) + i * 8 + lane / 8, word = (lane % 8) ^ (r % 8);
            xoff[i] = (Offset)((min((int64_t)r, m_end) * p.x_stride + word * 8) * 2);
        }
    };
    constexpr int kLoads = kBringW + kBringX;
    // stage i of the ring <- elements k .. of this part
    auto bring = [&](int k, auto i_) {
        T* const ws = stage_rows<T, i_.value, 0, kN>();
        T* const xs = stage_rows<T, i_.value, 1, kM>();
#pragma unroll
        for (int i = 0; i < kBringW; ++i) {
            const int at = (wave * (kN / 8) + i * 8) * kTileK;
            if (kGated && mat(i))
                load_lds16(w2r, ws + at, (int)woff[i], k * 2);
            else
                load_lds16(wr, ws + at, (int)woff[i], k * 2);
        }
#pragma unroll
        for (int i = 0; i < kBringX; ++i)
            load_lds16(xr, xs + (wave * (kM / 8) + i * 8) * kTileK, (int)xoff[i], k * 2);
    };
    // the same in two halves: into registers from any address, words past the
    // end of k zero, then into LDS
    x8 held[kLoads];
    auto fetch = [&](int k) {
        const int64_t at = k0 + k + (lane % 8 ^ lane / 8) * 8;  // of this lane's words
        const auto word = [&](const T* base, int64_t off) {
            const char* from = reinterpret_cast<const char*>(base) + off + (int64_t)k * 2;
            if (kDirect) return at < p.k ? *reinterpret_cast<const x8*>(from) : x8{};
            x8 v = {};
            if (at + 8 <= p.k) {
                __builtin_memcpy(&v, from, 16);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (at + e < p.k) v[e] = reinterpret_cast<const T*>(from)[e];
            }
            return v;
        };
#pragma unroll
        for (int i = 0; i < kBringW; ++i) held[i] = word(mat(i) ? w2base : wbase, woff[i]);
#pragma unroll
        for (int i = 0; i < kBringX; ++i) held[kBringW + i] = word(xbase, xoff[i]);
    };
    auto keep = [&](auto i_) {
        T* const ws = stage_rows<T, i_.value, 0, kN>();
        T* const xs = stage_rows<T, i_.value, 1, kM>();
#pragma unroll
        for (int i = 0; i < kBringW; ++i)
            *reinterpret_cast<x8*>(ws + (wave * (kN / 8) + i * 8) * kTileK + lane * 8) = held[i];
#pragma unroll
        for (int i = 0; i < kBringX; ++i)
            *reinterpret_cast<x8*>(xs + (wave * (kM / 8) + i * 8) * kTileK + lane * 8) =
                held[kBringW + i];
    };
    auto begin_tile = [&]() {
        place();
        if constexpr (kDirect) {
            each_of<kStages - 1>([&](auto i_) {
                if (i_.value < steps) bring(i_.value * kTileK, i_);
            });
        } else if (steps > 0) {
            fetch(0);
            keep(Int<0>{});
        }
    };
    begin_tile();
    for (;;) {
        f32x4 acc[kA][kB] = {};
        auto multiply = [&](auto i_) {
            const T* const ws = stage_rows<T, i_.value, 0, kN>();
            const T* const xs = stage_rows<T, i_.value, 1, kM>();
            x8 a[2][kA], b[2][kB];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int word = ((s * 4 + part) ^ (row % 8)) * 8;
#pragma unroll
                for (int i = 0; i < kA; ++i)
                    a[s][i] = *reinterpret_cast<const x8*>(ws + (wn + i * 16 + row) * kTileK + word);
#pragma unroll
                for (int j = 0; j < kB; ++j)
                    b[s][j] = *reinterpret_cast<const x8*>(xs + (wm + j * 16 + row) * kTileK + word);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < kB; ++j)
#pragma unroll
                    for (int i = 0; i < kA; ++i) acc[i][j] = mfma16(a[s][i], b[s][j], acc[i][j]);
            // the first half's reads, then the second's among the first's products
            constexpr int kReads = kA + kB, kProducts = kA * kB;
            __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
#pragma unroll
            for (int i = 0; i < kReads; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, kProducts >= 2 * kReads ? 2 : 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2 * kProducts, 0);
        };
        for (int t0 = 0; t0 < steps; t0 += kStages) {
            each_of<kStages>([&](auto i_) {
                const int t = t0 + i_.value;
                if (t >= steps) return;
                if constexpr (!kDirect) {
                    meet<0>();
                    if (t + 1 < steps) fetch((t + 1) * kTileK);
                    multiply(i_);
                    if (t + 1 < steps) keep(Int<(i_.value + 1) % kStages>{});
                    return;
                }
                // the loads of this step are older than those of the next ones
                if (t + kStages - 2 < steps)
                    meet<(kStages - 2) * kLoads>();
                else
                    meet<0>();
                // into the stage that every wave has multiplied
                if (t + kStages - 1 < steps)
                    bring((t + kStages - 1) * kTileK, Int<(i_.value + kStages - 1) % kStages>{});
                multiply(i_);
            });
        }
        if (rest) {  // what is left of k
            meet<0>();
            fetch(steps * kTileK);
            keep(Int<0>{});
            meet<0>();
            multiply(Int<0>{});
        }
        const int64_t m_out = m0 + wm, n_out = n0 + (kGated ? wn / 2 : wn);
        const int done = tile;
        tile += stride;
        if (tile < end) {
            meet<0>();
            begin_tile();
        }
        bool mine = true;
        if (kM * kN < 256 * 256 && gridDim.y > 1) {
            constexpr int64_t kSums = (int64_t)kM * kN;
            const Rsrc parts = buffer(partial + (int64_t)done * gridDim.y * kSums,
                                      (int64_t)gridDim.y * kSums * 4);
            const auto offset = [&](uint32_t y, int i, int j) {
                return (uint32_t)(y * kSums + ((i * kB + j) * kTileWaves * 64 + threadIdx.x) * 4) * 4;
            };
#pragma unroll
            for (int i = 0; i < kA; ++i)
#pragma unroll
                for (int j = 0; j < kB; ++j)
                    leave_part(parts, offset(blockIdx.y, i, j), acc[i][j]);
            mine = arrive_last(&counters[done], gridDim.y);
            if (mine) {
#pragma unroll
                for (int i = 0; i < kA; ++i)
#pragma unroll
                    for (int j = 0; j < kB; ++j) acc[i][j] = f32x4{};
                // a part at a time, its loads under way together
#pragma unroll(kA * kB < 16 ? 4 : 1)
                for (uint32_t y = 0; y < gridDim.y; ++y) {
                    f32x4 v[kA][kB];
#pragma unroll
                    for (int i = 0; i < kA; ++i)
#pragma unroll
                        for (int j = 0; j < kB; ++j) v[i][j] = take_part(parts, offset(y, i, j));
#pragma unroll
                    for (int i = 0; i < kA; ++i)
#pragma unroll
                        for (int j = 0; j < kB; ++j) acc[i][j] += v[i][j];
                }
            }
        }
        if (mine) {
#pragma unroll
            for (int j = 0; j < kB; ++j)
#pragma unroll
                for (int i = 0; i < kA; i += kGated ? 2 : 1) {
                    const int64_t at = m_out + j * 16 + row;
                    const int64_t c = n_out + (kGated ? i * 8 : i * 16) + part * 4;
                    if (at < p.m) put4<T, kGated>(p, at, c, acc[i][j], acc[kGated ? i + 1 : i][j]);
                }
        }
        if (tile >= end) break;
    }
}

constexpr uint32_t kUnits = 256;  // compute units

struct Work {
    uint32_t* counters = nullptr;
    float* partial = nullptr;
    uint64_t floats = 0;
};

template <class T, bool kGated, int kRows, int kTokens, int kWaves, int kAhead>
void stream_launch(const Linear<T>& p, const Work& work, hipStream_t stream) {
    constexpr int kMine = kRows * 16 / (kGated ? 2 : 1);
    constexpr uint64_t kSums = kRows * kTokens * 256;
    const uint32_t tiles = (uint32_t)groups(p.n, kMine);
    const int units = (int)groups(p.k, kUnit);
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
    const int64_t tiles = groups(p.n, 16), units = groups(p.k, kUnit);
    if (tiles <= 512 && units >= 32)
        stream_launch<T, kGated, kRows, kTokens, kTokens < 4 ? 16 : 8, kAhead>(p, work, stream);
    else if (tiles <= 2048 && units >= 16)
        stream_launch<T, kGated, kRows, kTokens, 8, kAhead>(p, work, stream);
    else
        stream_launch<T, kGated, kRows, kTokens, 4, kAhead>(p, work, stream);
}

template <class T, bool kGated, int kTokens>
void shared_launch(const Linear<T>& p, const Work& work, hipStream_t stream) {
    constexpr int kCols = kRowWaves * 16;
    constexpr uint64_t kAll = (uint64_t)kCols * kTokens * 16 * (kGated ? 2 : 1);
    const uint32_t tiles = (uint32_t)groups(p.n, kCols);
    const uint32_t chunks = (uint32_t)groups(p.k, shared_chunk(kGated));
    // as many workgroups as compute units, each wave with a chunk or more
    uint32_t split = 1;
    if (work.partial && tiles < kUnits)
        split = std::max(1u, std::min(kUnits / tiles, (chunks + kKGroups - 1) / kKGroups));
    while (split > 1 && tiles * split * kAll > work.floats) --split;
    linear_shared<T, kGated, kTokens><<<dim3(tiles, split), kRowWaves * kKGroups * 64, 0, stream>>>(
        p, work.counters, work.partial);
}

// A tile shape, over how many workgroups a tile's k is split, and the time in
// us that the pair is expected to take: a step of 64 elements of k takes each
// shape so long with a workgroup a compute unit; joining costs its start and
// the reading of the parts by the workgroup that comes last, at 60 GB/s.
// Measured: 128 x 4096 x 4096 by 64 x 128 in 4 parts 17.6 us (expected 18);
// 256 x 4096 x 4096 the same in 2 parts 22.6 (24); 1024 x 4096 x 4096 by
// 128 x 256 in 2 parts 45 (44), by 64 x 128 55 (68); 512 x 4096 x 14336 by
// 128 x 256 in 4 parts 75 (74); 512 x 14336 x 4096 with a gate by 256 x 256
// 116 (110), by 128 x 256 128 (138).
struct Shape {
    int m, n;
    double step;
    bool splits;  // 256 x 256 has too much to join
};
constexpr Shape kShapes[3] = {{64, 128, 0.5, true}, {128, 256, 1.05, true}, {256, 256, 1.65, false}};
struct Choice {
    int shape = 0;
    uint32_t split = 1;
    double us = 1e30;
};
Choice choose_tile(int64_t m, int64_t n, int64_t k, bool gated, const Work& work, int shapes) {
    Choice best;
    const int64_t steps = groups(k, kTileK);
    for (int i = 0; i < shapes; ++i) {
        const Shape& s = kShapes[i];
        const int64_t cols = gated ? s.n / 2 : s.n;
        const int64_t tiles = groups(m, s.m) * groups(n, cols);
        for (int64_t split = 1; split <= 16; ++split) {
            if (split > 1 && (!s.splits || !work.partial || tiles * split > kUnits ||
                              split * 2 > steps ||
                              tiles * split * s.m * s.n > (int64_t)work.floats))
                break;
            const int64_t rounds = (tiles * split + kUnits - 1) / kUnits;
            double us = rounds * ((steps + split - 1) / split) * s.step;
            if (split > 1) us += 2 + split * s.m * s.n * 4 / 60e3;
            if (us < best.us) best = {i, (uint32_t)split, us};
        }
    }
    return best;
}

template <class T, bool kGated, int kM, int kN, int kStages, bool kDirect>
void tile_launch(const Linear<T>& p, const Work& work, uint32_t split, hipStream_t stream) {
    constexpr int kCols = kGated ? kN / 2 : kN;
    const int tm = (int)groups(p.m, kM), tn = (int)groups(p.n, kCols);
    const int64_t tiles = (int64_t)tm * tn;
    const int64_t resident = kM == 64 ? 2 * kUnits : kUnits;  // workgroups the card holds at once
    linear_tile<T, kGated, kM, kN, kStages, kDirect>
        <<<dim3((uint32_t)std::min(tiles, resident), split), kTileWaves * 64, 0, stream>>>(
            p, tm, tn, work.counters, work.partial);
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
    // 24.6 us against 27.5 through LDS, 1 x 14336 x 4096 24.2 against 31 in
    // tiles, 1 x 128256 x 4096 184 against 172-179; from 8 tokens on it is 28.7
    // against 28.0, 212 against 176
    // (its grid has a workgroup for each 16 rows; a dispatch counts 2^32 lanes)
    if (wide && p.m <= 4 && p.n <= 1 << 26) return stream_waves<T, kGated, kGated ? 2 : 1, 1, 4>(p, work, stream);
    // rows that waves share through LDS, where it takes all waves of the card
    // to keep up with the memory and a tile's rows would be too few: 24 x 1024
    // x 8192 9.3 us against 13.7 in tiles, 24 x 4096 x 4096 13.4 against 15.4.
    // Tiles of larger matrices are as fast or faster where scratch lets them
    // share k (24 x 4096 x 14336 31 against 28.5, 24 x 8192 x 8192 with a gate
    // 65 against 60) and slower without (51 against 102, 65 against 78)
    if (wide && p.m <= 32 && p.n <= kRowWaves * 16 * (int)kUnits) {
        if (p.m <= 16) return shared_launch<T, kGated, 1>(p, work, stream);
        return shared_launch<T, kGated, 2>(p, work, stream);
    }
    // a tile's rows are addressed in 32 bits (strides may be less than k)
    // Rows that are not whole words, or further apart, go through registers: 24
    // x 4096 x 14336 48 us against 31, 256 x 4096 x 4096 44 against 23, 1 x
    // 14336 x 4096 46 against 24, 4099 x 14336 x 4096 909 against 417
    const bool near = std::max({p.x_stride, p.w_stride, p.w2_stride, (int64_t)p.k}) < (1 << 21);
    const Choice c = choose_tile(p.m, p.n, p.k, kGated, work, wide && near ? 3 : 2);
    if (!wide || !near)
        return c.shape ? tile_launch<T, kGated, 128, 256, 2, false>(p, work, c.split, stream)
                       : tile_launch<T, kGated, 64, 128, 2, false>(p, work, c.split, stream);
    if (c.shape == 0) return tile_launch<T, kGated, 64, 128, 3, true>(p, work, c.split, stream);
    if (c.shape == 1) return tile_launch<T, kGated, 128, 256, 3, true>(p, work, c.split, stream);
    tile_launch<T, kGated, 256, 256, 2, true>(p, work, c.split, stream);
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
    // the stride of a single row says nothing of how it can be read
    p.x_stride = a.m > 1 ? a.x_stride : 0;
    p.w_stride = a.n > 1 ? a.w_stride : 0;
    p.w2_stride = a.n > 1 ? a.w2_stride : 0;
    p.residual_stride = a.m > 1 ? a.residual_stride : 0;
    p.out_stride = a.m > 1 ? a.out_stride : 0;
    p.m = (int32_t)a.m;
    p.n = (int32_t)a.n;
    p.k = (int32_t)a.k;
    p.act = a.act;
    p.out_f32 = a.out_dtype == II_F32;
    const auto quad = [](const void* at, int64_t stride, int size) {
        return !at || (reinterpret_cast<uintptr_t>(at) % (4 * size) == 0 && stride % 4 == 0);
    };
    p.quads = quad(p.out, p.out_stride, p.out_f32 ? 4 : 2) && quad(p.bias, 0, 2) &&
              quad(p.bias2, 0, 2) && quad(p.residual, p.residual_stride, 2);
    Work work;
    if (a.work_bytes > kWorkHead) {
        work.counters = static_cast<uint32_t*>(a.work);
        work.partial = reinterpret_cast<float*>(static_cast<char*>(a.work) + kWorkHead);
        work.floats = (std::min<uint64_t>(a.work_bytes, II_WORK_BYTES) - kWorkHead) / 4;
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
    static const char* const kResidual = "residual";
    Rows out, scratch, r;
    uint64_t out_stride;
    if (__builtin_mul_overflow((uint64_t)(m > 1 ? a.out_stride : 0), osize, &out_stride))
        return fail(II_EOVERFLOW, "%s: the stride of out", fn);
    int rc = check_rows(fn, "out", a.out, m, n * osize, out_stride, osize, &out);
    if (rc || (rc = check_work(fn, a.work, a.work_bytes, &scratch)) ||
        (rc = check_apart(fn, "work", out, scratch)))
        return rc;
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
               {kResidual, a.residual, m, n, (uint64_t)a.residual_stride, false}};
    for (const auto& in : ins) {
        if (!in.p && !in.need) continue;
        uint64_t stride;
        if (__builtin_mul_overflow(in.rows > 1 ? in.stride : 0, size, &stride))
            return fail(II_EOVERFLOW, "%s: the stride of %s", fn, in.what);
        rc = check_rows(fn, in.what, in.p, in.rows, in.width * size, stride, size, &r);
        if (rc || (rc = check_apart(fn, in.what, scratch, r))) return rc;
        if (in.what == kResidual && in.p == a.out && a.out_dtype == a.dtype &&
            (m == 1 || a.residual_stride == a.out_stride))
            continue;  // each element is read by the lane that then writes it
        rc = check_apart(fn, in.what, out, r);
        if (rc) return rc;
    }
    return II_OK;
}

}  // namespace
}  // namespace ii

extern "C" int ii_linear(const ii_linear_args* a, hipStream_t stream) {
    if (!a) return ii::fail(II_EINVAL, "ii_linear: args is NULL");
    {
        const ii::Checks checks;
        if (const int rc = ii::check(*a)) return rc;
    }
    if (!a->m || !a->n) return II_OK;
    return a->dtype == II_BF16 ? ii::run<__bf16>(*a, stream) : ii::run<_Float16>(*a, stream);
}
