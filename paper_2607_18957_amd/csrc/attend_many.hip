// Attention of many queries a sequence over a paged key/value cache.
//
// A workgroup of eight waves takes 256 (query, head of the group) rows of a
// sequence and cache head, 32 a wave; keys and values go through LDS 64 tokens
// at a time, read once for all rows, an 8-bit cache unpacked on the way. The
// next 64 are under way in registers meanwhile, the one after that has its
// pages looked up. As for few queries, scores and results are formed
// transposed (S^T = K Q^T, O^T = V^T P^T), here by 32 x 32 x 16 products: a
// lane holds, of the one row lane mod 32, the scores of keys 8 (r / 4) +
// 4 (lane / 32) + r mod 4 of each 32, which are the second product's operand
// if each 16 keys are numbered in that order. V^T comes out of LDS by the
// transposing read in the same order, so nothing crosses lanes but the two
// halves' maxima.
//
// Bound by the matrix instructions, the exponentials and LDS about alike: 64
// keys of 32 rows take a wave's SIMD 1024 cycles of products, nearly as many of
// vector work, and LDS 256, which its eight waves want in turn; all waves are in
// the same phase, so the units are busy in turn, in 35%, 46% and 36% of the
// cycles. One prompt of 8000 tokens, 32 heads over 8, 8-bit cache: 583 us, 899
// TFLOP/s, up to 634 as the clocks go (16 rows a workgroup, as for few queries:
// 2753 us). No register spills: a reload waits for all loads before it, the next
// tile's too (847 us where some did).
#include <algorithm>

#include "attend.h"

namespace ii {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64, kRows = kWaves * 32;
constexpr int kTile = 64;  // keys in LDS at once

// Floats of a part: its rows' sums, then maxima and totals of the weights.
template <int kDim>
constexpr int part_floats() {
    return kRows * (kDim + 2);
}

// This wave's LDS accesses done, then every wave's; loads from memory go on.
__device__ inline void meet_lds() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The larger of the two lanes that share a row.
__device__ inline float max2(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
}

// The lowest n of 64 bits.
__device__ inline uint64_t low_bits(int n) {
    return n >= 64 ? ~0ull : (1ull << n) - 1;
}

template <class T, bool kQuant, int kDim>
__global__ __launch_bounds__(kThreads, 2) void attend_rows(Attend p, int row_tiles, int parts_most,
                                                          int part_keys, int least_rows,
                                                          float* partial) {
    using x8 = typename Vec<T>::x8;
    using x4 = typename Vec<T>::x4;
    constexpr int kQ = kDim / 16, kOut = kDim / 32;  // fragments of a row; of 32 positions of out
    constexpr int kWords = kDim * (kQuant ? 1 : 2) / 16;      // 16-byte words of a key
    constexpr int kBring = 2 * kTile * kWords / kThreads;     // words of a tile a thread brings
    constexpr int kKeys = kWords == 16 ? 2 : 1;               // of so many different tokens
    // LDS rows: eight lanes' words of a fragment, 16 lanes' of a transposing
    // read, meet all banks
    constexpr int kKRow = kDim + 8, kVRow = kDim + 16;
    __shared__ __attribute__((aligned(16))) T ks[2][kTile * kKRow];
    __shared__ __attribute__((aligned(16))) T vs[2][kTile * kVRow];
    __shared__ __attribute__((aligned(16))) T apart[2][kTile * kVRow];
    __shared__ uint8_t state[2][kTile];  // of a key: 1 not there, 2 its values lie in `apart`

    const int lane = threadIdx.x % 64, row = lane % 32, half = lane / 32;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int kv = blockIdx.x, b = blockIdx.z;
    const int my_part = blockIdx.y % parts_most;
    const int tile0 = row_tiles - 1 - blockIdx.y / parts_most;  // the longest first
    const Seq seq = sequence(p, b);
    const int rows = seq.n * p.group;
    if (rows <= least_rows) return;
    const int32_t* const table = p.pages + b * p.pages_stride;

    // what this thread brings of a tile: word i is of keys or of values (op),
    // of token key_of(i), word `word` of it
    const int word = threadIdx.x % kWords;
    const auto op_of = [](int i) { return kBring == 1 ? (int)threadIdx.x / (kThreads / 2) : i / kKeys; };
    const auto key_of = [](int i) {
        return kBring == 1 ? (int)threadIdx.x / kWords % kTile
                           : i % kKeys * (kThreads / kWords) + (int)threadIdx.x / kWords;
    };

    // rows past the tiles that the launch was shaped for: by one workgroup each
    for (int tile = tile0; tile * kRows < rows; tile += row_tiles) {
        const bool extra = tile >= row_tiles;
        const int t_first = tile * kRows / p.group;
        const int t_last = (min(rows, tile * kRows + kRows) - 1) / p.group;
        const Reach reach = reach_of(p, seq, t_first, t_last);
        const int parts = extra ? 1 : parts_of(reach, parts_most, part_keys);
        if (my_part >= parts) return;
        const int64_t keys = max((int64_t)0, reach.hi - reach.lo);
        const int64_t each = ((keys + parts - 1) / parts + kTile - 1) / kTile * kTile;
        const int64_t begin = reach.lo + my_part * each, end = min(reach.hi, begin + each);

        // this lane's row, and what the wave's rows see
        const int r0 = tile * kRows + wave * 32, r = r0 + row, t = r / p.group, g = r % p.group;
        const bool busy = r0 < rows;
        const Reach mine = reach_of(p, seq, min(r0, rows - 1) / p.group, min(r0 + 31, rows - 1) / p.group);
        const Reach own = reach_of(p, seq, min(t, seq.n - 1), min(t, seq.n - 1));

        // a negative scale goes to the queries, exactly, so that the largest
        // product is the largest score
        const float scale = fabsf(p.scale) * 1.44269504f;
        x8 q[kQ];
        const uint8_t* const qrow = p.q + (seq.first + min(t, seq.n - 1)) * p.q_row +
                                    ((int64_t)kv * p.group + g) * p.q_head;
#pragma unroll
        for (int f = 0; f < kQ; ++f) {
            u32x4 w = *reinterpret_cast<const u32x4*>(qrow + (f * 16 + half * 8) * 2);
            if (p.scale < 0) w ^= 0x80008000u;
            q[f] = __builtin_bit_cast(x8, w);
        }

        // the tile under way: pages of the one after it, words and scales
        int32_t page[kKeys];  // as loaded: widening it here would wait for it
        u32x4 held[kBring];
        uint32_t exponent[kBring];
        bool there[kKeys];
        auto look_up = [&](int64_t j0) {
#pragma unroll
            for (int i = 0; i < kKeys; ++i) {
                const int64_t j = j0 + key_of(i);
                page[i] = j < end ? table[j >> p.page_bits] : -1;
            }
        };
        auto load = [&](int64_t j0) {
#pragma unroll
            for (int i = 0; i < kKeys; ++i) there[i] = page[i] >= 0 && page[i] < p.num_pages;
#pragma unroll
            for (int i = 0; i < kBring; ++i) {
                held[i] = u32x4{};
                exponent[i] = 0;
                const int k = i % kKeys;
                if (!there[k]) continue;
                const int64_t in = (j0 + key_of(i)) & (((int64_t)1 << p.page_bits) - 1);
                const int64_t at = page[k];
                held[i] = *reinterpret_cast<const u32x4*>(
                    (op_of(i) ? p.v : p.k) + kv * p.head_stride + at * p.page_stride +
                    in * p.token_stride + word * 16);
                if (kQuant)
                    exponent[i] = (op_of(i) ? p.v_scale : p.k_scale)[at * p.scale_page_stride +
                                                                    kv * p.scale_head_stride +
                                                                    in * p.scale_token_stride + word / 2];
            }
        };
        auto keep = [&](int64_t j0, int buf) {
            // values that are not finite matter where some row sees a part alone
            const bool partly = j0 < reach.lo_max || j0 + kTile > reach.hi_min;
#pragma unroll
            for (int i = 0; i < kBring; ++i) {
                constexpr int kParts = kQuant ? 2 : 1;  // of 8 elements
                x8 v[kParts];
                if constexpr (kQuant) {
                    using x2 = typename Vec<T>::x2;
                    const float s = __builtin_bit_cast(float, exponent[i] << 23);
#pragma unroll
                    for (int w = 0; w < kParts; ++w)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const x2 lo = unpack(held[i][w * 2 + c], s, x2{}, false);
                            const x2 hi = unpack(held[i][w * 2 + c], s, x2{}, true);
                            v[w][c * 4] = lo[0];
                            v[w][c * 4 + 1] = lo[1];
                            v[w][c * 4 + 2] = hi[0];
                            v[w][c * 4 + 3] = hi[1];
                        }
                } else {
                    v[0] = __builtin_bit_cast(x8, held[i]);
                }
                const auto put = [&](T* to) {
#pragma unroll
                    for (int w = 0; w < kParts; ++w)
                        *reinterpret_cast<x8*>(to + word * 8 * kParts + w * 8) = v[w];
                };
                bool mend = false;
                if (partly) {
                    bool odd = false;
#pragma unroll
                    for (int w = 0; w < kParts; ++w) odd |= not_finite<T>(v[w]);
                    // the kWords lanes of a token agree
                    mend = op_of(i) && __ballot(odd) >> (lane / kWords * kWords) & low_bits(kWords);
                    if (mend) {  // out of the product, to the rows that see it
                        put(&apart[buf][key_of(i) * kVRow]);
#pragma unroll
                        for (int w = 0; w < kParts; ++w) v[w] = x8{};
                    }
                }
                put(op_of(i) ? &vs[buf][key_of(i) * kVRow] : &ks[buf][key_of(i) * kKRow]);
                if (op_of(i) && word == 0)
                    state[buf][key_of(i)] = (uint8_t)((there[i % kKeys] ? 0 : 1) | (mend ? 2 : 0));
            }
        };

        f32x16 o[kOut] = {};
        float top = -INFINITY, sum = 0;
        auto work = [&](int64_t j0, int buf) {
            const uint8_t st = state[buf][lane];
            const uint64_t holes = __ballot(st & 1), odd = __ballot(st & 2);
            f32x16 s[2] = {};
            const T* const kat = &ks[buf][row * kKRow + half * 8];
#pragma unroll
            for (int f = 0; f < kQ; ++f) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
                    s[kb] = mfma32(*reinterpret_cast<const x8*>(kat + kb * 32 * kKRow + f * 16), q[f],
                                   s[kb]);
                if (f % 2) __builtin_amdgcn_sched_barrier(0);  // no more words than registers
            }
            __builtin_amdgcn_sched_barrier(0);
            const bool edge = holes || j0 < mine.lo_max || j0 + kTile > mine.hi_min;
            float by = scale;
            uint64_t seen = ~0ull;
            if (edge) {
                const int to = (int)max((int64_t)0, min(own.hi - j0, (int64_t)kTile));
                const int from = (int)max((int64_t)0, min(own.lo - j0, (int64_t)kTile));
                seen = low_bits(to) & ~low_bits(from) & ~holes;
                const uint64_t at = seen >> (half * 4);
                by = 1.0f;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int bit = kb * 32 + e / 4 * 8 + e % 4;
                        s[kb][e] = at >> bit & 1 ? s[kb][e] * scale : -INFINITY;
                    }
            }
            float m = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) m = fmaxf(m, s[kb][e]);
            m = max2(m) * by;
            // sums are taken anew only where a maximum grows by more than 2^kGrow:
            // weights stay below that, and every sum keeps 24 bits
            constexpr float kGrow = std::is_same_v<T, _Float16> ? 2 : 8;
            if (__any(m > top + kGrow)) {
                const float next = fmaxf(top, m), fade = next == -INFINITY ? 1.0f : exp2f(top - next);
                top = next;
                sum *= fade;
#pragma unroll
                for (int n = 0; n < kOut; ++n) o[n] *= fade;
            }
            const float base = top == -INFINITY ? 0.0f : top - lift<T>(kGrow);
            x8 w[4];
            float sums[2] = {};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(s[kb][e], by, -base));
                    sums[e % 2] += x;
                    w[kb * 2 + e / 8][e % 8] = (T)x;
                }
            sum += sums[0] + sums[1];
            const T* const vat = &vs[buf][(half * 4 + lane % 16 / 4) * kVRow + row / 16 * 16 + lane % 4 * 4];
            const auto value = [&](int c, int n) {
                const x4 v0 = read_transposed<T>(vat + c * 16 * kVRow + n * 32);
                const x4 v1 = read_transposed<T>(vat + (c * 16 + 8) * kVRow + n * 32);
                return (x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
                for (int n = 0; n < kOut; ++n) o[n] = mfma32(value(c, n), w[c], o[n]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (odd) {  // keys that are not finite, for the rows that see them
                for (uint64_t left = odd; left; left &= left - 1) {
                    const int key = __builtin_ctzll(left), e = key / 8 % 2 * 4 + key % 4;
                    float mine_w = 0;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int x = 0; x < 8; ++x)
                            if (c == key / 16 && x == e) mine_w = (float)w[c][x];
                    const float weight = __shfl(mine_w, key / 4 % 2 * 32 + row);
                    const T* const at = &apart[buf][key * kVRow + half * 4];
                    if (seen >> key & 1)
#pragma unroll
                        for (int n = 0; n < kOut; ++n)
#pragma unroll
                            for (int x = 0; x < 16; ++x)
                                o[n][x] += weight * (float)at[n * 32 + x / 4 * 8 + x % 4];
                }
            }
        };

        int64_t j0 = begin;
        if (j0 < end) {
            look_up(j0);
            load(j0);
            look_up(j0 + kTile);
        }
        for (int buf = 0; j0 < end; j0 += kTile, buf ^= 1) {
            keep(j0, buf);
            if (j0 + kTile < end) {
                load(j0 + kTile);
                look_up(j0 + 2 * kTile);
            }
            meet_lds();
            if (busy && j0 < mine.hi && j0 + kTile > mine.lo) work(j0, buf);
        }

        sum += __shfl_xor(sum, 32);
        if (parts > 1) {
            constexpr int kFloats = part_floats<kDim>();
            const int64_t unit = ((int64_t)b * gridDim.x + kv) * row_tiles + tile;
            float* const to = partial + (unit * parts_most + my_part) * kFloats;
            const int at = wave * 32 + row;
#pragma unroll
            for (int n = 0; n < kOut; ++n)
#pragma unroll
                for (int x = 0; x < 16; x += 4)
                    *reinterpret_cast<f32x4*>(to + at * kDim + n * 32 + x * 2 + half * 4) =
                        f32x4{o[n][x], o[n][x + 1], o[n][x + 2], o[n][x + 3]};
            if (half == 0) {
                to[kRows * kDim + at] = top;
                to[kRows * (kDim + 1) + at] = sum;
            }
        } else if (r < rows) {
            const float inverse = sum == 0 ? 0.0f : 1.0f / sum;
            uint8_t* const to =
                p.out + (seq.first + t) * p.out_row + ((int64_t)kv * p.group + g) * p.out_head;
#pragma unroll
            for (int n = 0; n < kOut; ++n)
#pragma unroll
                for (int x = 0; x < 16; x += 4) {
                    x4 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = (T)(sum == 0 ? 0.0f : o[n][x + e] * inverse);
                    *reinterpret_cast<x4*>(to + (n * 32 + x * 2 + half * 4) * 2) = y;
                }
        }
        meet_lds();  // the next rows' first tile goes into LDS after every wave's last reads
    }
}

// Rows whose keys went to several workgroups: their parts joined, in order. A
// launch of its own, since the parts of 256 rows are up to some MB, which one
// workgroup reads at 60 GB/s and the card at 4 TB/s.
constexpr int kJoinThreads = 256;

template <class T, int kDim>
__global__ __launch_bounds__(kJoinThreads) void attend_join(Attend p, int row_tiles, int parts_most,
                                                           int part_keys, int least_rows,
                                                           const float* partial) {
    using x4 = typename Vec<T>::x4;
    constexpr int kLanes = kDim / 4, kHere = kJoinThreads / kLanes, kFloats = part_floats<kDim>();
    const int kv = blockIdx.x, b = blockIdx.z, r = blockIdx.y * kHere + threadIdx.x / kLanes;
    const int tile = r / kRows, at = r % kRows, d = threadIdx.x % kLanes * 4;
    const Seq seq = sequence(p, b);
    const int rows = seq.n * p.group;
    if (rows <= least_rows || r >= rows) return;
    const Reach reach = reach_of(p, seq, tile * kRows / p.group,
                                 (min(rows, tile * kRows + kRows) - 1) / p.group);
    const int parts = parts_of(reach, parts_most, part_keys);
    if (parts == 1) return;
    const int64_t unit = ((int64_t)b * gridDim.x + kv) * row_tiles + tile;
    const float* const from = partial + unit * parts_most * kFloats;
    float top = -INFINITY;
    for (int y = 0; y < parts; ++y)
        top = fmaxf(top, from[(int64_t)y * kFloats + kRows * kDim + at]);
    const float base = top == -INFINITY ? 0.0f : top;
    f32x4 v = {};
    float sum = 0;
#pragma unroll 4
    for (int y = 0; y < parts; ++y) {
        const float* const part = from + (int64_t)y * kFloats;
        const float by = __builtin_amdgcn_exp2f(part[kRows * kDim + at] - base);
        v += *reinterpret_cast<const f32x4*>(part + at * kDim + d) * by;
        sum += part[kRows * (kDim + 1) + at] * by;
    }
    const float inverse = sum == 0 ? 0.0f : 1.0f / sum;
    x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (T)(sum == 0 ? 0.0f : v[e] * inverse);
    *reinterpret_cast<x4*>(p.out + (seq.first + r / p.group) * p.out_row +
                           ((int64_t)kv * p.group + r % p.group) * p.out_head + d * 2) = y;
}

template <class T, bool kQuant, int kDim>
void launch_dim(const Attend& p, int64_t max_q, int64_t reach, int least_rows,
                const AttendWork& work, hipStream_t stream) {
    const int kv_heads = p.heads / p.group;
    // a grid's y counts to 65535; rows past it are taken in turn
    const int64_t row_tiles = std::min<int64_t>((max_q * p.group + kRows - 1) / kRows, 2048);
    const int64_t units = row_tiles * kv_heads * p.seqs, tiles = (reach + kTile - 1) / kTile;
    // Parts of a sequence by an expected time, us: 64 keys take 256 rows 2,
    // with a workgroup a compute unit; joining costs a launch and its parts'
    // way to memory and back.
    constexpr int64_t kUnits = 256;
    constexpr int kFloats = part_floats<kDim>();
    int64_t parts = 1;
    double best = 1e30;
    for (int64_t n = 1; n <= 32 && (n == 1 || (work.partial && n * 4 <= tiles && units * n <= 4 * kUnits &&
                                               units * n * kFloats <= (int64_t)work.floats)); ++n) {
        double us = (double)((units * n + kUnits - 1) / kUnits) * ((tiles + n - 1) / n) * 2;
        if (n > 1) us += 6 + units * n * kFloats * 8 / 3e6;
        if (us < best) best = us, parts = n;
    }
    // of a tile at least: a table without columns has none
    const int part_keys = (int)std::clamp<int64_t>((tiles + parts - 1) / parts * kTile, kTile, INT32_MAX / 2);
    attend_rows<T, kQuant, kDim>
        <<<dim3(kv_heads, (uint32_t)(row_tiles * parts), p.seqs), kThreads, 0, stream>>>(
            p, (int)row_tiles, (int)parts, part_keys, least_rows, work.partial);
    if (parts > 1)
        attend_join<T, kDim><<<dim3(kv_heads, (uint32_t)(row_tiles * kRows / (kJoinThreads * 4 / kDim)),
                                    p.seqs), kJoinThreads, 0, stream>>>(
            p, (int)row_tiles, (int)parts, part_keys, least_rows, work.partial);
}

}  // namespace

void attend_many(const Attend& p, int dtype, bool quant, int dim, int64_t max_q, int64_t reach,
                 int least_rows, const AttendWork& work, hipStream_t stream) {
    const auto with = [&](auto t, auto q) {
        using T = decltype(t);
        constexpr bool kQuant = decltype(q)::value;
        dim == 64 ? launch_dim<T, kQuant, 64>(p, max_q, reach, least_rows, work, stream)
                  : launch_dim<T, kQuant, 128>(p, max_q, reach, least_rows, work, stream);
    };
    const auto type = [&](auto q) {
        dtype == II_BF16 ? with(__bf16{}, q) : with(_Float16{}, q);
    };
    quant ? type(std::true_type{}) : type(std::false_type{});
}

}  // namespace ii
