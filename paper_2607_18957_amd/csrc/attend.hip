// ii_attend: attention of new tokens over a paged key/value cache.
#include <algorithm>

#include "attend.h"

namespace ii {
namespace {

// Scores are formed transposed, keys by queries (S^T = K Q^T), and so is the
// result (O^T = V^T P^T): with 16 x 16 x 32 products a lane then holds, of one
// query (its lane mod 16), the scores of keys 4 (lane / 16) + r of each 16,
// which are just the operand that the second product takes, if the 32 keys of
// a step are numbered 4 by 4: no score crosses lanes. V^T comes out of LDS by
// the transposing read, whose 16 lanes give 4 keys each of 16 positions.

constexpr int kStep = 32;  // keys a wave takes at once

// 8 or 16 bytes of codes (8-bit) or values of one key, as loaded: kWords words
// of 16 bytes a lane for a key of kDim elements, lane part (lane / 16) having
// bytes 64 c + 16 part of word c.
template <class T, bool kQuant, int kDim>
struct Loaded {
    static constexpr int kWords = kDim * (kQuant ? 1 : 2) / 64;
    u32x4 w[kWords];
    uint32_t scale;  // all scales of the key
};

// Elements of a loaded key: fragment f of kDim / 32 holds the 8 positions
// first_position<..>(f, part) .. + 8.
template <bool kQuant>
__device__ inline int first_position(int f, int part) {
    return kQuant ? f / 2 * 64 + part * 16 + f % 2 * 8 : f * 32 + part * 8;
}
template <class T, bool kQuant, int kDim>
__device__ inline typename Vec<T>::x8 fragment(const Loaded<T, kQuant, kDim>& l, int f, int part) {
    using x8 = typename Vec<T>::x8;
    using x2 = typename Vec<T>::x2;
    if constexpr (kQuant) {
        const uint32_t e = l.scale >> ((f / 2 * 2 + part / 2) * 8) & 255;
        const float scale = __builtin_bit_cast(float, e << 23);
        x8 v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t codes = l.w[f / 2][f % 2 * 2 + i];
            const x2 lo = unpack(codes, scale, x2{}, false), hi = unpack(codes, scale, x2{}, true);
            v[i * 4] = lo[0];
            v[i * 4 + 1] = lo[1];
            v[i * 4 + 2] = hi[0];
            v[i * 4 + 3] = hi[1];
        }
        return v;
    } else {
        return __builtin_bit_cast(x8, l.w[f]);
    }
}

// The largest of the four lanes that share lane mod 16, and their sum.
__device__ inline float max4(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    const uint32_t v = __builtin_bit_cast(uint32_t, x);
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
__device__ inline float sum4(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// ---------------------------------------------------------------------------
// Few queries a sequence: bound by reading the cache. A workgroup takes 16
// (query, head of the group) rows of a sequence and cache head over a part of
// its keys; its waves take steps of 32 keys in turn, each with its own running
// maximum and sum, and load the next step's keys and values while they work on
// one. 48 sequences of up to 8192 keys, 8 heads, 8 bits: 92 us, 4.4 TB/s (the
// vector units, which unpack the codes, are busy in 31% of the cycles); 2 of up
// to 131072 in bf16: 175 us, 5.0 TB/s. Waves join in LDS, parts in `work` by the
// last workgroup to arrive.
constexpr int kRowsHere = 16, kFewWaves = 4;

// The most rows of a sequence that are few. Measured, all as few against all as
// many, 8 heads, 8 bits, 16 sequences of up to 2001 keys and up to 64 rows 42 us
// against 61, 80 rows 36 against 61, 128 rows 53 against 60; 64 of up to 1001: 67
// against 77, 59 against 76, 115 against 79. Of up to 128 rows some are few, and
// both kernels run, one after the other: 76 and 112.
constexpr int kFewRows = 96;

constexpr int kPartsMost = 96;

template <int kDim>
constexpr int part_floats() {
    return kRowsHere * kDim + 2 * kRowsHere;  // sums, then maximum and total of each row
}

template <class T, bool kQuant, int kDim>
__global__ __launch_bounds__(kFewWaves * 64, 2) void attend_split(Attend p, int row_tiles, int parts_most,
                                                             int part_keys, int most_rows,
                                                             uint32_t* counters, float* partial) {
    using x8 = typename Vec<T>::x8;
    using x4 = typename Vec<T>::x4;
    using Key = Loaded<T, kQuant, kDim>;
    constexpr int kFrags = kDim / 32, kOut = kDim / 16;
    constexpr int kRowBytes = kDim * 2 + 32;  // 16 keys' words of one position apart in banks
    constexpr int kVs = kStep * kRowBytes / 2;
    constexpr int kOutRow = kDim + 4;
    __shared__ __attribute__((aligned(16))) T vs[kFewWaves * kVs];
    __shared__ float tops[kFewWaves][kRowsHere], sums[kFewWaves][kRowsHere];
    static_assert(kFewWaves * kVs * 2 >= kFewWaves * kRowsHere * kOutRow * 4 || kDim == 64);
    __shared__ __attribute__((aligned(16))) float outs[kDim == 64 ? kFewWaves * kRowsHere * kOutRow : 4];
    float* const red = kDim == 64 ? outs : reinterpret_cast<float*>(vs);

    const int lane = threadIdx.x % 64, row = lane % 16, part = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int kv = blockIdx.y, b = blockIdx.z;
    // Workgroups go to the 8 XCDs in turn. Short sequences have the first parts
    // alone, so parts are numbered from another place in each sequence and head:
    // with 8 parts the first would all be on one XCD.
    const int tile0 = blockIdx.x % row_tiles;
    const int my_part = (blockIdx.x / row_tiles + kv + b) % parts_most;
    const Seq seq = sequence(p, b);
    const int rows = seq.n * p.group;
    if (rows > most_rows) return;
    const uint8_t* const kbase = p.k + kv * p.head_stride;
    const uint8_t* const vbase = p.v + kv * p.head_stride;
    const int32_t* const table = p.pages + b * p.pages_stride;

    // rows past the tiles that the launch was shaped for: by one workgroup each
    for (int tile = tile0; tile * kRowsHere < rows; tile += row_tiles) {
        const bool extra = tile >= row_tiles;
        if (extra && my_part) return;
        // this lane's row: its query, head, and the keys it sees
        const int r = tile * kRowsHere + row, t = r / p.group, g = r % p.group;
        const bool live = r < rows;
        const int64_t pos = seq.len - seq.n + t;
        int64_t hi = live ? max((int64_t)0, min(pos + 1, p.capacity)) : 0;
        int64_t lo = live && p.window ? max((int64_t)0, pos - p.window + 1) : 0;
        const Reach all = reach_of(p, seq, tile * kRowsHere / p.group,
                                   min(rows - 1, tile * kRowsHere + kRowsHere - 1) / p.group);
        const int64_t hi_min = all.hi_min, lo_max = all.lo_max;
        const int64_t reach = max((int64_t)0, all.hi - all.lo);
        int parts = parts_of(all, parts_most, part_keys);
        if (extra) parts = 1;
        if (my_part >= parts) return;
        const int64_t each = ((reach + parts - 1) / parts + kStep - 1) / kStep * kStep;
        const int64_t begin = all.lo + my_part * each, end = min(all.hi, begin + each);

        x8 q[kFrags];
        const uint8_t* const qrow = p.q + (seq.first + min(t, seq.n - 1)) * p.q_row +
                                    ((int64_t)kv * p.group + g) * p.q_head;
#pragma unroll
        for (int f = 0; f < kFrags; ++f)
            q[f] = *reinterpret_cast<const x8*>(qrow + first_position<kQuant>(f, part) * 2);
        const float scale = p.scale * 1.44269504f;

        f32x4 o[kOut] = {};
        float top = -INFINITY, sum = 0;
        // keys 0 .. 15 and 16 .. 31 of a step: this lane's is `row` of each. The
        // next step's keys are requested as soon as these are multiplied, its
        // values as soon as these are in LDS, its pages a step before: one set
        // of registers, so that none of them spills, which would wait for it
        Key k[2], v[2];
        int32_t page[2];  // as loaded: widening it there would wait for it
        int64_t at[2], sat[2];
        bool held[2];
        auto look_up = [&](int64_t j0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t j = j0 + h * 16 + row;
                page[h] = j < end ? table[j >> p.page_bits] : -1;
            }
        };
        auto locate = [&](int64_t j0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                held[h] = page[h] >= 0 && page[h] < p.num_pages;
                const int64_t in = (j0 + h * 16 + row) & (((int64_t)1 << p.page_bits) - 1);
                const int64_t pg = page[h];
                at[h] = pg * p.page_stride + in * p.token_stride + part * 16;
                sat[h] = pg * p.scale_page_stride + kv * p.scale_head_stride +
                         in * p.scale_token_stride;
            }
        };
        auto load = [&](Key(&to)[2], const uint8_t* base, const uint8_t* scales) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                to[h] = Key{};
                if (!held[h]) continue;
#pragma unroll
                for (int c = 0; c < Key::kWords; ++c)
                    to[h].w[c] = *reinterpret_cast<const u32x4*>(base + at[h] + c * 64);
                if (kQuant && kDim == 128)
                    to[h].scale = *reinterpret_cast<const uint32_t*>(scales + sat[h]);
                else if (kQuant)
                    to[h].scale = *reinterpret_cast<const uint16_t*>(scales + sat[h]);
            }
        };
        constexpr int64_t kTurn = kFewWaves * kStep;
        T* const mine = vs + wave * kVs;
        auto work = [&](int64_t j0) {
            const uint64_t there0 = __ballot(held[0]), there1 = __ballot(held[1]);
            const uint32_t there = (uint32_t)(there0 & 0xffff) | (uint32_t)(there1 & 0xffff) << 16;
            const bool more = j0 + kTurn < end;
            f32x4 s[2] = {};
#pragma unroll
            for (int f = 0; f < kFrags; ++f)
#pragma unroll
                for (int h = 0; h < 2; ++h) s[h] = mfma16(fragment(k[h], f, part), q[f], s[h]);
            __builtin_amdgcn_sched_barrier(0);
            if (more) {
                locate(j0 + kTurn);
                look_up(j0 + 2 * kTurn);
                load(k, kbase, p.k_scale);
            }
            __builtin_amdgcn_sched_barrier(0);
            bool odd = false;  // values that are not finite
            const bool edge = j0 < lo_max || j0 + kStep > hi_min;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    const x8 x = fragment(v[h], f, part);
                    if (edge && not_finite<T>(x)) odd = true;
                    *reinterpret_cast<x8*>(mine + (h * 16 + row) * (kRowBytes / 2) +
                                           first_position<kQuant>(f, part)) = x;
                }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load(v, vbase, p.v_scale);
            __builtin_amdgcn_sched_barrier(0);
            const bool whole = there == 0xffffffffu && !edge;
            float m = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[h][e] *= scale;
                    if (!whole) {
                        const int at = h * 16 + part * 4 + e;
                        const int64_t j = j0 + at;
                        if (!(there >> at & 1) || j < lo || j >= hi) s[h][e] = -INFINITY;
                    }
                    m = fmaxf(m, s[h][e]);
                }
            m = max4(m);
            if (__any(m > top)) {
                const float next = fmaxf(top, m), keep = next == -INFINITY ? 1.0f : exp2f(top - next);
                top = next;
                sum *= keep;
#pragma unroll
                for (int n = 0; n < kOut; ++n) o[n] *= keep;
            }
            const float base = top == -INFINITY ? 0.0f : top - lift<T>(0);
            x8 w;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[h][e] = __builtin_amdgcn_exp2f(s[h][e] - base);
                    sum += s[h][e];
                    w[h * 4 + e] = (T)s[h][e];
                }
            if (edge && __any(odd)) {
                // zero such keys and add what those queries have of them that see them
                const uint64_t b0 = __ballot(odd);
                const uint32_t bad = (uint32_t)((b0 | b0 >> 16 | b0 >> 32 | b0 >> 48) & 0xffff);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        for (int from = 0; from < 4; ++from) {
                            if (!(bad >> (from * 4 + e) & 1)) continue;
                            T* const key = mine + (h * 16 + from * 4 + e) * (kRowBytes / 2);
                            const float weight = __shfl((float)w[h * 4 + e], from * 16 + row);
                            const int at = h * 16 + from * 4 + e;
                            const bool seen = there >> at & 1 && j0 + at >= lo && j0 + at < hi;
#pragma unroll
                            for (int n = 0; n < kOut; ++n)
#pragma unroll
                                for (int x = 0; x < 4; ++x) {
                                    const float v = (float)key[n * 16 + part * 4 + x];
                                    if (seen) o[n][x] += weight * v;
                                }
                            __builtin_amdgcn_wave_barrier();
                            for (int d = lane; d < kDim; d += 64) key[d] = (T)0.0f;
                        }
            }
            __builtin_amdgcn_sched_barrier(0);
            const T* const from = mine + (part * 4 + row / 4) * (kRowBytes / 2) + row % 4 * 4;
#pragma unroll
            for (int n = 0; n < kOut; ++n) {
                const x4 v0 = read_transposed<T>(from + n * 16);
                const x4 v1 = read_transposed<T>(from + 16 * (kRowBytes / 2) + n * 16);
                o[n] = mfma16(__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7), w, o[n]);
            }
        };
        int64_t j0 = begin + wave * kStep;
        if (j0 < end) {
            look_up(j0);
            locate(j0);
            look_up(j0 + kTurn);
            load(k, kbase, p.k_scale);
            load(v, vbase, p.v_scale);
        }
        for (; j0 < end; j0 += kTurn) work(j0);

        // join the waves
        sum = sum4(sum);
        if (part == 0) {
            tops[wave][row] = top;
            sums[wave][row] = sum;
        }
        __syncthreads();
        float all_top = tops[0][row], all_sum = 0;
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) all_top = fmaxf(all_top, tops[w][row]);
        const float base = all_top == -INFINITY ? 0.0f : all_top;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w)
            all_sum += sums[w][row] * __builtin_amdgcn_exp2f(tops[w][row] - base);
        const float keep = __builtin_amdgcn_exp2f(top - base);
#pragma unroll
        for (int n = 0; n < kOut; ++n)
            *reinterpret_cast<f32x4*>(&red[(wave * kRowsHere + row) * kOutRow + n * 16 + part * 4]) =
                o[n] * keep;
        __syncthreads();
        if (wave == 0 && part == 0) {
            tops[0][row] = all_top;
            sums[0][row] = all_sum;
        }
        __syncthreads();
        // a thread's quads of the joined rows, in red[0]
        constexpr int kQuads = kRowsHere * kDim / 4;
        for (int e = threadIdx.x; e < kQuads; e += kFewWaves * 64) {
            float* const at = &red[e / (kDim / 4) * kOutRow + e % (kDim / 4) * 4];
            f32x4 v = *reinterpret_cast<f32x4*>(at);
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w)
                v += *reinterpret_cast<f32x4*>(at + w * kRowsHere * kOutRow);
            *reinterpret_cast<f32x4*>(at) = v;
        }
        if (parts > 1) {
            constexpr int kFloats = part_floats<kDim>();
            const int64_t unit = ((int64_t)b * gridDim.y + kv) * row_tiles + tile;
            const Rsrc left = buffer(partial + unit * parts_most * kFloats, (int64_t)parts * kFloats * 4);
            const uint32_t here = my_part * kFloats * 4;
            for (int e = threadIdx.x; e < kQuads; e += kFewWaves * 64)
                leave_part(left, here + e * 16,
                           *reinterpret_cast<f32x4*>(
                               &red[e / (kDim / 4) * kOutRow + e % (kDim / 4) * 4]));
            if (threadIdx.x < kRowsHere / 4) {
                const int e = threadIdx.x * 4;
                const f32x4 tp = {tops[0][e], tops[0][e + 1], tops[0][e + 2], tops[0][e + 3]};
                const f32x4 sm = {sums[0][e], sums[0][e + 1], sums[0][e + 2], sums[0][e + 3]};
                leave_part(left, here + (kQuads * 4 + e) * 4, tp);
                leave_part(left, here + (kQuads * 4 + kRowsHere + e) * 4, sm);
            }
            if (!arrive_last(&counters[unit], parts)) continue;
            // maxima and totals first, all at once, then the sums, many parts'
            // loads under way together: each waits for memory some us
            float* const fade = red + kRowsHere * kOutRow;  // [part][row]: maxima, then factors
            float* const totals = fade + kPartsMost * kRowsHere;
            static_assert(2 * kPartsMost <= (kFewWaves - 1) * kOutRow);
            for (int i = threadIdx.x; i < parts * 4; i += kFewWaves * 64) {
                const uint32_t at = (i / 4 * kFloats + kQuads * 4 + i % 4 * 4) * 4;
                *reinterpret_cast<f32x4*>(&fade[i * 4]) = take_part(left, at);
                *reinterpret_cast<f32x4*>(&totals[i * 4]) = take_part(left, at + kRowsHere * 4);
            }
            __syncthreads();
            constexpr int kStride = kFewWaves * 4;
            float best = -INFINITY, total = 0;
            for (int y = wave * 4 + part; y < parts; y += kStride)
                best = fmaxf(best, fade[y * kRowsHere + row]);
            best = max4(best);
            if (part == 0) tops[wave][row] = best;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) best = fmaxf(best, tops[w][row]);
            const float from = best == -INFINITY ? 0.0f : best;
            for (int y = wave * 4 + part; y < parts; y += kStride) {
                float& f = fade[y * kRowsHere + row];
                f = __builtin_amdgcn_exp2f(f - from);
                total += f * totals[y * kRowsHere + row];
            }
            total = sum4(total);
            __syncthreads();
            if (part == 0) sums[wave][row] = total;
            constexpr int kMine = kQuads / (kFewWaves * 64);
            f32x4 v[kMine] = {};
#pragma unroll 8
            for (int y = 0; y < parts; ++y)
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    const int e = threadIdx.x + i * kFewWaves * 64;
                    v[i] += take_part(left, (y * kFloats + e * 4) * 4) *
                            fade[y * kRowsHere + e / (kDim / 4)];
                }
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int e = threadIdx.x + i * kFewWaves * 64;
                *reinterpret_cast<f32x4*>(&red[e / (kDim / 4) * kOutRow + e % (kDim / 4) * 4]) = v[i];
            }
            __syncthreads();
            if (wave == 0 && part == 0) {
#pragma unroll
                for (int w = 1; w < kFewWaves; ++w) total += sums[w][row];
                sums[0][row] = total;
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < kQuads; e += kFewWaves * 64) {
            const int rr = e / (kDim / 4), d = e % (kDim / 4) * 4, at = tile * kRowsHere + rr;
            if (at >= rows) continue;
            const float total = sums[0][rr], inverse = total == 0 ? 0.0f : 1.0f / total;
            const f32x4 v = *reinterpret_cast<f32x4*>(&red[rr * kOutRow + d]) * inverse;
            x4 y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = (T)(total == 0 ? 0.0f : v[x]);
            *reinterpret_cast<x4*>(p.out + (seq.first + at / p.group) * p.out_row +
                                   ((int64_t)kv * p.group + at % p.group) * p.out_head + d * 2) = y;
        }
        __syncthreads();
    }
}

template <class T, bool kQuant, int kDim>
void launch_dim(const Attend& p, int64_t max_q, int64_t reach, int most_rows,
                const AttendWork& work, hipStream_t stream) {
    const int kv_heads = p.heads / p.group;
    const int64_t row_tiles = (max_q * p.group + kRowsHere - 1) / kRowsHere;
    const int64_t units = row_tiles * kv_heads * p.seqs;
    // Parts of a sequence, of 512 keys or more. The card holds 512 workgroups:
    // few units take as many, so that none comes second; ragged ones in large
    // numbers three times as many, so that long ones do not come last. Measured
    // with 512, 1024, 1536, 2048: 16 units of up to 131072 keys 184, 204, 210,
    // 208 us; 64 of up to 20001 58, 63, 58, 81; 256 of up to 8001 83, 78, 69, 73;
    // 384 of up to 8192 165, 144, 113, 121. Parts of 256 keys: 1 x 4001 20 us
    // against 18.
    int64_t part_keys = 512, parts = 1;
    if (work.partial && units <= (int64_t)kWorkCounters) {
        parts = std::min<int64_t>({(reach + part_keys - 1) / part_keys,
                                   (units <= 128 ? 512 : 1536) / units, kPartsMost,
                                   (int64_t)(work.floats / (units * part_floats<kDim>()))});
        parts = std::max<int64_t>(1, parts);
        part_keys = std::max<int64_t>(part_keys, (reach + parts - 1) / parts);
    }
    attend_split<T, kQuant, kDim>
        <<<dim3((uint32_t)(row_tiles * parts), kv_heads, p.seqs), kFewWaves * 64, 0, stream>>>(
            p, (int)row_tiles, (int)parts, (int)std::min<int64_t>(part_keys, INT32_MAX / 2),
            most_rows, work.counters, work.partial);
}

// Attention of the sequences with up to most_rows (query, head of a group)
// rows.
void attend_few(const Attend& p, int dtype, bool quant, int dim, int64_t max_q, int64_t reach,
                int most_rows, const AttendWork& work, hipStream_t stream) {
    const auto with = [&](auto t, auto q) {
        using T = decltype(t);
        constexpr bool kQuant = decltype(q)::value;
        dim == 64 ? launch_dim<T, kQuant, 64>(p, max_q, reach, most_rows, work, stream)
                  : launch_dim<T, kQuant, 128>(p, max_q, reach, most_rows, work, stream);
    };
    const auto type = [&](auto q) {
        dtype == II_BF16 ? with(__bf16{}, q) : with(_Float16{}, q);
    };
    quant ? type(std::true_type{}) : type(std::false_type{});
}

int run(const ii_attend_args& a, const ii_cache& c, hipStream_t stream) {
    const char* fn = "ii_attend";
    const Checks checks;
    CacheRows held;
    int rc = check_cache(fn, c, false, &held);
    if (rc) return rc;
    if (!half_type(a.dtype)) return fail(II_EINVAL, "%s: dtype %d", fn, a.dtype);
    const bool quant = c.dtype == II_FP8_E4M3;
    if (!quant && c.dtype != a.dtype)
        return fail(II_EINVAL, "%s: a cache of type %d, queries of type %d", fn, c.dtype, a.dtype);
    if (a.reserved) return fail(II_EINVAL, "%s: reserved is %d", fn, a.reserved);
    if (a.heads < 1 || a.heads % c.heads || a.heads > 65535)
        return fail(II_EINVAL, "%s: %d query heads over %d cache heads", fn, a.heads, c.heads);
    if (a.rows < 0 || a.rows > INT32_MAX || a.seqs < 0 || a.seqs > 65535 || a.max_q < 0 ||
        a.max_len < 0 || a.window < 0 || a.rows * a.heads > 1 << 30)
        return fail(II_EINVAL, "%s: a size is out of range", fn);
    if (a.columns < 0 || a.columns > ((int64_t)1 << 40) / c.page || a.pages_stride < 0)
        return fail(II_EINVAL, "%s: a page table of %lld columns, stride %lld", fn,
                    (long long)a.columns, (long long)a.pages_stride);
    uint64_t pages_stride;
    if (__builtin_mul_overflow((uint64_t)(a.seqs > 1 ? a.pages_stride : 0), (uint64_t)4, &pages_stride))
        return fail(II_EOVERFLOW, "%s: the stride of pages", fn);
    if (!std::isfinite(a.scale)) return fail(II_EINVAL, "%s: scale is not finite", fn);
    if (!a.q_start && a.rows != a.seqs)
        return fail(II_EINVAL, "%s: %lld rows for %lld sequences without q_start", fn,
                    (long long)a.rows, (long long)a.seqs);
    if (!a.rows || !a.seqs) return II_OK;
    Rows q, out, table, lengths, starts, scratch;
    if ((rc = check_heads(fn, "out", a.out, a.rows, a.heads, c.dim, a.out_row_stride,
                          a.out_head_stride, 2, true, &out)) ||
        (rc = check_heads(fn, "q", a.q, a.rows, a.heads, c.dim, a.q_row_stride, a.q_head_stride, 2,
                          false, &q)) ||
        (rc = check_rows(fn, "pages", a.pages, a.seqs, (uint64_t)a.columns * 4, pages_stride, 4,
                         &table)) ||
        (rc = check_rows(fn, "lengths", a.lengths, 1, (uint64_t)a.seqs * 4, 0, 4, &lengths)) ||
        (rc = check_rows(fn, "q_start", a.q_start, a.q_start ? 1 : 0, ((uint64_t)a.seqs + 1) * 4, 0,
                         4, &starts)) ||
        (rc = check_work(fn, a.work, a.work_bytes, &scratch)) ||
        (rc = check_apart(fn, "work", out, scratch)))
        return rc;
    for (const Rows& written : {out, scratch}) {
        if ((rc = check_apart(fn, "q", written, q)) || (rc = check_apart(fn, "pages", written, table)) ||
            (rc = check_apart(fn, "lengths", written, lengths)) ||
            (rc = check_apart(fn, "q_start", written, starts)))
            return rc;
        for (const Rows& r : held.all)
            if ((rc = check_apart(fn, "the cache", written, r))) return rc;
    }
    const int64_t size = quant ? 1 : 2;
    Attend p;
    p.q = static_cast<const uint8_t*>(a.q);
    p.k = static_cast<const uint8_t*>(c.k);
    p.v = static_cast<const uint8_t*>(c.v);
    p.k_scale = c.k_scale;
    p.v_scale = c.v_scale;
    p.out = static_cast<uint8_t*>(a.out);
    p.q_row = a.q_row_stride * 2;
    p.q_head = a.q_head_stride * 2;
    p.out_row = a.out_row_stride * 2;
    p.out_head = a.out_head_stride * 2;
    p.page_stride = c.page_stride * size;
    p.head_stride = c.head_stride * size;
    p.token_stride = c.token_stride * size;
    p.scale_page_stride = c.scale_page_stride;
    p.scale_head_stride = c.scale_head_stride;
    p.scale_token_stride = c.scale_token_stride;
    p.pages = a.pages;
    p.lengths = a.lengths;
    p.q_start = a.q_start;
    p.pages_stride = a.pages_stride;
    p.capacity = a.columns * c.page;
    p.rows = a.rows;
    // lengths are 32-bit: a window of 2^31 hides nothing, and the sums of positions
    // and windows below stay far from 64 bits' ends
    p.window = a.window <= INT32_MAX ? a.window : 0;
    p.num_pages = c.pages;
    p.seqs = (int32_t)a.seqs;
    p.heads = a.heads;
    p.group = a.heads / c.heads;
    p.page_bits = __builtin_ctz(c.page);
    p.scale = a.scale;
    AttendWork work;
    if (a.work_bytes > kWorkHead) {
        work.counters = static_cast<uint32_t*>(a.work);
        work.partial = reinterpret_cast<float*>(static_cast<char*>(a.work) + kWorkHead);
        work.floats = (std::min<uint64_t>(a.work_bytes, II_WORK_BYTES) - kWorkHead) / 4;
    }
    const int64_t max_q = a.q_start ? std::max<int64_t>(1, std::min(a.max_q, a.rows)) : 1;
    const int64_t reach_q = a.max_len > 0 ? std::min(a.max_len, p.capacity) : p.capacity;
    const int64_t reach = p.window ? std::min(reach_q, p.window + max_q) : reach_q;
    // Sequences of many rows go to one kernel, the others to another. The call
    // does not read the sizes, so both are launched unless all sequences have
    // max_q queries.
    const bool many = max_q * p.group > kFewRows, mixed = a.rows < a.seqs * max_q;
    if (many)
        attend_many(p, a.dtype, quant, c.dim, max_q, reach, mixed ? kFewRows : 0, work, stream);
    if (!many || mixed)
        attend_few(p, a.dtype, quant, c.dim, many ? std::max(1, kFewRows / p.group) : max_q, reach,
                   many ? kFewRows : INT32_MAX, work, stream);
    return launched(fn);
}

}  // namespace
}  // namespace ii

extern "C" int ii_attend(const ii_attend_args* a, const ii_cache* c, hipStream_t stream) {
    if (!a || !c) return ii::fail(II_EINVAL, "ii_attend: an argument is NULL");
    return ii::run(*a, *c, stream);
}
