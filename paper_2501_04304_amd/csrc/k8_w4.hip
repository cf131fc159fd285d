// Weights in 4 bits with a scale and a zero for every group of 32, 64 or 128 inputs, and their products with few rows.
//
// Per output and group:  lo = min(0, min w), hi = max(0, max w), s = (hi - lo) * (1/15) with the 4 lowest bits of its pattern
// cleared (0 below 2^-96), zero = clamp(rne(-lo / s), 0, 15), code = clamp(rne(w / s) + zero, 0, 15) (both quotients times 1/s),
// value s (code - zero).  The layout (include/dgq.h) is the product's: a unit is 16 outputs x 128 inputs, 1 KiB of codes of which
// a lane's 16 bytes are its part of four operands of the 16 x 16 x 32 matrix instructions, and behind all codes one word for each
// group, its scale with the zero in the 4 lowest bits.
#include <algorithm>
#include <cmath>

#include "vectors.h"

namespace dgq {
namespace {

constexpr int kUnit = 128;  // inputs
constexpr float kLeastScale = 0x1p-96f;
constexpr uint32_t kNaNWord = 0x7fc00000u;

// A lane's place in a unit: row r of 16, and of every 32 inputs (j) the eight from 8 q on.
struct Lane {
    int r, q;
    __device__ Lane() : r(threadIdx.x & 15), q(threadIdx.x >> 4 & 3) {}
};

// One row's part of a unit for a lane, four times eight inputs; from C on 0.
template <class T>
struct RowPart {
    T x[4][8];
    __device__ void load(const T *row, int k0, int C) {
        if (k0 + 104 <= C) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; i += kVec<T>) {
                    const loose<T, kVec<T>> v = *reinterpret_cast<const loose<T, kVec<T>> *>(row + k0 + 32 * j + i);
#pragma unroll
                    for (int e = 0; e < kVec<T>; ++e) x[j][i + e] = v[e];
                }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[j][i] = k0 + 32 * j + i < C ? row[k0 + 32 * j + i] : (T)0.f;
        }
    }
};

// nibble of input i (0 .. 7) of a lane's word
__device__ constexpr int nibble(int i) { return i % 2 ? 4 + i / 2 : i / 2; }

// over the lanes of a row
__device__ float row_min(float x) {  // NaN if one is
    x = __builtin_elementwise_minimum(x, __shfl_xor(x, 16));
    return __builtin_elementwise_minimum(x, __shfl_xor(x, 32));
}
__device__ float row_max(float x) {
    x = __builtin_elementwise_maximum(x, __shfl_xor(x, 16));
    return __builtin_elementwise_maximum(x, __shfl_xor(x, 32));
}

// ---- packing ---------------------------------------------------------------------------------------------------------
// A wavefront per unit, four neighbours of a row of units to a workgroup: a lane reads what its 16 bytes of codes stand for, lines
// of memory meet in four loads.  Bound by the bytes of w (8192 x 8192 bf16 31.5 us, 5.4 TB/s).
template <class T, int J>  // J: words of 32 inputs in a group
__global__ __launch_bounds__(256) void k_w4_pack(const T *__restrict__ w, int64_t w_row, W4 m) {
    const uint32_t wide = (m.T + 3) / 4, tile = blockIdx.x / wide;
    const int t = (blockIdx.x - tile * wide) * 4 + (threadIdx.x >> 6);
    if (t >= m.T) return;
    const int64_t unit = (int64_t)tile * m.T + t;
    const Lane l;
    const int o = tile * 16 + l.r, k0 = t * kUnit + l.q * 8;
    RowPart<T> part;
    part.load(w + min(o, m.O - 1) * w_row, k0, o < m.O ? m.C : 0);
    float f[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) f[j][i] = (float)part.x[j][i];
    uint32_t code[4], word[4 / J];
#pragma unroll
    for (int g = 0; g < 4 / J; ++g) {
        float lo = 0.f, hi = 0.f;  // NaN once a weight is
#pragma unroll
        for (int j = g * J; j < g * J + J; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lo = __builtin_elementwise_minimum(lo, f[j][i]);
                hi = __builtin_elementwise_maximum(hi, f[j][i]);
            }
        lo = row_min(lo), hi = row_max(hi);
        const float all = hi - lo;
        const bool bad = !(all <= 0x1.fffffep127f);
        float s = __uint_as_float(__float_as_uint(all * (float)(1.0 / 15)) & ~15u);
        if (!(s >= kLeastScale)) s = 0.f;
        const float inv = s > 0.f ? 1.0f / s : 0.f, zero = fminf(fmaxf(rintf(-lo * inv), 0.f), 15.f);
        word[g] = bad ? kNaNWord : __float_as_uint(s) | (uint32_t)zero;
        // w / s plus 3 2^22 has rne(w / s) in its lowest bits
        const int from = (int)zero - __float_as_int(0x1.8p23f);
#pragma unroll
        for (int j = g * J; j < g * J + J; ++j) {
            code[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = __float_as_int(f[j][i] * inv + 0x1.8p23f) + from;
                code[j] |= (uint32_t)min(max(c, 0), 15) << (4 * nibble(i));
            }
            if (bad) code[j] = 0;
        }
    }
    reinterpret_cast<uint4 *>(m.codes)[unit * 64 + (threadIdx.x & 63)] = uint4{code[0], code[1], code[2], code[3]};
    if (l.q == 0)
#pragma unroll
        for (int g = 0; g < 4 / J; ++g) m.words()[(unit * 16 + l.r) * (4 / J) + g] = word[g];
}

// A wavefront per unit: its stores are whole rows of the unit, one next to the other, whose lanes pick their codes' words.  past:
// the values are whole lines of memory and go past the caches (8192 x 8192 bf16 25.5 us, 6.6 TB/s, and 33 without; behind k_w4_pack
// 57 for both and 65).  Rows that begin inside a line lose by that (8191 x 8191 fp16 behind its packing 103 and 89).
template <class T, int J>
__global__ __launch_bounds__(256) void k_w4_unpack(W4 m, T *__restrict__ w, bool past) {
    constexpr int V = kVec<T>, kLanes = kUnit / V, kRows = 64 / kLanes;  // lanes to a row, rows at a time
    const uint32_t wide = (m.T + 3) / 4, tile = blockIdx.x / wide;
    const int t = (blockIdx.x - tile * wide) * 4 + (threadIdx.x >> 6);
    if (t >= m.T) return;
    const int64_t unit = (int64_t)tile * m.T + t;
    const int lane = threadIdx.x & 63, at = lane % kLanes * V, up = lane / kLanes, j = at / 32, q = at / 8 % 4, k = t * kUnit + at;
    const uint32_t *codes = reinterpret_cast<const uint32_t *>(m.codes) + unit * 256 + 64 * q + j;
    const uint32_t *words = m.words() + unit * (64 / J) + j / J;
    uint32_t code[16 / kRows], word[16 / kRows];
#pragma unroll
    for (int n = 0; n < 16 / kRows; ++n) code[n] = codes[4 * (n * kRows + up)], word[n] = words[(n * kRows + up) * (4 / J)];
#pragma unroll
    for (int n = 0; n < 16 / kRows; ++n) {
        const int o = tile * 16 + n * kRows + up;
        if (o >= m.O) return;
        const float s = __uint_as_float(word[n] & ~15u);
        const int zero = word[n] & 15;
        const uint32_t own = code[n] >> at % 8 * 2;  // (the nibbles of 4 .. 7 lie two above those of 0 .. 3)
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)((int)(own >> (4 * nibble(i)) & 15) - zero) * s;
        T *to = w + (int64_t)o * m.C + k;
        past ? store_past(to, m.C - k, f) : store_vector(to, m.C - k, f);
    }
}

// ---- products --------------------------------------------------------------------------------------------------------
//   y[m, o] = sum_g s (sum_{k in g} x[m, k] (code - zero))
// on the matrix cores, 16 rows of x by 16 outputs by 32 inputs, in fp16.  A nibble below the exponent of 1024 is 1024 + code (at
// bits 0 .. 3) or 1024 + 16 code (at 4 .. 7), less 1024 + zero or times 1/16 less 64 + zero it is code - zero, exactly: nine
// instructions for eight codes (Kim et al., arXiv 2211.10017, with the zeros folded in).  Rows of fp16 are what they are; those
// of bf16 and fp32 are taken a unit (128 inputs) at a time by a power of two that brings its largest to 2^14 .. 2^15, bf16 as
// one fp16, fp32 as two (x = h + l, each rounded to nearest: off by 2^-23 x at most).  l is kept 2^12 times as large, which
// brings it up to 2^15 too, and has sums of its own: at h's scale it would leave fp16's normal numbers 2^16 below the unit's
// largest (2 % of the time, 5 % at groups of 32).  What lies more than 2^28 below that loses bits, fp32 to 2^-51 of it, bf16 to
// 2^-39.  The groups' sums meet in fp32 with their scales and those powers.
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));

union Piece {  // a lane's 8 numbers of an operand
    half2v p[4];
    uint32_t w[4];
    half8 all;
};

template <class T>
constexpr int kPieces = sizeof(T) == 4 ? 2 : 1;
constexpr float kSecond = 0x1p12f;  // the second piece's own power

// x & mask | bits in one instruction: both constants stay in registers (as literals they take two)
__device__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) { return (x & mask) | bits; }

// code - zero of a lane's eight codes.  zero: of the group's word.
struct Expand {
    uint32_t nibble0 = 0x000f000fu, nibble1 = 0x00f000f0u, one = 0x64006400u;
    struct Zero {
        _Float16 low, high;  // -(1024 + zero), -(64 + zero)
    };
    __device__ Expand() { asm("" : "+s"(nibble0), "+s"(nibble1), "+v"(one)); }
    __device__ static Zero zero(uint32_t word) {
        const uint16_t low = 0xe400u | (word & 15), high = 0xd400u | (word & 15) << 4;
        return {__builtin_bit_cast(_Float16, low), __builtin_bit_cast(_Float16, high)};
    }
    __device__ half8 operator()(uint32_t code, const Zero &zero) const {
        const half2v part{(_Float16)(1.f / 16), (_Float16)(1.f / 16)}, low{zero.low, zero.low}, high{zero.high, zero.high};
        Piece p;
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const uint32_t two = i ? code >> 8 : code;
            p.w[i] = and_or(two, nibble0, one);
            p.w[i + 1] = and_or(two, nibble1, one);
            p.p[i] += low;
            p.p[i + 1] = __builtin_elementwise_fma(p.p[i + 1], part, high);
        }
        return p.all;
    }
};

// Its inputs as operands; returns what their sums are to be multiplied by.
template <class T>
__device__ float convert(const T (&x)[4][8], Piece (&a)[4][kPieces<T>]) {
    if constexpr (std::is_same_v<T, _Float16>) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) a[j][0].all[i] = x[j][i];
        return 1.f;
    } else {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = __builtin_elementwise_maximum(top, fabsf((float)x[j][i]));
        const int e = max((int)(__float_as_uint(row_max(top)) >> 23 & 255), 15);  // 15: 2^-112
        const float down = __uint_as_float((uint32_t)(268 - e) << 23);     // 2^(14 - (e - 127)); e = 255 (infinity): 2^-114
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x0 = (float)x[j][2 * i], x1 = (float)x[j][2 * i + 1];
                const half2v h = __builtin_convertvector((float2v{x0 * down, x1 * down}), half2v);
                a[j][0].p[i] = h;
                if constexpr (kPieces<T> > 1)  // what h leaves is exact, and so are products with powers of two: l is rounded once
                    a[j][1].p[i] = __builtin_convertvector(
                        (float2v{fmaf(x0, down, -(float)h[0]) * kSecond, fmaf(x1, down, -(float)h[1]) * kSecond}), half2v);
            }
        return __uint_as_float((uint32_t)(e - 14) << 23);
    }
}

// How a product is cut: a workgroup has `tiles` times `shares` wavefronts, one for each of its tiles of 16 outputs and each share
// of the units (every shares-th), for 16 rows of x.  The rows of `chunk` units at a time are brought into fp16 by all of them and
// wait in LDS, 1, 4 or 16 rows (1 << row_shift).  splits: workgroups (blockIdx.z) that have a part of the units each, where there
// are few outputs and many inputs; their sums meet in a second kernel.
struct Cut {
    int32_t tiles, shares, splits, chunk, row_shift;
};

// Bound by the bytes of the weights (1 x 8192 -> 28672 bf16 23.8 us, 5.2 TB/s; a read of as many bytes takes 21) and, from 16
// rows on, by the vector pipes: 55 instructions to a unit of one tile beside four matrix instructions (fp32: 4 more a group, and
// eight), 130 (bf16) or 230 (fp32) to bring 16 rows of a unit into fp16, once for all tiles of a workgroup.  A wavefront's next
// kAhead units are on their way while it works on as many, and the rows of the next chunk while all work on this one.  Small
// products are bound by latency: 2 x 320 -> 1280 5.1 us, 32 x 1280 -> 16640 fp32 11.8 (rows 2, their conversion 2, ten units a
// wavefront 3.8, the slowest SIMD 2.6, the sums 1).
// kAhead: 8 x 4096 -> 11000 bf16 11.3 us with two, 11.8 with three, 12.4 with four; 1 x 8192 -> 28672 fp16 23.6, 22.5 and 22.6.
template <int J, bool ONCE>
constexpr int kAhead = ONCE && J > 1 ? 3 : 2;
// Wavefronts of a workgroup, as many as registers allow.
template <class T>
constexpr int kMaxWaves = sizeof(T) == 4 ? 12 : 16;

template <int J, int AHEAD>
struct Units {
    uint4 code[AHEAD];
    uint32_t word[AHEAD][4 / J];
};

// Codes, or codes that no cache need keep.
template <bool ONCE>
__device__ uint4 read_codes(const char *p) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    if constexpr (!ONCE) return *reinterpret_cast<const uint4 *>(p);
    const words v = __builtin_nontemporal_load(reinterpret_cast<const words *>(p));
    return {v.x, v.y, v.z, v.w};
}

template <class T, class Y, int J, int SHIFT, bool ONCE>
__global__ __launch_bounds__(64 * kMaxWaves<T>) void k_w4_matvec(const T *__restrict__ x, int64_t x_row, int32_t M, W4 m, Cut cut,
                                                   const float *__restrict__ bias, int32_t silu_on, Y *__restrict__ y,
                                                   float *__restrict__ parts) {
    constexpr int P = kPieces<T>, AHEAD = kAhead<J, ONCE>;
    constexpr bool kPowers = !std::is_same_v<T, _Float16>;
    extern __shared__ uint4 lds[];  // [chunk][4 j][P][4 q][rows], then the powers [chunk][16]; later the sums
    const unsigned tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    constexpr int shift = SHIFT, rows = 1 << shift;
    float *powers = reinterpret_cast<float *>(lds + cut.chunk * 16 * P * rows);
    const Lane l;
    const int tile = wave % cut.tiles, share = wave / cut.tiles, row0 = blockIdx.y * 16;
    const int64_t unit0 = (int64_t)min((int)blockIdx.x * cut.tiles + tile, m.R - 1) * m.T;  // behind the last: that again, not written
    const char *codes = reinterpret_cast<const char *>(m.codes) + unit0 * 1024;  // the tile's, the same for all lanes
    const char *words = reinterpret_cast<const char *>(m.words() + unit0 * (64 / J));
    const Expand expand;

    // units first, first + shares, .. of a chunk that ends at `end` (its last again where there are no more)
    auto fetch = [&](Units<J, AHEAD> &to, int first, int end) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int t = min(first + d * cut.shares, end - 1);
            to.code[d] = read_codes<ONCE>(codes + (uint32_t)(t * 1024 + lane * 16));  // (a tile has less than 2^24 bytes)
            const uint32_t *w = reinterpret_cast<const uint32_t *>(words + (uint32_t)(t * (256 / J) + l.r * (16 / J)));
#pragma unroll
            for (int g = 0; g < 4 / J; ++g) to.word[d][g] = w[g];
        }
    };
    const int begin = (int)((int64_t)m.T * blockIdx.z / cut.splits), stop = (int)((int64_t)m.T * (blockIdx.z + 1) / cut.splits);
    Units<J, AHEAD> now, next;
    fetch(now, begin + share, min(begin + cut.chunk, stop));

    // this lane's row, and its units of a chunk: first, first + step, ..
    const int per = 16 >> shift, first = wave * per + (l.r >> shift), step = waves * per, row = l.r & (rows - 1);
    const T *mine = x + min(row0 + row, M - 1) * x_row;
    RowPart<T> part;
    part.load(mine, min(begin + first, stop - 1) * kUnit + 8 * l.q, m.C);

    float4v out{};
    for (int t0 = begin; t0 < stop; t0 += cut.chunk) {
        const int end = min(t0 + cut.chunk, stop);
        if (t0 > begin) __syncthreads();
        for (int u = first; t0 + u - (l.r >> shift) < end; u += step) {
            if (u != first) part.load(mine, min(t0 + u, stop - 1) * kUnit + 8 * l.q, m.C);
            Piece a[4][P];
            const float power = convert(part.x, a);
            if (t0 + u >= end) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int p = 0; p < P; ++p)
                    lds[((((u * 4 + j) * P + p) * 4 + l.q) << shift) + row] = *reinterpret_cast<uint4 *>(a[j][p].w);
            if (kPowers && l.q == 0)
                for (int i = row; i < 16; i += rows) powers[u * 16 + i] = power;
        }
        __syncthreads();
        if (end < stop) part.load(mine, min(end + first, stop - 1) * kUnit + 8 * l.q, m.C);

        // a batch of units from t on with what is there, the next one on its way
        auto batch = [&](int t, const Units<J, AHEAD> &with, Units<J, AHEAD> &next) {
            const bool same = t + AHEAD * cut.shares < end;
            fetch(next, same ? t + AHEAD * cut.shares : min(end + share, stop - 1), same ? end : min(end + cut.chunk, stop));
            __builtin_amdgcn_sched_barrier(0);  // they set out before the work below, not after it
#pragma unroll
            for (int d = 0; d < AHEAD; ++d) {
                if (t + d * cut.shares >= end) break;
                const int u = t - t0 + d * cut.shares;
                half8 a[4][P];
                const uint4 *from = lds + (((u * 16 * P + l.q) << shift) + row);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int p = 0; p < P; ++p) a[j][p] = *reinterpret_cast<const half8 *>(from + ((4 * (j * P + p)) << shift));
                float4v power;
                if (kPowers) power = *reinterpret_cast<const float4v *>(powers + u * 16 + 4 * l.q);
                const uint32_t c[4] = {with.code[d].x, with.code[d].y, with.code[d].z, with.code[d].w};
                float4v sum{};
#pragma unroll
                for (int g = 0; g < 4 / J; ++g) {
                    float4v acc[P] = {};
                    const Expand::Zero zero = Expand::zero(with.word[d][g]);
#pragma unroll
                    for (int j = g * J; j < g * J + J; ++j) {
                        const half8 b = expand(c[j], zero);
#pragma unroll
                        for (int p = 0; p < P; ++p) acc[p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[j][p], b, acc[p], 0, 0, 0);
                    }
                    const float s = __uint_as_float(with.word[d][g] & ~15u);
                    if constexpr (P > 1)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[0][i] = fmaf(acc[1][i], 1 / kSecond, acc[0][i]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = g ? fmaf(s, acc[0][i], sum[i]) : s * acc[0][i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = kPowers ? fmaf(sum[i], power[i], out[i]) : out[i] + sum[i];
            }
        };
        for (int t = t0 + share; t < end; t += AHEAD * cut.shares) {
            batch(t, now, next);
            t += AHEAD * cut.shares;
            if (t >= end) {
                now = next;
                break;
            }
            batch(t, next, now);
        }
    }
    __syncthreads();
    // [shares][16 rows][tiles][16]
    float *sums = reinterpret_cast<float *>(lds);
    const int wide = 16 * cut.tiles, all = 16 * wide;
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[share * all + (4 * l.q + i) * wide + tile * 16 + l.r] = out[i];
    __syncthreads();
    const int have = min(16, M - row0);
    for (int e = tid; e < have * wide; e += waves * 64) {
        float v = 0.f;
        for (int w = 0; w < cut.shares; ++w) v += sums[w * all + e];
        const int o = blockIdx.x * wide + e % wide;
        if (o >= m.O) continue;
        const int64_t to = (int64_t)(row0 + e / wide) * m.O + o;
        if (cut.splits > 1) {
            parts[(int64_t)blockIdx.z * M * m.O + to] = v;
            continue;
        }
        if (bias) v += bias[o];
        y[to] = (Y)(silu_on ? silu(v) : v);
    }
}

// The splits' sums, in their order.
template <class Y>
__global__ __launch_bounds__(256) void k_w4_join(const float *__restrict__ parts, int32_t splits, int32_t M, int32_t O,
                                                 const float *__restrict__ bias, int32_t silu_on, Y *__restrict__ y) {
    const int n = M * O, e = blockIdx.x * 256 + threadIdx.x;
    if (e >= n) return;
    float v = 0.f;
#pragma unroll 8
    for (int i = 0; i < splits; ++i) v += parts[(int64_t)i * n + e];
    if (bias) v += bias[e % O];
    y[e] = (Y)(silu_on ? silu(v) : v);
}

// Bytes of LDS for a chunk, and for the sums behind it.
template <class T>
int lds_bytes(const Cut &c) {
    return std::max(c.chunk * ((256 * kPieces<T> << c.row_shift) + 64), c.tiles * c.shares * 1024);
}

template <class T>
Cut cut_of(int32_t M, const W4 &m, int tiles, int shares, int splits) {
    Cut c{tiles, shares, splits, 0, 0};
    while (c.row_shift < 4 && (1 << c.row_shift) < M) c.row_shift += 2;
    const int step = tiles * shares * (16 >> c.row_shift), units = (m.T + splits - 1) / splits;  // step: units that the wavefronts bring at once
    // as many times that as fit, in parts alike: what is alone on a CU, by its number or by its registers, may have most of the LDS
    const int64_t groups = (int64_t)((m.R + tiles - 1) / tiles) * ((M + 15) / 16) * splits;
    const int most = std::max((groups <= 256 || tiles * shares > 6 ? 131072 : 65536) / lds_bytes<T>({tiles, shares, splits, step, c.row_shift}), 1);
    const int parts = (units + most * step - 1) / (most * step), each = (units + parts - 1) / parts;
    c.chunk = (each + step - 1) / step * step;
    return c;
}

// Wavefronts share the rows' conversion: tiles such that workgroups fill the 256 CUs in few rounds and wavefronts the four SIMDs
// of each alike (64 x 8192 -> 28672 bf16 a twelfth less with twelve tiles than with eight), and the units cut among what is left:
// of twelve for few rows (3 x 7997 -> 22282 bf16 28 us with six wavefronts, 22 with twelve; 1 x 4096 -> 16384 9.5 with eight, 11 with
// sixteen), in at most four parts where they take several chunks (35 x 9158 -> 1901 bf16 19 in four, 22 in eight).
// Where that leaves more than half of the CUs without work and units enough to pay for a second kernel, every tile's units are
// split among workgroups (29 x 6477 -> 103 fp32 23 us in one part, 8 in eight; 2 x 19840 -> 30 bf16 18 and 7; at 20 units they are
// level): 6 to a part, which take one conversion, or 10 of few rows.
struct Ways {
    int tiles, shares, splits;
};
Ways ways_for(int32_t M, int32_t R, int32_t T, int most) {
    const int64_t blocks = (M + 15) / 16, all = R * blocks;
    int tiles = 1, shares = 1, splits = 1;
    double least = 1e30;
    for (int t = 1; t <= most; ++t) {
        // rounds of the CUs (many even out), times a tile's work on a SIMD and the rows' conversion, as long for 16 rows
        const double groups = (double)((R + t - 1) / t * blocks) / 256, rounds = groups > 2 ? groups : std::ceil(groups);
        const double cost = rounds * ((t + 3) / 4 + (M > 4 ? 1 : 0.25)) + 1e-3 * rounds;  // of equals the fewest rounds
        if (cost < least) least = cost, tiles = t;
    }
    while (shares * 2 * tiles <= (M > 4 ? most : 12) && shares * 2 <= std::min(T, M > 4 && T > 24 ? 4 : 8)) shares *= 2;
    // one conversion for all units (10: the most that was measured)
    if (M > 4 && T <= 10 && tiles > 1 && tiles * shares < T) tiles = (T + shares - 1) / shares;
    if (all < 128 && T >= (M > 4 ? 20 : 48)) {
        splits = (int)(M > 4 ? std::min<int64_t>(512 / all, T / 6) : std::min<int64_t>(256 / all, T / 10));
        for (shares = 1; shares * 2 <= (M > 4 ? 4 : 8) && shares * 2 * splits <= T;) shares *= 2;
    }
    return {tiles, shares, splits};
}

// Whether the codes go past the caches.  The 256 MB next to memory seldom hold weights of 100 MB until their next use, and reads
// that leave no lines there are faster: bf16 1 x 8192 -> 28672 23.8 us against 26.2, four rows 26.7 and 27.8, 131072 outputs 100 and
// 106.  Smaller weights that are used again at once lose (1 x 8192 -> 16384 16.2 and 15.4), more than 16 rows read them several
// times, and fp32 rows are not bound by them (30.8 and 29.0).
bool read_once(int32_t M, const W4 &m) { return M <= 16 && m.units() >= 100000000 / 1024; }

template <class F>
void by_group(int32_t group, F f) {
    group == 32 ? f(std::integral_constant<int, 1>{}) : group == 64 ? f(std::integral_constant<int, 2>{}) : f(std::integral_constant<int, 4>{});
}

}  // namespace

hipError_t launch_w4_pack(const void *w, int32_t dtype, int64_t w_row, const W4 &m, hipStream_t st) {
    by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        by_group(m.group, [&](auto j) {
            k_w4_pack<T, j.value><<<(unsigned)m.R * ((m.T + 3) / 4), 256, 0, st>>>(static_cast<const T *>(w), w_row, m);
        });
    });
    return hipGetLastError();
}

hipError_t launch_w4_unpack(const W4 &m, int32_t dtype, void *w, hipStream_t st) {
    by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        const bool past = (reinterpret_cast<uintptr_t>(w) | (uint64_t)m.C * sizeof(T)) % 128 == 0;
        by_group(m.group, [&](auto j) {
            k_w4_unpack<T, j.value><<<(unsigned)m.R * ((m.T + 3) / 4), 256, 0, st>>>(m, static_cast<T *>(w), past);
        });
    });
    return hipGetLastError();
}

size_t w4_matvec_workspace_bytes(int32_t M, const W4 &m) {
    const Ways w = ways_for(M, m.R, m.T, 10);  // (splits are for few tiles, whatever the type)
    return w.splits > 1 ? (size_t)w.splits * M * m.O * sizeof(float) : 0;
}

hipError_t launch_w4_matvec(const W4Product &p, const W4 &m, void *workspace, hipStream_t st) {
    hipError_t e = hipSuccess;
    float *parts = static_cast<float *>(workspace);
    by_dtype(p.dtype, [&](auto xt) {
        using T = decltype(xt);
        const Ways w = ways_for(p.M, m.R, m.T, kMaxWaves<T>);
        const Cut c = cut_of<T>(p.M, m, w.tiles, w.shares, w.splits);
        by_output<T>(p.out_dtype, [&](auto yt) {
            using Y = decltype(yt);
            Y *y = static_cast<Y *>(p.y);
            by_group(m.group, [&](auto j) {
                constexpr int J = decltype(j)::value;
                const dim3 grid((m.R + c.tiles - 1) / c.tiles, (p.M + 15) / 16, c.splits);
                auto go = [&](auto shift, auto once) {
                    constexpr int S = decltype(shift)::value;
                    constexpr bool ONCE = decltype(once)::value;
                    e = DGQ_ENSURE_LDS((k_w4_matvec<T, Y, J, S, ONCE>), lds_bytes<T>(c));
                    if (e == hipSuccess)
                        k_w4_matvec<T, Y, J, S, ONCE><<<grid, 64 * c.tiles * c.shares, lds_bytes<T>(c), st>>>(
                            static_cast<const T *>(p.x), p.x_row, p.M, m, c, p.bias, p.act == DGQ_ACT_SILU, y, parts);
                };
                auto by_rows = [&](auto once) {
                    c.row_shift == 0   ? go(std::integral_constant<int, 0>{}, once)
                    : c.row_shift == 2 ? go(std::integral_constant<int, 2>{}, once)
                                       : go(std::integral_constant<int, 4>{}, once);
                };
                if constexpr (sizeof(T) == 2) {
                    if (read_once(p.M, m)) return by_rows(std::true_type{});
                }
                by_rows(std::false_type{});
            });
            if (e == hipSuccess && c.splits > 1)
                k_w4_join<Y><<<(p.M * m.O + 255) / 256, 256, 0, st>>>(parts, c.splits, p.M, m.O, p.bias, p.act == DGQ_ACT_SILU, y);
        });
    });
    return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace dgq
