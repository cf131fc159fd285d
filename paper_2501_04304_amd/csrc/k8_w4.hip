// Weights in 4 bits with a scale and a zero for every group of 32, 64 or 128 inputs, and their products with few rows.
//
// Per output and group:  lo = min(0, min w), hi = max(0, max w), s = (hi - lo) * (1/15) with the 4 lowest bits of its pattern
// cleared (0 below 2^-96), zero = clamp(rne(-lo / s), 0, 15), code = clamp(rne(w / s) + zero, 0, 15) (both quotients times 1/s),
// value s (code - zero).  The layout (include/dgq.h) is the product's: a unit is 16 outputs x 128 inputs, 1 KiB of codes of which
// a lane's 16 bytes are its part of four operands of the 16 x 16 x 32 matrix instructions, and behind all codes one word for each
// group, its scale with the zero in the 4 lowest bits.
#include <algorithm>

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

// Inputs k .. k + 7 of a row, those from C on 0.
template <class T>
__device__ void load_eight(const T *row, int k, int C, float (&f)[8]) {
    constexpr int V = kVec<T>;
#pragma unroll
    for (int v = 0; v < 8 / V; ++v) {
        float part[V];
        load_vector(row + k + v * V, C - k - v * V, part);
#pragma unroll
        for (int i = 0; i < V; ++i) f[v * V + i] = part[i];
    }
}

// nibble of input i (0 .. 7) of a lane's word
__device__ constexpr int nibble(int i) { return i % 2 ? 4 + i / 2 : i / 2; }

// over the lanes of a row
__device__ float row_min(float x) { return x = fminf(x, __shfl_xor(x, 16)), fminf(x, __shfl_xor(x, 32)); }
__device__ float row_max(float x) { return x = fmaxf(x, __shfl_xor(x, 16)), fmaxf(x, __shfl_xor(x, 32)); }

// ---- packing ---------------------------------------------------------------------------------------------------------
// A wavefront per unit.  Bound by the bytes of w.
template <class T, int J>  // J: words of 32 inputs in a group
__global__ __launch_bounds__(256) void k_w4_pack(const T *__restrict__ w, int64_t w_row, W4 m) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= m.units()) return;
    const Lane l;
    const int o = (int)(unit / m.T) * 16 + l.r, k0 = (int)(unit % m.T) * kUnit + l.q * 8;
    const T *row = w + o * w_row;
    float f[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (o < m.O) load_eight(row, k0 + 32 * j, m.C, f[j]);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) f[j][i] = 0.f;
    }
    uint32_t code[4], word[4 / J];
#pragma unroll
    for (int g = 0; g < 4 / J; ++g) {
        float lo = 0.f, hi = 0.f, none = 0.f;  // none: NaN once a weight is not finite
#pragma unroll
        for (int j = g * J; j < g * J + J; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lo = fminf(lo, f[j][i]);
                hi = fmaxf(hi, f[j][i]);
                none = fmaf(f[j][i], 0.f, none);
            }
        lo = row_min(lo), hi = row_max(hi);
        none += __shfl_xor(none, 16);
        none += __shfl_xor(none, 32);
        const float all = hi - lo;
        const bool bad = !(all <= 0x1.fffffep127f) || none != none;
        float s = __uint_as_float(__float_as_uint(all * (float)(1.0 / 15)) & ~15u);
        if (!(s >= kLeastScale)) s = 0.f;
        const float inv = s > 0.f ? 1.0f / s : 0.f, zero = fminf(fmaxf(rintf(-lo * inv), 0.f), 15.f);
        word[g] = bad ? kNaNWord : __float_as_uint(s) | (uint32_t)zero;
#pragma unroll
        for (int j = g * J; j < g * J + J; ++j) {
            code[j] = 0;
            if (bad) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                code[j] |= (uint32_t)fminf(fmaxf(rintf(f[j][i] * inv) + zero, 0.f), 15.f) << (4 * nibble(i));
        }
    }
    reinterpret_cast<uint4 *>(m.codes)[unit * 64 + (threadIdx.x & 63)] = uint4{code[0], code[1], code[2], code[3]};
    if (l.q == 0)
#pragma unroll
        for (int g = 0; g < 4 / J; ++g) m.words()[(unit * 16 + l.r) * (4 / J) + g] = word[g];
}

template <class T, int J>
__global__ __launch_bounds__(256) void k_w4_unpack(W4 m, T *__restrict__ w) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= m.units()) return;
    const Lane l;
    const int o = (int)(unit / m.T) * 16 + l.r, k0 = (int)(unit % m.T) * kUnit + l.q * 8;
    if (o >= m.O) return;
    const uint4 all = reinterpret_cast<const uint4 *>(m.codes)[unit * 64 + (threadIdx.x & 63)];
    const uint32_t code[4] = {all.x, all.y, all.z, all.w};
    T *row = w + (int64_t)o * m.C;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t word = m.words()[(unit * 16 + l.r) * (4 / J) + j / J];
        const float s = __uint_as_float(word & ~15u);
        constexpr int V = kVec<T>;
        const int zero = word & 15;
#pragma unroll
        for (int v = 0; v < 8 / V; ++v) {
            float f[V];
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = (float)((int)(code[j] >> (4 * nibble(v * V + i)) & 15) - zero) * s;
            const int k = k0 + 32 * j + v * V;
            store_vector(row + k, m.C - k, f);
        }
    }
}

// ---- products --------------------------------------------------------------------------------------------------------
//   y[m, o] = sum_g s (sum_{k in g} x[m, k] (code - zero))
// on the matrix cores, 16 rows of x by 16 outputs by 32 inputs, in fp16.  A code becomes 1 + code / 16 by its place below the
// exponent of 1 (two instructions for a pair), and less 1 + zero / 16 it is (code - zero) / 16, exactly.  Rows of fp16 are what
// they are; those of bf16 and fp32 are taken a unit (128 inputs) at a time by a power of two that brings its largest to 2^14 .. 2^15,
// bf16 as one fp16, fp32 as two (x = h + l, each rounded to nearest: off by 2^-23 x at most); what lies 2^29 below the unit's
// largest loses bits, to 2^-39 of that.  The groups' sums meet in fp32 with their scales and those powers.
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

// (code - zero) / 16 of a lane's eight codes; less: -(1 + zero / 16), twice
__device__ Piece expand(uint32_t code, half2v less) {
    Piece p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p.w[i] = ((i < 2 ? code << (6 - 4 * i) : code >> (4 * i - 6)) & 0x03c003c0u) | 0x3c003c00u;
        p.p[i] += less;
    }
    return p;
}

// One row's part of a unit for a lane (four times eight inputs), and what its sums are to be multiplied by.
template <class T>
struct RowPart {
    Piece a[4][kPieces<T>];
    float power;
    __device__ void load(const T *row, int k0, int C) {
        if constexpr (std::is_same_v<T, _Float16>) {
            power = 1.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = k0 + 32 * j;
                if (k + 8 <= C) a[j][0].all = *reinterpret_cast<const loose<T, 8> *>(row + k);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) a[j][0].all[i] = k + i < C ? row[k + i] : (T)0.f;
            }
        } else {
            float f[4][8], top = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) load_eight(row, k0 + 32 * j, C, f[j]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[j][i]));
            const int e = max((int)(__float_as_uint(row_max(top)) >> 23), 15);  // 15: 2^-112
            const float down = __uint_as_float((uint32_t)(268 - e) << 23);     // 2^(14 - (e - 127)); e = 255 (infinity): 2^-114
            power = __uint_as_float((uint32_t)(e - 14) << 23);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2v v{f[j][2 * i] * down, f[j][2 * i + 1] * down};
#pragma unroll
                    for (int n = 0; n < kPieces<T>; ++n) {
                        a[j][n].p[i] = __builtin_convertvector(v, half2v);
                        if (n + 1 < kPieces<T>) v -= __builtin_convertvector(a[j][n].p[i], float2v);
                    }
                }
        }
    }
};

// A wavefront of a workgroup takes a share of the units of 16 NT outputs, for 16 RT rows; their sums meet in LDS.
template <class T, class Y, int RT, int NT, int J>
__global__ __launch_bounds__(512) void k_w4_matvec(const T *__restrict__ x, int64_t x_row, int32_t M, W4 m,
                                                   const float *__restrict__ bias, int32_t silu_on, Y *__restrict__ y) {
    extern __shared__ float sums[];  // [waves][16 RT rows][16 NT]
    const int tid = threadIdx.x, waves = blockDim.x >> 6, wave = tid >> 6;
    const Lane l;
    const int tile0 = blockIdx.x * NT, row0 = blockIdx.y * 16 * RT;
    const T *rows[RT];
    int64_t unit0[NT];  // tiles behind the last are the last again, and not written
#pragma unroll
    for (int t = 0; t < RT; ++t) rows[t] = x + min(row0 + 16 * t + l.r, M - 1) * x_row;
#pragma unroll
    for (int n = 0; n < NT; ++n) unit0[n] = (int64_t)min(tile0 + n, m.R - 1) * m.T;
    float4v out[RT][NT] = {};
    const int t0 = (int)((int64_t)m.T * wave / waves), t1 = (int)((int64_t)m.T * (wave + 1) / waves);
    for (int t = t0; t < t1; ++t) {
        uint32_t code[NT][4], word[NT][4 / J];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint4 c = reinterpret_cast<const uint4 *>(m.codes)[(unit0[n] + t) * 64 + (tid & 63)];
            code[n][0] = c.x, code[n][1] = c.y, code[n][2] = c.z, code[n][3] = c.w;
#pragma unroll
            for (int g = 0; g < 4 / J; ++g) word[n][g] = m.words()[((unit0[n] + t) * 16 + l.r) * (4 / J) + g];
        }
        RowPart<T> part[RT];
        float power[RT][4];  // of the rows 4 q .. 4 q + 3, as the products' results lie
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            part[rt].load(rows[rt], t * kUnit + 8 * l.q, m.C);
#pragma unroll
            for (int i = 0; i < 4; ++i) power[rt][i] = std::is_same_v<T, _Float16> ? 1.f : __shfl(part[rt].power, 4 * l.q + i);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int g = 0; g < 4 / J; ++g) {
                const _Float16 z = (_Float16)fmaf((float)(word[n][g] & 15), -1.f / 16, -1.f);
                const float s = __uint_as_float(word[n][g] & ~15u);
                float4v acc[RT] = {};
#pragma unroll
                for (int j = g * J; j < g * J + J; ++j) {
                    const Piece b = expand(code[n][j], half2v{z, z});
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int p = 0; p < kPieces<T>; ++p)
                            acc[rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(part[rt].a[j][p].all, b.all, acc[rt], 0, 0, 0);
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[rt][n][i] = fmaf(s * acc[rt][i], power[rt][i], out[rt][n][i]);
            }
    }
    constexpr int W = 16 * NT, ALL = 16 * RT * W;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[wave * ALL + (16 * rt + 4 * l.q + i) * W + 16 * n + l.r] = out[rt][n][i];
    __syncthreads();
    for (int e = tid; e < ALL; e += blockDim.x) {
        float v = 0.f;
        for (int w = 0; w < waves; ++w) v += sums[w * ALL + e];
        const int row = row0 + e / W, o = tile0 * 16 + e % W;
        if (row >= M || o >= m.O) continue;
        v = bias ? fmaf(v, 16.f, bias[o]) : v * 16.f;
        y[(int64_t)row * m.O + o] = (Y)(silu_on ? silu(v) : v);
    }
}

template <class F>
void by_group(int32_t group, F f) {
    group == 32 ? f(std::integral_constant<int, 1>{}) : group == 64 ? f(std::integral_constant<int, 2>{}) : f(std::integral_constant<int, 4>{});
}

}  // namespace

hipError_t launch_w4_pack(const void *w, int32_t dtype, int64_t w_row, const W4 &m, hipStream_t st) {
    by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        by_group(m.group, [&](auto j) {
            k_w4_pack<T, j.value><<<(unsigned)((m.units() + 3) / 4), 256, 0, st>>>(static_cast<const T *>(w), w_row, m);
        });
    });
    return hipGetLastError();
}

hipError_t launch_w4_unpack(const W4 &m, int32_t dtype, void *w, hipStream_t st) {
    by_dtype(dtype, [&](auto t) {
        using T = decltype(t);
        by_group(m.group, [&](auto j) {
            k_w4_unpack<T, j.value><<<(unsigned)((m.units() + 3) / 4), 256, 0, st>>>(m, static_cast<T *>(w));
        });
    });
    return hipGetLastError();
}

hipError_t launch_w4_matvec(const W4Product &p, const W4 &m, hipStream_t st) {
    const int waves = std::min(m.T, 8);
    by_dtype(p.dtype, [&](auto xt) {
        using T = decltype(xt);
        by_output<T>(p.out_dtype, [&](auto yt) {
            using Y = decltype(yt);
            by_group(m.group, [&](auto j) {
                auto go = [&](auto rt) {
                    constexpr int RT = decltype(rt)::value, NT = 1;
                    const dim3 grid((m.R + NT - 1) / NT, (p.M + 16 * RT - 1) / (16 * RT));
                    k_w4_matvec<T, Y, RT, NT, decltype(j)::value><<<grid, 64 * waves, waves * RT * NT * 1024, st>>>(
                        static_cast<const T *>(p.x), p.x_row, p.M, m, p.bias, p.act == DGQ_ACT_SILU, static_cast<Y *>(p.y));
                };
                p.M <= 16 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 2>{});
            });
        });
    });
    return hipGetLastError();
}

}  // namespace dgq
