// Cross-attention to ragged rows of the 8-bit cache (k5_kv.hip).
//
// With codes c, block scales s_k, s_v and a query q of head width d, over the rows j of its request:
//   l_j = s_k (q . c_j) / sqrt(d),   out = sum_j p_j s_v c'_j,   p = softmax(l).
// One pass with a running maximum.  The value scale joins the exponent, so a block's scale costs nothing per element:
//   t_j = l_j log2(e) + log2(s_v),  M = running max of t,  u_j = 2^(t_j - M),
//   O = sum u_j c'_j,  D = sum u_j / s_v,  out = O / D,
// and u_j is at most 1 in units of what its row adds, whatever the blocks' scales are.  (A block of zero values takes the
// largest scale seen so far in its place: its O is 0 with any, its share of D is right with any.)
//
// Codes are exact in fp16.  Queries are multiplied by a power of two that brings the row's largest element to
// [2^14, 2^15): an fp16 or bf16 query is then exact in one fp16 (bf16 elements below 2^-28 of the row's largest lose
// bits), an fp32 query is two (22 bits).  u is rounded to one fp16 for 16-bit outputs (2^-11; D sums the
// rounded ones, so a row that takes most of the weight adds no error), to two for fp32 ones.  Sums are fp32.
#include <cfloat>
#include <type_traits>

#include "dgq_internal.h"

namespace dgq {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float8v __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoMax = -1e30f;   // M before the first row: finite, so that M - M stays 0
constexpr float kLift = 6.f;       // u carries 2^6, away from fp16's subnormals
constexpr float kSlack = 8.f;      // M is raised only when a row exceeds it by 2^8: u stays below 2^15
constexpr float kLargeMax = 0x1p18f;

struct AttnArgs {
    KvQueries q;
    KvCache c;
    const int32_t *table, *lengths;
    void *out;
    float *part;     // splits > 1: [splits][rows * Hq][d], then (M, D) [splits][rows * Hq][2]
    int32_t width, G, splits, tiles;  // tiles: row tiles of all requests together (a bound when packed)
};

// 8 bytes (code + 128) -> 8 fp16: 0x6400 | byte is 1024 + byte exactly.
__device__ half8 to_half8(uint32_t lo, uint32_t hi) {
    uint32_t w[4] = {__builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u),
                     __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)};
    half8 r;
    for (int i = 0; i < 4; ++i) {
        const half2v h = __builtin_bit_cast(half2v, w[i]) - half2v{(_Float16)1152.f, (_Float16)1152.f};
        r[2 * i] = h[0], r[2 * i + 1] = h[1];
    }
    return r;
}

// 8 elements of a query, 4 of an output: 16-byte aligned, 4-element aligned
__device__ float8v load8(const float *p) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    return float8v{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}
__device__ float8v load8(const _Float16 *p) { return __builtin_convertvector(*reinterpret_cast<const half8 *>(p), float8v); }
__device__ float8v load8(const __bf16 *p) {
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    float8v r;
    r[0] = __uint_as_float(w.x << 16), r[1] = __uint_as_float(w.x & 0xffff0000u);
    r[2] = __uint_as_float(w.y << 16), r[3] = __uint_as_float(w.y & 0xffff0000u);
    r[4] = __uint_as_float(w.z << 16), r[5] = __uint_as_float(w.z & 0xffff0000u);
    r[6] = __uint_as_float(w.w << 16), r[7] = __uint_as_float(w.w & 0xffff0000u);
    return r;
}
template <class T>
__device__ void store4(T *p, float a, float b, float c, float d) {
    typedef T vec __attribute__((ext_vector_type(4)));
    *reinterpret_cast<vec *>(p) = vec{(T)a, (T)b, (T)c, (T)d};
}

struct Rows {  // of one request
    int32_t b;
    int64_t first;  // of all queries' rows
    int32_t n;      // queries
    int32_t tile;   // row tile within the request
};

// The request that row tile `t` belongs to; n = 0: none.
__device__ Rows find_rows(const AttnArgs &a, int32_t t) {
    const int lane = threadIdx.x & 63;
    if (!a.q.offsets) {
        const int32_t per = (int32_t)(((int64_t)a.q.N * a.G + 31) / 32);
        const int32_t b = t / per;
        return {b, (int64_t)b * a.q.N, a.q.N, t - b * per};
    }
    int64_t seen = 0;
    for (int b0 = 0; b0 < a.q.B; b0 += 64) {
        const int b = b0 + lane;
        int32_t lo = 0, n = 0;
        if (b < a.q.B) {
            lo = min(max(a.q.offsets[b], 0), a.q.N);
            n = max(min(a.q.offsets[b + 1], a.q.N) - lo, 0);
        }
        const int64_t mine = ((int64_t)n * a.G + 31) / 32;
        int64_t ends = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t x = __shfl_up(ends, o);
            if (lane >= o) ends += x;
        }
        const uint64_t above = __ballot(seen + ends > t);
        if (above) {
            const int l = __ffsll((unsigned long long)above) - 1;
            return {b0 + l, __shfl(lo, l), __shfl(n, l), (int32_t)(t - seen - __shfl(ends - mine, l))};
        }
        seen += __shfl(ends, 63);
    }
    return {0, 0, 0, 0};
}

__device__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ float other_half(float x) { return __shfl_xor(x, 32); }

// One wavefront: 32 rows (a row is a query and one of the G heads that share a cached head) against the tiles of one
// split of the request's rows.  S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 instructions: a lane holds column
// (lane & 31) of both, so a row's statistics are its lane's (and the other half's), and the products of S^T are the
// operand of O^T without a move, with V's slots stored in the order in which S^T leaves them.
// T: type of q and out.  NP: 32-dim steps of the head width.
template <class T, int NP>
__global__ __launch_bounds__(256) void k_xattn_kv(AttnArgs a) {
    constexpr bool kTwo = std::is_same<T, float>::value;  // two fp16 pieces
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int d = a.c.d, e16 = kv_padded(d), S = a.c.S, H = a.c.H;
    // waves of a workgroup: neighbouring splits, then row tiles, of one head
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int split = (int)(wave % a.splits);
    const int64_t task = wave / a.splits;
    const int h = (int)(task / a.tiles);
    if (h >= H) return;
    const Rows rows = find_rows(a, (int32_t)(task % a.tiles));
    if (rows.n == 0) return;
    const int64_t length = min((int64_t)max(a.lengths[rows.b], 0), (int64_t)a.width * S);
    const int32_t n_tiles = (int32_t)((length + 31) / 32), per = (n_tiles + a.splits - 1) / a.splits;
    const int32_t t0 = split * per, t1 = min(t0 + per, n_tiles);
    if (a.splits > 1 && t0 >= t1) return;  // the join knows which splits hold something

    // ---- the queries ----
    const int64_t m = (int64_t)rows.tile * 32 + col;  // row of the request
    const bool live = m < (int64_t)rows.n * a.G;
    const int64_t n = live ? m / a.G : 0;
    const int head = h * a.G + (int)(live ? m - n * a.G : 0);
    const int64_t at = a.q.offsets ? (rows.first + n) * a.q.row : rows.b * a.q.batch + n * a.q.row;
    const T *q = static_cast<const T *>(a.q.q) + at + head * a.q.head;
    half8 qh[2 * NP], ql[kTwo ? 2 * NP : 1];
    float q_scale;
    {
        float8v x[2 * NP];
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < 2 * NP; ++s) {
            const int e = (s >> 1) * 32 + half * 16 + (s & 1) * 8;
            x[s] = live && e < d ? load8(q + e) : float8v(0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[s][i]) & 0x7fffffffu);
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        // 2^up brings the largest to [2^14, 2^15); a row that is not finite gives NaN throughout
        const int up = min(14 + 127 - (int)(top >> 23), 126);
        const float lift = top ? __uint_as_float((uint32_t)(127 + up) << 23) : 1.f;
        q_scale = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : 1.f / lift;
        q_scale *= kLog2e / sqrtf((float)d);
#pragma unroll
        for (int s = 0; s < 2 * NP; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = x[s][i] * lift;
                const _Float16 hi = (_Float16)y;
                qh[s][i] = hi;
                if constexpr (kTwo) ql[s][i] = (_Float16)(y - (float)hi);
            }
    }

    // ---- the rows ----
    float16v O[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[i][r] = 0.f;
    float M = kNoMax, D = 0.f, v_top = 0.f;
    const int32_t *entries = a.table + (int64_t)rows.b * a.width;
    for (int32_t t = t0; t < t1; ++t) {
        const int32_t block = entries[t * 32 / S];
        if (block < 0 || block >= a.c.n_blocks) continue;
        const int64_t slice = (int64_t)block * H + h;
        const uint8_t *tile = a.c.codes + slice * kv_slice_bytes(S, d) + (int64_t)(t * 32 % S / 32) * 64 * e16;
        const float2 scale = reinterpret_cast<const float2 *>(a.c.scales)[slice];

        uint4 kw[NP], vw[NP];
#pragma unroll
        for (int s = 0; s < NP; ++s)  // a last half that is not there reads V's first bytes, against zeros of q
            kw[s] = *reinterpret_cast<const uint4 *>(tile + ((2 * s + half) * 32 + col) * 16);
#pragma unroll
        for (int s = 0; s < NP; ++s)  // dims that are not there repeat the last one; nothing reads their sums
            vw[s] = *reinterpret_cast<const uint4 *>(tile + 32 * e16 + min(s * 32 + col, e16 - 1) * 32 + half * 16);

        float16v x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = 0.f;
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            const half8 k0 = to_half8(kw[s].x, kw[s].y), k1 = to_half8(kw[s].z, kw[s].w);
            x = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, qh[2 * s], x, 0, 0, 0);
            x = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, qh[2 * s + 1], x, 0, 0, 0);
            if constexpr (kTwo) {
                x = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, ql[2 * s], x, 0, 0, 0);
                x = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, ql[2 * s + 1], x, 0, 0, 0);
            }
        }

        v_top = scale.y > v_top ? scale.y : v_top;
        float s_v = scale.y == 0.f ? v_top : scale.y;
        if (s_v == 0.f) s_v = 1.f;
        const float mult = q_scale * scale.x, shift = __builtin_amdgcn_logf(s_v);
        const int left = (int)min(length - (int64_t)t * 32, (int64_t)32);  // rows of this tile
        if (left < 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + 4 * half + (r & 3) >= left) x[r] = -FLT_MAX;
        }
        float top = x[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
        top = fmaf(fmaxf(top, other_half(top)), mult, shift);  // mult is not negative
        if (__any(top > M + kSlack)) {
            const float to = fmaxf(M, top), less = exp2_of(M - to);
            M = to;
            D *= less;
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) O[i][r] *= less;
        }
        // One rounding, next to M; M's own is common to all rows.  Where it could reach 1, t is rounded before M is taken off.
        const float off = shift - M + kLift;
        if (__any(fabsf(M) > kLargeMax)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = exp2_of(fmaf(x[r], mult, shift) - M + kLift);
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = exp2_of(fmaf(x[r], mult, off));
        }
        if (left < 32) {  // whatever stood there, and whatever it became with a scale of 0
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + 4 * half + (r & 3) >= left) x[r] = 0.f;
        }
        half8 ph[2], pl[2];
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            const half2v hi = __builtin_convertvector(float2v{x[r], x[r + 1]}, half2v);
            ph[r >> 3][r & 7] = hi[0], ph[r >> 3][(r & 7) + 1] = hi[1];
            if constexpr (kTwo) {
                const half2v lo = __builtin_convertvector(float2v{x[r] - (float)hi[0], x[r + 1] - (float)hi[1]}, half2v);
                pl[r >> 3][r & 7] = lo[0], pl[r >> 3][(r & 7) + 1] = lo[1];
            }
        }
        // One fp16: the sum of what is multiplied, so that a lone large u rounds without an error in out.  That needs every u
        // that counts in D among fp16's normals: beside the values of a block of a far larger scale it may not be, while its
        // weight is all of D.
        if (kTwo || s_v < v_top * 0x1p-6f) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += x[r];
        } else {
#pragma unroll
            for (int r = 0; r < 16; r += 2)
                sum = __builtin_amdgcn_fdot2(half2v{ph[r >> 3][r & 7], ph[r >> 3][(r & 7) + 1]},
                                             half2v{(_Float16)1.f, (_Float16)1.f}, sum, false);
        }
        D = fmaf(sum, 1.f / s_v, D);
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            const half8 v0 = to_half8(vw[s].x, vw[s].y), v1 = to_half8(vw[s].z, vw[s].w);
            O[s] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v0, ph[0], O[s], 0, 0, 0);
            O[s] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v1, ph[1], O[s], 0, 0, 0);
            if constexpr (kTwo) {
                O[s] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v0, pl[0], O[s], 0, 0, 0);
                O[s] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v1, pl[1], O[s], 0, 0, 0);
            }
        }
    }
    D += other_half(D);
    if (!live) return;

    const int64_t row = (rows.first + n) * a.q.Hq + head;
    if (a.splits > 1) {
        const int64_t all = a.q.rows() * a.q.Hq, p = split * all + row;
        float *to = a.part + p * d;
#pragma unroll
        for (int s = 0; s < NP; ++s)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int e = s * 32 + 8 * (r >> 2) + 4 * half;
                if (e < d) *reinterpret_cast<float4 *>(to + e) = float4{O[s][r], O[s][r + 1], O[s][r + 2], O[s][r + 3]};
            }
        if (half == 0) reinterpret_cast<float2 *>(a.part + a.splits * all * d)[p] = float2{M, D};
        return;
    }
    const float inv = D == 0.f ? 0.f : 1.f / D;
    T *to = static_cast<T *>(a.out) + row * d;
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int e = s * 32 + 8 * (r >> 2) + 4 * half;
            if (e < d)
                store4(to + e, O[s][r] * inv, O[s][r + 1] * inv, O[s][r + 2] * inv, O[s][r + 3] * inv);
        }
}

// The splits of one row (query and head) added up: out = sum 2^(M_i - M) O_i / sum 2^(M_i - M) D_i.
template <class T>
__global__ __launch_bounds__(256) void k_xattn_kv_join(AttnArgs a) {
    const int d = a.c.d, lane = threadIdx.x & 63;
    const int64_t all = a.q.rows() * a.q.Hq, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= all) return;
    const int64_t n = row / a.q.Hq;
    int32_t b = -1;
    if (!a.q.offsets) {
        b = (int32_t)(n / a.q.N);
    } else {
        for (int i = lane; i < a.q.B && b < 0; i += 64)
            if (a.q.offsets[i] <= n && n < a.q.offsets[i + 1]) b = i;
        const uint64_t found = __ballot(b >= 0);
        if (!found) return;  // a row that no request has is left as it was
        b = __shfl(b, __ffsll((unsigned long long)found) - 1);
    }
    const int64_t length = min((int64_t)max(a.lengths[b], 0), (int64_t)a.width * a.c.S);
    const int32_t n_tiles = (int32_t)((length + 31) / 32), per = (n_tiles + a.splits - 1) / a.splits;
    const int active = per ? (n_tiles + per - 1) / per : 0;
    const float2 *stats = reinterpret_cast<const float2 *>(a.part + a.splits * all * d) + row;
    float M = kNoMax;
    for (int i = 0; i < active; ++i) M = fmaxf(M, stats[i * all].x);
    float D = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < active; ++i) {
        const float2 s = stats[i * all];
        const float w = exp2_of(s.x - M);
        D = fmaf(w, s.y, D);
        for (int j = 0; j < 4; ++j)
            if (lane + 64 * j < d) o[j] = fmaf(w, a.part[(i * all + row) * d + lane + 64 * j], o[j]);
    }
    const float inv = D == 0.f ? 0.f : 1.f / D;
    T *to = static_cast<T *>(a.out) + row * d;
    for (int j = 0; j < 4; ++j)
        if (lane + 64 * j < d) to[lane + 64 * j] = (T)(o[j] * inv);
}

struct Plan {
    int32_t tiles, splits;
};

// Row tiles, and into how many parts each request's rows are split: only where the tiles alone leave the chip's
// 256 x 8 wavefronts empty, and no part below four tiles of 32 rows.
Plan plan_of(int32_t B, int64_t rows, bool packed, int32_t Hq, int32_t Hkv, int64_t slots) {
    const int64_t G = Hq / Hkv;
    const int64_t tiles = packed ? rows * G / 32 + B : B * ((rows / B * G + 31) / 32);
    const int64_t waves = tiles * Hkv;
    const int64_t most = std::max<int64_t>(1, slots / 128);
    const int64_t want = 2048 / std::max<int64_t>(1, waves);
    return {(int32_t)tiles, (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min(want, most), 256))};
}

template <class T>
hipError_t launch(const AttnArgs &a, hipStream_t st) {
    const int64_t waves = (int64_t)a.tiles * a.c.H * a.splits;
    const dim3 grid((uint32_t)((waves + 3) / 4));
    auto go = [&](auto np) { k_xattn_kv<T, decltype(np)::value><<<grid, 256, 0, st>>>(a); };
    switch ((a.c.d + 31) / 32) {
        case 1: go(std::integral_constant<int, 1>{}); break;
        case 2: go(std::integral_constant<int, 2>{}); break;
        case 3: go(std::integral_constant<int, 3>{}); break;
        case 4: go(std::integral_constant<int, 4>{}); break;
        case 5: go(std::integral_constant<int, 5>{}); break;
        case 6: go(std::integral_constant<int, 6>{}); break;
        case 7: go(std::integral_constant<int, 7>{}); break;
        default: go(std::integral_constant<int, 8>{}); break;
    }
    if (a.splits > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int64_t all = a.q.rows() * a.q.Hq;
        k_xattn_kv_join<T><<<(uint32_t)((all + 3) / 4), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

size_t xattn_kv_workspace_bytes(int32_t B, int64_t rows, bool packed, int32_t Hq, int32_t Hkv, int32_t d, int64_t slots) {
    const Plan p = plan_of(B, rows, packed, Hq, Hkv, slots);
    return p.splits > 1 ? (size_t)p.splits * rows * Hq * (d + 2) * sizeof(float) : 0;
}

hipError_t launch_xattn_kv(const KvQueries &q, const KvCache &c, const int32_t *table, int32_t width,
                           const int32_t *lengths, void *out, void *workspace, hipStream_t st) {
    const Plan p = plan_of(q.B, q.rows(), q.offsets != nullptr, q.Hq, c.H, (int64_t)width * c.S);
    const AttnArgs a{q, c, table, lengths, out, static_cast<float *>(workspace), width, q.Hq / c.H, p.splits, p.tiles};
    return q.dtype == DGQ_F32 ? launch<float>(a, st) : q.dtype == DGQ_F16 ? launch<_Float16>(a, st) : launch<__bf16>(a, st);
}

}  // namespace dgq
