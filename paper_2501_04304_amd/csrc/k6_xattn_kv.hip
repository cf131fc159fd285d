// Cross-attention to ragged rows of the 8-bit cache (k5_kv.hip).
//
// With codes c, block scales s_k, s_v and a query q of head width d, over the rows j of its request:
//   l_j = s_k (q . c_j) / sqrt(d),   out = sum_j p_j s_v c'_j,   p = softmax(l).
// One pass with a running maximum.  The value scale joins the exponent, so a block's scale costs nothing per element:
//   t_j = l_j log2(e) + log2(s_v),  M = running max of t,  u_j = 2^(t_j - M),
//   O = sum u_j c'_j,  D = sum u_j / s_v,  out = O / D,
// and u_j is at most 1 in units of what its row adds, whatever the blocks' scales are.  (A block of zero values takes the
// least scale that a block may have: its O is 0 with any, its share of D is right with any.)
//
// Codes are exact in fp16.  Queries are multiplied by a power of two that brings the row's largest element to
// [2^14, 2^15): an fp16 or bf16 query is then exact in one fp16 (elements below 2^-28 of the row's largest lose
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
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float float8v __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWideRows = 128;       // rows of a workgroup of the kernel for many
constexpr float kNoMax = -FLT_MAX;  // M before the first row: below every logit, and finite, so that M - M stays 0
constexpr float kLift = 6.f;       // u carries 2^6, away from fp16's subnormals
constexpr float kSlack = 8.f;      // M is raised only when a row exceeds it by 2^8: u stays below 2^15
constexpr float kLargeMax = 0x1p18f;
constexpr uint32_t kLeastScaleBits = __builtin_bit_cast(uint32_t, kKvLeastScale);

struct AttnArgs {
    KvQueries q;
    KvCache c;
    const int32_t *table, *lengths;
    void *out;
    float *part;     // splits > 1: [splits][rows * Hq][d], then (M, D) [splits][rows * Hq][2]
    int32_t width, G, tiles;  // tiles: row tiles of all requests together (a bound when packed)
    int32_t rows;             // rows of a row tile, for the kernel of short requests
    int32_t splits, chunk;    // a split is `chunk` tiles of 32 slots; as many as the table's width could fill
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

// 8 loaded elements; 4 of an output, 4-element aligned
__device__ float8v as_floats(const float *p) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    return float8v{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}
__device__ float8v as_floats(const _Float16 *p) { return __builtin_convertvector(*reinterpret_cast<const half8 *>(p), float8v); }
__device__ float8v as_floats(const __bf16 *p) {
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

struct Rows {  // a row tile of one request; a row is a query and one of the G heads that share a cached head
    int32_t b;
    int64_t first;  // first query of the request among all
    int32_t n;      // its queries; 0: there is no such tile
    int32_t tile;   // row tile within the request
    // row `m` of the request: fewer than 2^31 (query, head) rows in a call
    __device__ bool has(const AttnArgs &a, int64_t m) const { return m < (int64_t)n * a.G; }
    __device__ static uint2 parts(const AttnArgs &a, int64_t m) {  // (query, head of the group)
        if (a.G == 1) return uint2{(uint32_t)m, 0};
        const uint32_t i = (uint32_t)m / (uint32_t)a.G;
        return uint2{i, (uint32_t)m - i * (uint32_t)a.G};
    }
    __device__ const void *query(const AttnArgs &a, int h, int64_t m, int size) const {
        const uint2 p = parts(a, m);
        const int64_t at = a.q.offsets ? (first + p.x) * a.q.row : b * a.q.batch + p.x * a.q.row;
        return static_cast<const char *>(a.q.q) + (at + (int64_t)(h * a.G + (int)p.y) * a.q.head) * size;
    }
    __device__ int64_t out(const AttnArgs &a, int h, int64_t m) const {
        const uint2 p = parts(a, m);
        return (first + p.x) * a.q.Hq + (h * a.G + (int)p.y);
    }
};

// The request that row tile `t` (of R rows) belongs to.
__device__ Rows find_rows(const AttnArgs &a, int32_t t, int32_t R) {
    const int lane = threadIdx.x & 63;
    if (!a.q.offsets) {
        const int32_t per = (int32_t)(((int64_t)a.q.N * a.G + R - 1) / R);
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
        const int64_t mine = ((int64_t)n * a.G + R - 1) / R;
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

// Rows of a request: a multiple of 32 below 2^31 holds them.
__device__ int32_t length_of(const AttnArgs &a, int32_t b) {
    return __builtin_amdgcn_readfirstlane(min(max(a.lengths[b], 0), a.width * a.c.S));
}

__device__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// The root of 2^x.  M moves by more than fp32's range where scales lie far apart, and D, which holds 1 / scale, moves the
// other way: D times the root, twice, stays in range.
__device__ float half_of(float x) { return exp2_of(0.5f * x); }

// What fp16 leaves of x f, in fp16: one mixed-precision instruction (of x - hi the compiler makes three).
__device__ _Float16 rest_of(float x, float f, _Float16 hi) { return (_Float16)fmaf(x, f, -(float)hi); }

// One lane's share of a query: element 8 s + i is dim dim_of(s) + i.  Raw: as loaded.
template <class T, int N8>
struct Raw {
    uint4 w[N8 * (sizeof(T) == 4 ? 2 : 1)];
};
template <class T, int N8, class F>
__device__ void load_query(Raw<T, N8> &raw, const T *q, bool live, int d, F dim_of) {
    constexpr int n = sizeof(T) == 4 ? 2 : 1;
#pragma unroll
    for (int s = 0; s < N8; ++s) {
        const int e = dim_of(s);
        const bool in = live && e < d;
#pragma unroll
        for (int i = 0; i < n; ++i) raw.w[s * n + i] = in ? reinterpret_cast<const uint4 *>(q + e)[i] : uint4{0, 0, 0, 0};
    }
}
// The fp16 pieces.  Lanes that differ in the bits of `mask` (32, or 48) hold the rest of the row.  Returns what a product is
// multiplied with to be a logit in log2 units.
template <class T, int N8>
__device__ float split_query(const Raw<T, N8> &raw, int d, int mask, half8 (&hi)[N8], half8 *lo) {
    constexpr int n = sizeof(T) == 4 ? 2 : 1;
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < N8; ++s) {
        const float8v x = as_floats(reinterpret_cast<const T *>(&raw.w[s * n]));
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    }
    if (mask & 16) top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    // 2^up brings the largest to [2^14, 2^15); a row that is not finite gives NaN throughout
    const int up = min(14 + 127 - (int)(top >> 23), 126);
    const float lift = top ? __uint_as_float((uint32_t)(127 + up) << 23) : 1.f;
#pragma unroll
    for (int s = 0; s < N8; ++s) {
        const float8v x = as_floats(reinterpret_cast<const T *>(&raw.w[s * n]));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = x[i] * lift;
            hi[s][i] = (_Float16)y;
            if constexpr (std::is_same<T, float>::value) lo[s][i] = rest_of(x[i], lift, hi[s][i]);
        }
    }
    const float back = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : 1.f / lift;
    return back * (kLog2e / sqrtf((float)d));
}

// ---- 32 rows between memory and the lanes of the matrix cores ------------------------------------------------------------
// A lane of an operand has a whole half row: loads and stores in that order touch 32 rows in 16-byte pieces (103 us for 16 x
// 4096 x 10 x 64 fp32 rows in and out with one slot to attend to, 84 this way; a copy takes 63).  So rows cross memory 128 bytes to 8 lanes
// and change places in 4 KiB of LDS of the wavefront's own, without a barrier: LDS serves a wavefront in order.  A 16-byte
// unit u of row r is at unit u ^ (r & 7): no bank twice either way.
constexpr int kSwapBytes = 4096;
template <class T>
constexpr int kUnit = 16 / (int)sizeof(T);  // elements
template <class T, int NP>
constexpr int kChunks = sizeof(T) == 4 ? NP : (NP + 1) / 2;  // of 128 bytes of a row

__device__ void wave_order() {  // LDS accesses of the wavefront's lanes stay on their side
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A lane's place: unit lane % 8 of rows lane / 8 + 8 i.  row: their elements in memory, null where there are none.
template <class T, int NP>
struct Swap {
    uint4 w[kChunks<T, NP> * 4];
    __device__ void load(const T *const (&row)[4], int d) {
        const int unit = threadIdx.x & 7;
#pragma unroll
        for (int c = 0; c < kChunks<T, NP>; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = (c * 8 + unit) * kUnit<T>;
                w[c * 4 + i] = row[i] && e < d ? *reinterpret_cast<const uint4 *>(row[i] + e) : uint4{0, 0, 0, 0};
            }
    }
    // to the order of a B operand: element 8 s + i of a lane is dim 32 (s / 2) + 16 half + 8 (s % 2) + i of row `col`
    __device__ void spread(uint4 *lds, Raw<T, 2 * NP> &raw) const {
        const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
        constexpr int per = 8 / kUnit<T>;  // units of 8 elements
#pragma unroll
        for (int c = 0; c < kChunks<T, NP>; ++c) {
            wave_order();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (lane >> 3) + 8 * i;
                lds[r * 8 + ((lane & 7) ^ (r & 7))] = w[c * 4 + i];
            }
            wave_order();
#pragma unroll
            for (int s = 0; s < 2 * NP; ++s) {
                constexpr int dims = 8 * kUnit<T>;  // of a chunk
                if ((s >> 1) * 32 / dims != c) continue;
                const int u = ((s >> 1) * 32 % dims + half * 16 + (s & 1) * 8) / kUnit<T>;
#pragma unroll
                for (int i = 0; i < per; ++i) raw.w[s * per + i] = lds[col * 8 + ((u + i) ^ (col & 7))];
            }
        }
    }
};
// O^T as the products leave it, times `inv` of the lane's column, to rows in memory.
template <class T, int NP>
__device__ void store_rows(uint4 *lds, const float16v (&O)[NP], float inv, T *const (&row)[4], int d) {
    typedef T vec __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    constexpr int dims = 8 * kUnit<T>;
#pragma unroll
    for (int c = 0; c < kChunks<T, NP>; ++c) {
        wave_order();
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            if (s * 32 / dims != c) continue;
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int e = s * 32 % dims + 8 * (r >> 2) + 4 * half, u = e / kUnit<T>;
                vec *to = reinterpret_cast<vec *>(lds + col * 8 + (u ^ (col & 7))) + (e % kUnit<T>) / 4;
                *to = vec{(T)(O[s][r] * inv), (T)(O[s][r + 1] * inv), (T)(O[s][r + 2] * inv), (T)(O[s][r + 3] * inv)};
            }
        }
        wave_order();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (lane >> 3) + 8 * i, e = (c * 8 + (lane & 7)) * kUnit<T>;
            if (row[i] && e < d) *reinterpret_cast<uint4 *>(row[i] + e) = lds[r * 8 + ((lane & 7) ^ (r & 7))];
        }
    }
}

// Over the lanes that hold one column: the other half's, and with kMask 48 the four of a 16-lane column.
template <int kMask>
__device__ float column_max(float x) {
    auto fold = [](float x, auto swap) {
        const auto r = swap(__float_as_uint(x));
        return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    };
    if (kMask & 16) x = fold(x, [](uint32_t u) { return __builtin_amdgcn_permlane16_swap(u, u, false, false); });
    return fold(x, [](uint32_t u) { return __builtin_amdgcn_permlane32_swap(u, u, false, false); });
}

// Two weights u = 2^(x mult + off) in fp16 pieces, and their sum: of one piece, the sum of what is multiplied, so that a lone
// large u rounds without an error in out.
template <bool kTwo, class X, class P>
__device__ void weigh_two(const X &x, int r, float mult, float off, float &sum, P &ph, P &pl) {
    const float2v u{exp2_of(fmaf(x[r], mult, off)), exp2_of(fmaf(x[r + 1], mult, off))};
    const half2v hi = __builtin_convertvector(u, half2v);
    ph[r >> 3][r & 7] = hi[0], ph[r >> 3][(r & 7) + 1] = hi[1];
    if constexpr (kTwo) {
        float one = 1.f;
        asm("" : "+s"(one));  // a factor that the compiler cannot take out
        pl[r >> 3][r & 7] = rest_of(u[0], one, hi[0]), pl[r >> 3][(r & 7) + 1] = rest_of(u[1], one, hi[1]);
        sum += u[0] + u[1];
    } else {
        sum = __builtin_amdgcn_fdot2(hi, half2v{(_Float16)1.f, (_Float16)1.f}, sum, false);
    }
}

// The running sums of a lane's column (one row).
struct Column {
    float M = kNoMax, D = 0.f;
};

// A tile's logits x become weights, and M and D move on.  `left` of its 32 slots are rows; slot_of(r) is the slot of x[r].
// v_scale, v_top: bits of the tile's value scale and of the largest so far (not negative: their order is the numbers').
// rescale(f): multiply O by f.
// Nearly every tile is whole, with a scale like the others', and does not raise M: what others need is behind branches that
// leave the straight line's registers alone (O in a second copy of the line would cost 80 more).
template <bool kTwo, int R, int kMask, class X, class Slot, class Rescale, class P>
__device__ void weights(X &x, float mult, uint32_t v_scale, uint32_t &v_top, int left, Slot slot_of, Column &c, Rescale rescale, P &ph, P &pl) {
    // A block of zero values has a scale of 0 and takes the least there is: its codes are zeros, so its O is 0 and its share of D
    // right with any, and M is raised by rows that add nothing only where it is far below them.
    v_scale = max(v_scale, kLeastScaleBits);
    v_top = max(v_top, v_scale);
    if (left < 32) {
        asm volatile("");  // a branch: as selects it would cost every tile 30 instructions
        if (mult == 0.f) mult = FLT_MIN;  // so that it takes -inf to -inf; 0 to the others all the same
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (slot_of(r) >= left) x[r] = -INFINITY;
    }
    float most = x[0];
#pragma unroll
    for (int r = 1; r + 1 < R; r += 2) most = fmaxf(fmaxf(most, x[r]), x[r + 1]);
    most = column_max<kMask>(fmaxf(most, x[R - 1]));
    float shift = __builtin_amdgcn_logf(__uint_as_float(v_scale)), inv = __builtin_amdgcn_rcpf(__uint_as_float(v_scale));
    // mult is not negative, so this is the largest of the rows' own t, to the bit: a product and a sum rounded apart may be the
    // next number, which is 2^64 times the weight away where t is a billion
    const float top = fmaf(most, mult, shift);
    if (__any(top > c.M + kSlack)) {
        const float to = fmaxf(c.M, top), half = half_of(c.M - to);
        c.M = to;
        c.D = c.D * half * half;
        rescale(half * half);
    }
    float off = shift - c.M + kLift;  // one rounding, next to M; M's own is common to all rows
    if (__any(fabsf(c.M) > kLargeMax)) {  // where it could reach 1: t is rounded before M is taken off
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = fmaf(x[r], mult, shift) - c.M;
        mult = 1.f, off = kLift, most = top - c.M;
    }
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < R; r += 2) weigh_two<kTwo>(x, r, mult, off, sum, ph, pl);
    // What a row adds to D, u / s_v, may count where u itself does not: beside the values of a block of a far larger scale u is
    // below fp16's normals, or below fp32's, while its weight may be all of D.  Then D takes powers of their own, measured against
    // the tile's largest.
    if (v_scale + ((kTwo ? 64u : 6u) << 23) < v_top) {
        asm volatile("" : "+v"(off));  // else the straight line keeps its exponents for this branch: 1 to 8 registers
        const float over = fmaf(most, mult, off), half = half_of(over - shift);
        sum = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) sum += exp2_of(fmaf(x[r], mult, off) - over);
        sum *= half, inv = half;
    }
    c.D = fmaf(sum, inv, c.D);
}

// ---- many rows: a workgroup takes 128 rows through all of the request's slots ---------------------------------------------
// S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 instructions: a lane holds column (lane & 31) of both, so a row's statistics
// are its lane's (and the other half's), and the products of S^T are the operand of O^T without a move, with V's slots
// stored in the order in which S^T leaves them.
// Two tiles of 32 slots are a stage: each wavefront loads K or V of one of them (a stage ahead, in registers), makes fp16 of it
// once for all four, and puts it into LDS in units of 16 bytes, one operand of one lane, so that every read and write of 64
// lanes is 1 KiB without a bank met twice (2 x 4096 x 24 x 128 over 4000 rows: 1057 us with every wavefront converting for
// itself).  Two stages of LDS and one barrier a stage: a stage's place was last read in front of the barrier before.
// Bound by both pipes in turn, with narrow heads mostly by vector instructions: of 64-dim bf16 heads over 1024 rows 117 for a tile of
// 32 x 32 beside 8 products, 16 of them exponentials of two issue slots each, vector pipes busy 66 % and matrix pipes 29 % of the time;
// of 128-dim heads 44 % and 35 %.  Exponentials placed by hand among
// the next tile's products gained 3 % on 128 dims and cost the narrow heads a wavefront of occupancy, 10 to 25 % (121 us
// for 110 at 16 x 4096 x 10 x 64 fp32); so did both tiles' logits up front.
// T: type of q and out.  NP: 32-dim steps of the head width.
// wavefronts to a SIMD that the registers leave (and LDS: two workgroups of 160 dims fill it; 8 x 512 x 40 x 160 over 2048 rows:
// 489 us in fp32 and 299 in bf16, 629 and 489 with one)
constexpr int wide_waves(int NP) { return NP <= 1 ? 4 : NP <= 2 ? 3 : NP <= 5 ? 2 : 1; }
template <class T, int NP>
__global__ __launch_bounds__(256, wide_waves(NP)) void k_xattn_kv(AttnArgs a) {
    constexpr bool kTwo = std::is_same<T, float>::value;  // two fp16 pieces
    constexpr bool kAhead = !kTwo && NP <= 6 && NP != 5;   // 5: a second wavefront instead; 7 and 8: no registers left
    constexpr int kPart = NP * 128;                       // units of K or V of a tile
    extern __shared__ uint4 lds[];                        // [K, V][2 stages][2 tiles][kPart]; before and after, swap places
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int d = a.c.d, e16 = kv_padded(d), S = a.c.S, H = a.c.H, shift_S = __ffs(S) - 1;
    const int h = (int)(blockIdx.x / (uint32_t)a.tiles);
    const Rows rows = find_rows(a, (int32_t)(blockIdx.x % (uint32_t)a.tiles), kWideRows);
    if (rows.n == 0) return;
    // block numbers and scales of 64 blocks, one a lane, whether the request reaches them or not: they do not wait for its length
    int32_t block0 = 0, id = -1;
    float k_scale = 0.f, v_scale = 0.f;
    auto look_up = [&](int32_t first) {
        block0 = first;
        id = first + lane < a.width ? a.table[(int64_t)rows.b * a.width + first + lane] : -1;
        if (id >= a.c.n_blocks) id = -1;
        if (id >= 0) {
            const float2 scale = reinterpret_cast<const float2 *>(a.c.scales)[(int64_t)id * H + h];
            k_scale = scale.x, v_scale = scale.y;
        }
    };
    const int64_t m0 = (int64_t)rows.tile * kWideRows + wave * 32 + (lane >> 3);  // and 8, 16, 24 further: this lane's rows
    uint4 *swap_at = lds + wave * (kSwapBytes / 16);  // in the stages' place, before and after
    Swap<T, NP> fetched;
    {
        const T *row[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            row[i] = rows.has(a, m0 + 8 * i) ? static_cast<const T *>(rows.query(a, h, m0 + 8 * i, sizeof(T))) : nullptr;
        fetched.load(row, d);
    }
    look_up(0);
    const int32_t length = length_of(a, rows.b), n_tiles = (length + 31) / 32, n_stages = (n_tiles + 1) / 2;

    uint4 ahead[NP];
    const int my_tile = wave >> 1, my_part = wave & 1;
    // This wavefront's share of a stage.  64 blocks hold whole stages (64 slots): a stage needs one look-up.
    auto load = [&](int32_t st) {
        if ((int32_t)(((int64_t)st * 64) >> shift_S) - block0 >= 64) look_up((int32_t)(((int64_t)st * 64) >> shift_S));
        const int32_t t = 2 * st + my_tile;
        if (t >= n_tiles) return;
        const int32_t block = __builtin_amdgcn_readlane(id, ((t * 32) >> shift_S) - block0);
        if (block < 0) return;
        const uint8_t *tile = a.c.codes + ((int64_t)block * H + h) * kv_slice_bytes(S, d) + (int64_t)(t & ((S >> 5) - 1)) * 64 * e16;
        // the last half step of K may not be there (then the bytes of V behind it meet zeros of q), nor the last dims of V
        // (they repeat the last one; nothing reads their sums)
#pragma unroll
        for (int s = 0; s < NP; ++s)
            ahead[s] = *reinterpret_cast<const uint4 *>(
                tile + (my_part ? 32 * e16 + min(s * 32 + col, e16 - 1) * 32 + half * 16 : ((2 * s + half) * 32 + col) * 16));
    };
    auto keep = [&](int32_t st) {
        uint4 *to = lds + ((my_part * 2 + (st & 1)) * 2 + my_tile) * kPart;
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            const half8 lo = to_half8(ahead[s].x, ahead[s].y), hi = to_half8(ahead[s].z, ahead[s].w);
            // K: [chunk of 16 dims][its halves][slot]; V: [32 dims][halves of the tile][half][dim]
            const int at = my_part ? (s * 4 + half) * 32 + col : (2 * s + half) * 64 + col;
            to[at] = __builtin_bit_cast(uint4, lo);
            to[at + (my_part ? 64 : 32)] = __builtin_bit_cast(uint4, hi);
        }
    };
    // what a stage's tiles are multiplied with, and whether they are there; before the look-up moves on
    struct Stage {
        float ks[2];
        uint32_t vs[2];
        bool there[2];
    };
    auto terms_of = [&](int32_t st) {
        Stage x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = min(((2 * st + i) * 32 >> shift_S) - block0, 63);
            x.there[i] = 2 * st + i < n_tiles && __builtin_amdgcn_readlane(id, at) >= 0;
            x.ks[i] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale), at));
            x.vs[i] = __builtin_amdgcn_readlane(__float_as_uint(v_scale), at);
        }
        return x;
    };

    load(0);
    half8 qh[2 * NP], ql[kTwo ? 2 * NP : 1];
    Raw<T, 2 * NP> raw;
    fetched.spread(swap_at, raw);
    const float q_scale = split_query(raw, d, 32, qh, ql);
    __syncthreads();
    float16v O[NP];
    Column sums;
    uint32_t v_top = 0;
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[s][r] = 0.f;

    Stage now = terms_of(0);
    keep(0);
    __syncthreads();
    for (int32_t st = 0; st < n_stages; ++st) {
        const bool more = st + 1 < n_stages;
        if (more) load(st + 1);
        const Stage then = terms_of(st + 1);
        // Operands ahead of their products where the registers are there: the first of a stage are waited for, no others.
        half8 kf[2 * NP], vf[2 * NP];
        auto read_v = [&](int i) {
            const uint4 *V = lds + ((2 + (st & 1)) * 2 + i) * kPart;
#pragma unroll
            for (int s = 0; s < 2 * NP; ++s) vf[s] = __builtin_bit_cast(half8, V[((s >> 1) * 4 + (s & 1) * 2 + half) * 32 + col]);
        };
        auto read_k = [&](int i) {
            const uint4 *K = lds + ((st & 1) * 2 + i) * kPart;
#pragma unroll
            for (int s = 0; s < 2 * NP; ++s) kf[s] = __builtin_bit_cast(half8, K[((s >> 1) * 2 + half) * 64 + (s & 1) * 32 + col]);
        };
        read_k(0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (!kAhead && i == 1) read_k(1);
            float16v x;
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = 0.f;
#pragma unroll
            for (int s = 0; s < 2 * NP; ++s) {
                x = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[s], qh[s], x, 0, 0, 0);
                if constexpr (kTwo) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[s], ql[s], x, 0, 0, 0);
            }
            if constexpr (kAhead) {
                read_v(i);
                if (i == 0) read_k(1);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!now.there[i]) continue;
            half8 ph[2], pl[2];
            weights<kTwo, 16, 32>(
                x, q_scale * now.ks[i], now.vs[i], v_top, length - (2 * st + i) * 32,
                [&](int r) { return 8 * (r >> 2) + 4 * half + (r & 3); }, sums,
                [&](float less) {
#pragma unroll
                    for (int s = 0; s < NP; ++s)
#pragma unroll
                        for (int r = 0; r < 16; ++r) O[s][r] *= less;
                },
                ph, pl);
            if constexpr (!kAhead) read_v(i);
#pragma unroll
            for (int s = 0; s < 2 * NP; ++s) {
                O[s >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[s], ph[s & 1], O[s >> 1], 0, 0, 0);
                if constexpr (kTwo) O[s >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[s], pl[s & 1], O[s >> 1], 0, 0, 0);
            }
        }
        if (more) keep(st + 1);
        __syncthreads();
        now = then;
    }

    const float D = sums.D + __shfl_xor(sums.D, 32), inv = D == 0.f ? 0.f : 1.f / D;
    T *row[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) row[i] = rows.has(a, m0 + 8 * i) ? static_cast<T *>(a.out) + rows.out(a, h, m0 + 8 * i) * d : nullptr;
    store_rows<T, NP>(swap_at, O, inv, row, d);
}

constexpr int short_waves(bool two, int NP) { return NP <= 1 ? 4 : NP <= 2 ? 3 : NP <= (two ? 3 : 4) ? 2 : 1; }

// ---- many rows, short requests: all of a request's tiles fit LDS ----------------------------------------------------------
// A workgroup makes fp16 of the request's K and V once and takes a.rows rows through them, 32 to a wavefront at a time, with
// no barrier after the first; the next 32 queries are loaded while these are worked on.  Bound by the queries' and the
// output's bytes and by what the exponentials add to their time: 16 x 4096 x 10 x 64 over 77 rows takes 89 us in fp32 and 59 in
// bf16, 79 and 47 over one row (100 and 69 in stages; a copy of the bytes 63 and 31).
template <class T, int NP>
__global__ __launch_bounds__(256, short_waves(sizeof(T) == 4, NP)) void k_xattn_kv_short(AttnArgs a) {
    constexpr bool kTwo = std::is_same<T, float>::value;
    constexpr int kPart = NP * 128;  // units of K or V of a tile
    extern __shared__ uint4 lds[];   // a swap place for each wavefront, then [tiles][K, V][kPart] as in k_xattn_kv
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int d = a.c.d, e16 = kv_padded(d), S = a.c.S, H = a.c.H, shift_S = __ffs(S) - 1;
    const int h = (int)(blockIdx.x / (uint32_t)a.tiles);
    const Rows rows = find_rows(a, (int32_t)(blockIdx.x % (uint32_t)a.tiles), a.rows);
    if (rows.n == 0) return;
    const int64_t all_rows = (int64_t)rows.n * a.G, m0 = (int64_t)rows.tile * a.rows;
    const int32_t here = (int32_t)min((int64_t)a.rows, all_rows - m0);
    uint4 *swap_at = lds + wave * (kSwapBytes / 16), *tiles = lds + 4 * (kSwapBytes / 16);
    Swap<T, NP> next;
    auto fetch = [&](int32_t at) {
        const T *row[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t m = at + (lane >> 3) + 8 * i;
            row[i] = m < here ? static_cast<const T *>(rows.query(a, h, m0 + m, sizeof(T))) : nullptr;
        }
        next.load(row, d);
    };
    fetch(wave * 32);

    // at most 64 blocks: a lane looks one up, whether the request reaches it or not
    int32_t id = lane < a.width ? a.table[(int64_t)rows.b * a.width + lane] : -1;
    const int32_t length = length_of(a, rows.b);
    const int32_t n_tiles = (length + 31) / 32;
    if (id >= a.c.n_blocks) id = -1;
    float2 scale{0.f, 0.f};
    if (id >= 0) scale = reinterpret_cast<const float2 *>(a.c.scales)[(int64_t)id * H + h];
    constexpr int kBatch = NP <= 2 ? 4 : 2;  // parts whose loads are under way together
    for (int p0 = wave; p0 < 2 * n_tiles; p0 += 4 * kBatch) {
        uint4 w[kBatch][NP];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int p = p0 + 4 * j, t = p >> 1, part = p & 1;
            if (p >= 2 * n_tiles) break;
            const int32_t block = max(__builtin_amdgcn_readlane(id, (t * 32) >> shift_S), 0);  // what is not there is not used
            const uint8_t *tile = a.c.codes + ((int64_t)block * H + h) * kv_slice_bytes(S, d) + (int64_t)(t & ((S >> 5) - 1)) * 64 * e16;
#pragma unroll
            for (int s = 0; s < NP; ++s)
                w[j][s] = *reinterpret_cast<const uint4 *>(
                    tile + (part ? 32 * e16 + min(s * 32 + col, e16 - 1) * 32 + half * 16 : ((2 * s + half) * 32 + col) * 16));
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int p = p0 + 4 * j, part = p & 1;
            if (p >= 2 * n_tiles) break;
#pragma unroll
            for (int s = 0; s < NP; ++s) {
                const int at = part ? (s * 4 + half) * 32 + col : (2 * s + half) * 64 + col;
                tiles[p * kPart + at] = __builtin_bit_cast(uint4, to_half8(w[j][s].x, w[j][s].y));
                tiles[p * kPart + at + (part ? 64 : 32)] = __builtin_bit_cast(uint4, to_half8(w[j][s].z, w[j][s].w));
            }
        }
    }
    __syncthreads();

    for (int32_t at = wave * 32; at < here; at += 128) {
        half8 qh[2 * NP], ql[kTwo ? 2 * NP : 1];
        Raw<T, 2 * NP> raw;
        next.spread(swap_at, raw);
        const float q_scale = split_query(raw, d, 32, qh, ql);
        if (at + 128 < here) fetch(at + 128);
        float16v O[NP];
#pragma unroll
        for (int s = 0; s < NP; ++s)
#pragma unroll
            for (int r = 0; r < 16; ++r) O[s][r] = 0.f;
        Column sums;
        uint32_t v_top = 0;
        for (int32_t t = 0; t < n_tiles; ++t) {
            const int block = (t * 32) >> shift_S;
            if (__builtin_amdgcn_readlane(id, block) < 0) continue;
            const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale.x), block));
            const uint32_t vs = __builtin_amdgcn_readlane(__float_as_uint(scale.y), block);
            const uint4 *K = tiles + t * 2 * kPart, *V = K + kPart;
            float16v x;
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = 0.f;
#pragma unroll
            for (int s = 0; s < 2 * NP; ++s) {
                const half8 k = __builtin_bit_cast(half8, K[((s >> 1) * 2 + half) * 64 + (s & 1) * 32 + col]);
                x = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, qh[s], x, 0, 0, 0);
                if constexpr (kTwo) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, ql[s], x, 0, 0, 0);
            }
            half8 ph[2], pl[2];
            weights<kTwo, 16, 32>(
                x, q_scale * ks, vs, v_top, length - t * 32,
                [&](int r) { return 8 * (r >> 2) + 4 * half + (r & 3); }, sums,
                [&](float less) {
#pragma unroll
                    for (int s = 0; s < NP; ++s)
#pragma unroll
                        for (int r = 0; r < 16; ++r) O[s][r] *= less;
                },
                ph, pl);
#pragma unroll
            for (int s = 0; s < 2 * NP; ++s) {
                const half8 v = __builtin_bit_cast(half8, V[((s >> 1) * 4 + (s & 1) * 2 + half) * 32 + col]);
                O[s >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, ph[s & 1], O[s >> 1], 0, 0, 0);
                if constexpr (kTwo) O[s >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pl[s & 1], O[s >> 1], 0, 0, 0);
            }
        }
        const float D = sums.D + __shfl_xor(sums.D, 32), inv = D == 0.f ? 0.f : 1.f / D;
        T *row[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t m = at + (lane >> 3) + 8 * i;
            row[i] = m < here ? static_cast<T *>(a.out) + rows.out(a, h, m0 + m) * d : nullptr;
        }
        store_rows<T, NP>(swap_at, O, inv, row, d);
    }
}

// ---- few rows: a workgroup takes 16 rows through one split of the request's slots ----------------------------------------
// Bound by the cache's bytes, or by latency.  The four wavefronts take a quarter of the split's tiles each and add up in
// LDS; the tiles of one are loaded while the one before is worked on, with block numbers and scales fetched for all of a
// wavefront's tiles at once.  16 x 16 x 32 instructions: half the statistics and half the sums of a 32-row tile that would
// be empty for the most part.  Row m of the u-th K operand is slot 16 (m / 8) + 8 u + m % 8, which leaves a lane with the 8
// slots that stand together in V.  32 bf16 queries of 4 heads each over 1 .. 8192 rows of 8 heads of 128: 53 us and 5 for the
// join, 269 MB, where a stream of reads takes 39; one fp32 query over 32768 rows of 8 heads of 64: 10 and 4.
// NC: 64-dim steps of the head width.  Up to 128 dims a wavefront holds two tiles in registers; above, one, whose K is loaded
// again behind its products with q and V behind those with P: two workgroups to a CU then instead of one (2 x 1024 x 8 x 160
// over 2048 rows: 76 us in fp32 and 68 in bf16, 146 and 136 with two tiles; narrow heads lose 5 to 15 % by it).
template <int NC>
struct FewTile {
    uint4 k[2][NC];
    uint2 v[4 * NC];
};

template <class T, int NC>
__global__ __launch_bounds__(256, 2) void k_xattn_kv_few(AttnArgs a) {
    constexpr bool kTwo = std::is_same<T, float>::value;
    constexpr bool kRefill = NC >= 3;  // one tile in registers
    constexpr int kPitch = 68;  // floats of one row's 64 dims in LDS
    __shared__ float part[4][16][kPitch], stats[2][4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = lane >> 4, col = lane & 15;
    const int d = a.c.d, e16 = kv_padded(d), S = a.c.S, H = a.c.H, shift_S = __ffs(S) - 1;
    const int split = (int)(blockIdx.x % (uint32_t)a.splits);
    const int64_t task = blockIdx.x / (uint32_t)a.splits;
    const int h = (int)(task / a.tiles);
    const Rows rows = find_rows(a, (int32_t)(task % a.tiles), 16);
    if (rows.n == 0) return;
    // A wavefront's tiles, and its block numbers (at most 64), do not wait for the length.
    const int32_t per = a.chunk / 4, t0 = split * a.chunk, w0 = t0 + wave * per, block0 = (int32_t)(((int64_t)w0 * 32) >> shift_S);
    int32_t id = block0 + lane < a.width ? a.table[(int64_t)rows.b * a.width + block0 + lane] : -1;
    const int64_t m = (int64_t)rows.tile * 16 + col;
    const bool live = rows.has(a, m);
    Raw<T, 2 * NC> raw;
    load_query(raw, live ? static_cast<const T *>(rows.query(a, h, m, sizeof(T))) : nullptr, live, d,
               [&](int s) { return (s >> 1) * 64 + group * 16 + (s & 1) * 8; });
    const int32_t length = length_of(a, rows.b), n_tiles = (length + 31) / 32;
    if (split > 0 && t0 >= n_tiles) return;  // the join knows how many splits there are
    const int32_t w1 = min(min(w0 + per, t0 + a.chunk), n_tiles);
    if (id >= a.c.n_blocks) id = -1;
    float k_scale = 0.f, v_scale = 0.f;
    if (id >= 0 && w0 < w1) {
        const float2 scale = reinterpret_cast<const float2 *>(a.c.scales)[(int64_t)id * H + h];
        k_scale = scale.x, v_scale = scale.y;
    }

    half8 qh[2 * NC], ql[kTwo ? 2 * NC : 1];
    float q_scale;
    floatx4 O[4 * NC];
#pragma unroll
    for (int i = 0; i < 4 * NC; ++i) O[i] = floatx4(0.f);
    Column sums;
    uint32_t v_top = 0;
    const int k_at = (group * 32 + 16 * (col >> 3) + (col & 7)) * 16;
    const int v_at = 32 * e16 + col * 32 + (group & 1) * 16 + (group >> 1) * 8;
    const int n_dims = e16 / 16;

    auto tile_of = [&](int32_t t) {
        const int32_t block = max(__builtin_amdgcn_readlane(id, ((t * 32) >> shift_S) - block0), 0);
        return a.c.codes + ((int64_t)block * H + h) * kv_slice_bytes(S, d) + (int64_t)(t & ((S >> 5) - 1)) * 64 * e16;
    };
    auto load_k = [&](FewTile<NC> &x, const uint8_t *tile) {
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (4 * s + group < n_dims) x.k[u][s] = *reinterpret_cast<const uint4 *>(tile + k_at + s * 2048 + u * 128);
    };
    auto load_v = [&](FewTile<NC> &x, const uint8_t *tile) {
#pragma unroll
        for (int i = 0; i < 4 * NC; ++i)
            if (i < n_dims) x.v[i] = *reinterpret_cast<const uint2 *>(tile + v_at + i * 512);
    };
    auto load = [&](FewTile<NC> &x, int32_t t) {
        const uint8_t *tile = tile_of(t);
        load_k(x, tile);
        load_v(x, tile);
    };
    auto work = [&](FewTile<NC> &w, int32_t t) {
        const int at = ((t * 32) >> shift_S) - block0;
        const bool there = __builtin_amdgcn_readlane(id, at) >= 0;
        if (!kRefill && !there) return;
        const uint8_t *next = tile_of(kRefill ? min(t + 1, w1 - 1) : t);
        const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale), at));
        const uint32_t vs = __builtin_amdgcn_readlane(__float_as_uint(v_scale), at);
        floatx4 acc[2] = {floatx4(0.f), floatx4(0.f)};
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const half8 k0 = to_half8(w.k[u][s].x, w.k[u][s].y), k1 = to_half8(w.k[u][s].z, w.k[u][s].w);
                acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qh[2 * s], acc[u], 0, 0, 0);
                acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qh[2 * s + 1], acc[u], 0, 0, 0);
                if constexpr (kTwo) {
                    acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, ql[2 * s], acc[u], 0, 0, 0);
                    acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, ql[2 * s + 1], acc[u], 0, 0, 0);
                }
            }
        if (kRefill) load_k(w, next);
        if (kRefill && !there) return load_v(w, next);
        float x[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) x[r] = acc[r >> 2][r & 3];
        half8 ph[1], pl[1];
        weights<kTwo, 8, 48>(
            x, q_scale * ks, vs, v_top, length - t * 32,
            [&](int r) { return 16 * (group >> 1) + 8 * (r >> 2) + 4 * (group & 1) + (r & 3); }, sums,
            [&](float less) {
#pragma unroll
                for (int i = 0; i < 4 * NC; ++i) O[i] *= less;
            },
            ph, pl);
#pragma unroll
        for (int i = 0; i < 4 * NC; ++i)
            if (i < n_dims) {
                const half8 v = to_half8(w.v[i].x, w.v[i].y);
                O[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph[0], O[i], 0, 0, 0);
                if constexpr (kTwo) O[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl[0], O[i], 0, 0, 0);
            }
        if (kRefill) load_v(w, next);
    };
    FewTile<NC> x;
#pragma unroll
    for (int s = 0; s < NC; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u) x.k[u][s] = uint4{0, 0, 0, 0};  // chunks that are not there: finite
    if (w0 < w1) load(x, w0);
    if constexpr (!kRefill) {
        FewTile<NC> y;
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) y.k[u][s] = uint4{0, 0, 0, 0};
        q_scale = split_query(raw, d, 48, qh, ql);
        for (int32_t t = w0; t < w1; t += 2) {
            if (t + 1 < w1) load(y, t + 1);
            work(x, t);
            if (t + 1 < w1) {
                if (t + 2 < w1) load(x, t + 2);
                work(y, t + 1);
            }
        }
    } else {
        q_scale = split_query(raw, d, 48, qh, ql);
        for (int32_t t = w0; t < w1; ++t) work(x, t);
    }

    // ---- the four wavefronts' sums ----
    float M = sums.M, D = sums.D;
    D += __shfl_xor(D, 16);
    D += __shfl_xor(D, 32);
    if (group == 0) stats[0][wave][col] = M, stats[1][wave][col] = D;
    __syncthreads();
    const float all_M = fmaxf(fmaxf(stats[0][0][col], stats[0][1][col]), fmaxf(stats[0][2][col], stats[0][3][col]));
    const float mine = exp2_of(M - all_M);  // of O
    const int row = threadIdx.x >> 4, quad = threadIdx.x & 15;
    float row_M = kNoMax, row_D = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) row_M = fmaxf(row_M, stats[0][w][row]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float half = half_of(stats[0][w][row] - row_M);
        row_D = fmaf(stats[1][w][row] * half, half, row_D);
    }
    const int64_t out_m = (int64_t)rows.tile * 16 + row;
    const bool out_live = rows.has(a, out_m);
    const int64_t out_row = out_live ? rows.out(a, h, out_m) : 0;
    const bool alone = n_tiles <= a.chunk;
    const int64_t all = a.q.rows() * a.q.Hq, p = split * all + out_row;
    const float inv = alone ? (row_D == 0.f ? 0.f : 1.f / row_D) : 1.f;
#pragma unroll
    for (int s = 0; s < NC; ++s) {
        if (s) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<floatx4 *>(&part[wave][col][i * 16 + group * 4]) = O[4 * s + i] * mine;
        __syncthreads();
        const int e = s * 64 + quad * 4;
        if (out_live && e < d) {
            floatx4 sum = floatx4(0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += *reinterpret_cast<const floatx4 *>(&part[w][row][quad * 4]);
            sum *= inv;
            if (alone) store4(static_cast<T *>(a.out) + out_row * d + e, sum[0], sum[1], sum[2], sum[3]);
            else *reinterpret_cast<floatx4 *>(a.part + p * d + e) = sum;
        }
    }
    if (!alone && out_live && quad == 0) reinterpret_cast<float2 *>(a.part + a.splits * all * d)[p] = float2{row_M, row_D};
}

// The request of row `n`, a query among all, or -1.
__device__ int32_t request_of(const AttnArgs &a, int64_t n) {
    if (!a.q.offsets) return (int32_t)(n / a.q.N);
    int32_t b = -1;
    for (int i = threadIdx.x & 63; i < a.q.B && b < 0; i += 64)
        if (a.q.offsets[i] <= n && n < a.q.offsets[i + 1]) b = i;
    const uint64_t found = __ballot(b >= 0);
    return found ? __shfl(b, __ffsll((unsigned long long)found) - 1) : -1;
}

// The splits of one row (query and head) added up: out = sum 2^(M_i - M) O_i / sum 2^(M_i - M) D_i, for at most kJoinFew: a
// wavefront has a row, a lane a quad of dims and one of 64 / quads runs of splits, and nothing waits for another wavefront
// (2 x 256 x 8 x 64 fp32 over 2048 rows, 3 splits: the call takes 18 us, 24 with a workgroup to a row; 1 x 1 x 8 x 256 over 8000
// rows, 16 splits: 21 and 20, so it is for at most 2048 / d of them).
constexpr int kJoinFew = 16;
template <class T>
__global__ __launch_bounds__(256) void k_xattn_kv_join_few(AttnArgs a) {
    const int d = a.c.d, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t all = a.q.rows() * a.q.Hq, row = (int64_t)blockIdx.x * 4 + wave;
    if (row >= all) return;
    const int32_t b = request_of(a, row / a.q.Hq);
    if (b < 0) return;  // a row that no request has is left as it was
    const int active = ((length_of(a, b) + 31) / 32 + a.chunk - 1) / a.chunk;
    if (active <= 1) return;  // the only split has written out itself
    float2 mine{kNoMax, 0.f};
    if (lane < active) mine = reinterpret_cast<const float2 *>(a.part + a.splits * all * d)[lane * all + row];
    float M = mine.x;
    for (int o = 8; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 16));
    M = __shfl(M, 0);
    const float half = lane < active ? half_of(mine.x - M) : 0.f, weight = half * half;
    float D = mine.y * half * half;
    for (int o = 8; o; o >>= 1) D += __shfl_xor(D, o, 16);
    D = __shfl(D, 0);
    const int quads = d / 4, runs = min(64 / quads, active), run = lane / quads, quad = lane - run * quads;
    floatx4 sum = floatx4(0.f);
    for (int i0 = run; i0 - run < active; i0 += 4 * runs) {
        floatx4 part[4];  // four loads under way
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * runs;
            part[j] = floatx4(0.f);
            if (run < runs && i < active) part[j] = *reinterpret_cast<const floatx4 *>(a.part + (i * all + row) * d + quad * 4);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += part[j] * __shfl(weight, (i0 + j * runs) & 63);
    }
    floatx4 total = sum;
    for (int r = 1; r < runs; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) total[j] += __shfl(sum[j], (lane + r * quads) & 63);
    if (lane < quads) {
        const float inv = D == 0.f ? 0.f : 1.f / D;
        store4(static_cast<T *>(a.out) + row * d + quad * 4, total[0] * inv, total[1] * inv, total[2] * inv, total[3] * inv);
    }
}

// The same for more splits: a workgroup has a row; threads are a quad of dims and one of 256 / quads runs of splits, whose sums
// meet in LDS.
template <class T>
__global__ __launch_bounds__(256) void k_xattn_kv_join(AttnArgs a) {
    __shared__ float sums[256][4], weight[256], top[4], total[4];
    const int d = a.c.d, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t all = a.q.rows() * a.q.Hq, row = blockIdx.x, n = row / a.q.Hq;
    const int32_t b = request_of(a, n);
    if (b < 0) return;  // a row that no request has is left as it was
    const int active = ((length_of(a, b) + 31) / 32 + a.chunk - 1) / a.chunk;
    if (active <= 1) return;  // the only split has written out itself
    const float2 *stats = reinterpret_cast<const float2 *>(a.part + a.splits * all * d) + row;
    const int quads = d / 4, runs = 256 / quads, quad = tid % quads, run = tid / quads;
    float M = kNoMax;
    for (int i = tid; i < active; i += 256) M = fmaxf(M, stats[i * all].x);
    for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    if (lane == 0) top[wave] = M;
    __syncthreads();
    M = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    float D = 0.f;
    floatx4 sum = floatx4(0.f);
    for (int i0 = 0; i0 < active; i0 += 256) {
        __syncthreads();
        if (i0 + tid < active) {
            const float2 s = stats[(i0 + tid) * all];
            const float half = half_of(s.x - M);
            weight[tid] = half * half;
            D = fmaf(s.y * half, half, D);
        }
        __syncthreads();
        const int here = min(active - i0, 256);
        if (run < runs) {
#pragma unroll 4
            for (int i = run; i < here; i += runs)
                sum += *reinterpret_cast<const floatx4 *>(a.part + ((i0 + i) * all + row) * d + quad * 4) * weight[i];
        }
    }
    for (int o = 32; o; o >>= 1) D += __shfl_xor(D, o);
    if (lane == 0) total[wave] = D;
    *reinterpret_cast<floatx4 *>(sums[tid]) = sum;
    __syncthreads();
    D = total[0] + total[1] + total[2] + total[3];
    if (tid < quads) {
        for (int i = 1; i < runs; ++i) sum += *reinterpret_cast<const floatx4 *>(sums[i * quads + tid]);
        const float inv = D == 0.f ? 0.f : 1.f / D;
        store4(static_cast<T *>(a.out) + row * d + tid * 4, sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv);
    }
}

enum Kernel { kFew, kShort, kLong };
struct Plan {
    Kernel kernel;
    int64_t tiles;
    int32_t rows, splits, chunk;
    int64_t groups(int32_t Hkv) const { return tiles * Hkv * splits; }  // workgroups
};
constexpr int kFewChunk = 16;
// LDS for the tiles of a short request: what lets three workgroups to a CU in, with their swap places (64 KiB, two: 231 rows of 64
// dims at batch 16 take 170 us, 158 in stages).
constexpr int kShortBytes = 32 * 1024;
constexpr int tile_bytes(int d) { return (d + 31) / 32 * 4096; }  // fp16 of a tile's K and V

// Which kernel, its row tiles, and into how many parts each request's slots are split.
// fp32: queries are; false where it isn't known, which takes as many splits or more.
Plan plan_of(int32_t B, int64_t rows, bool packed, int32_t Hq, int32_t Hkv, int32_t d, int64_t slots, bool fp32) {
    const int64_t G = Hq / Hkv;
    auto tiles_of_rows = [&](int64_t R) { return packed ? rows * G / R + B : B * ((rows / B * G + R - 1) / R); };
    const int64_t wide = tiles_of_rows(kWideRows), slot_tiles = (slots + 31) / 32;
    // 128 rows at a time leave part of the chip idle below 256 workgroups; 16 at a time convert and multiply for half-empty tiles
    // above.  Where they meet: at 128 over few slots (2 x 1024 x 8 x 128 bf16 over 77 rows: 9 us, 11 by 16; half the rows: 9 and 7),
    // at 192 over more (4 x 900 x 6 x 160 over 512 rows: 29 and 39; 2 x 1024 x 8: 28 and 27), at 256 with narrow heads, whose long
    // rows keep the statistics busy (4 x 900 x 6 x 64 over 2048 rows: 53 and 41; 8 x 256 x 16: 52 and 54).
    const int64_t enough = slot_tiles <= 8 ? 128 : d <= 64 ? 256 : 192;
    if (rows * G > 16 * (int64_t)B && wide * Hkv >= enough) {
        if (slot_tiles * tile_bytes(d) > kShortBytes) return {kLong, wide, kWideRows, 1, 0};
        // 128 rows at a time, as often as leaves some 1536 workgroups (six to a CU: lengths differ)
        const int64_t times = std::max<int64_t>(1, std::min<int64_t>(16, wide * Hkv / 1536));
        return {kShort, tiles_of_rows(128 * times), (int32_t)(128 * times), 1, 0};
    }
    const int64_t tiles = tiles_of_rows(16), groups = tiles * Hkv;
    // Parts for what the chip holds at once, three workgroups to a CU or two: more of them wait for a place while the last ones run
    // (32 bf16 queries of 128 dims over 1 .. 8192 rows: 84 us with 1024, 57 with 768, 71 with 512; in fp32, over 2048 .. 4096 rows,
    // 52, 58 and 46; of 160 dims 71, 78 and 67).  None below kFewChunk tiles or above 256 (what one can look up).
    const int64_t held = d <= 64 || (d <= 128 && !fp32) ? 768 : 512;
    const int64_t want = std::max<int64_t>(1, held / std::max<int64_t>(1, groups));
    const int64_t least = std::min<int64_t>(kFewChunk, slot_tiles), part = std::max(least, (slot_tiles + want - 1) / want);
    const int64_t chunk = std::min<int64_t>(256, (part + 3) / 4 * 4);
    return {kFew, tiles, 16, (int32_t)std::max<int64_t>(1, (slot_tiles + chunk - 1) / chunk), (int32_t)chunk};
}

template <class T>
hipError_t launch(const AttnArgs &a, Kernel kernel, hipStream_t st) {
    if (kernel != kFew) {
        const dim3 grid((uint32_t)((int64_t)a.tiles * a.c.H));
        hipError_t e = hipSuccess;
        auto go = [&](auto np) {
            constexpr int NP = decltype(np)::value;
            if (kernel == kShort) {
                const int bytes = (int)(((int64_t)a.width * a.c.S + 31) / 32) * tile_bytes(a.c.d) + 4 * kSwapBytes;
                e = DGQ_ENSURE_LDS((k_xattn_kv_short<T, NP>), kShortBytes + 4 * kSwapBytes);
                if (e == hipSuccess) k_xattn_kv_short<T, NP><<<grid, 256, bytes, st>>>(a);
            } else {
                constexpr int bytes = NP * 16384;
                e = DGQ_ENSURE_LDS((k_xattn_kv<T, NP>), bytes);
                if (e == hipSuccess) k_xattn_kv<T, NP><<<grid, 256, bytes, st>>>(a);
            }
        };
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
        return e == hipSuccess ? hipGetLastError() : e;
    }
    const dim3 grid((uint32_t)((int64_t)a.tiles * a.c.H * a.splits));
    switch ((a.c.d + 63) / 64) {
        case 1: k_xattn_kv_few<T, 1><<<grid, 256, 0, st>>>(a); break;
        case 2: k_xattn_kv_few<T, 2><<<grid, 256, 0, st>>>(a); break;
        case 3: k_xattn_kv_few<T, 3><<<grid, 256, 0, st>>>(a); break;
        default: k_xattn_kv_few<T, 4><<<grid, 256, 0, st>>>(a); break;
    }
    if (a.splits > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int64_t all = a.q.rows() * a.q.Hq;
        if (a.splits <= kJoinFew && a.splits * a.c.d <= 2048) k_xattn_kv_join_few<T><<<(uint32_t)((all + 3) / 4), 256, 0, st>>>(a);
        else k_xattn_kv_join<T><<<(uint32_t)all, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

size_t xattn_kv_workspace_bytes(int32_t B, int64_t rows, bool packed, int32_t Hq, int32_t Hkv, int32_t d, int64_t slots) {
    const Plan p = plan_of(B, rows, packed, Hq, Hkv, d, slots, false);
    return p.splits > 1 ? (size_t)p.splits * rows * Hq * (d + 2) * sizeof(float) : 0;
}

bool xattn_kv_fits(int32_t B, int64_t rows, bool packed, int32_t Hq, int32_t Hkv, int32_t d, int64_t slots) {
    const Plan p = plan_of(B, rows, packed, Hq, Hkv, d, slots, false);
    return p.groups(Hkv) <= kMaxGroups && (p.splits == 1 || rows * Hq <= kMaxGroups);
}

int xattn_kv_kernel(int32_t B, int64_t rows, bool packed, int32_t Hq, int32_t Hkv, int32_t d, int64_t slots) {
    const Plan p = plan_of(B, rows, packed, Hq, Hkv, d, slots, false);
    return p.kernel == kFew ? p.splits > 1 : p.kernel == kShort ? 2 : 3;
}

int32_t xattn_kv_rows(int32_t B, int64_t rows, bool packed, int32_t Hq, int32_t Hkv, int32_t d, int64_t slots) {
    return plan_of(B, rows, packed, Hq, Hkv, d, slots, false).rows;
}

hipError_t launch_xattn_kv(const KvQueries &q, const KvCache &c, const int32_t *table, int32_t width,
                           const int32_t *lengths, void *out, void *workspace, hipStream_t st) {
    const Plan p = plan_of(q.B, q.rows(), q.offsets != nullptr, q.Hq, c.H, c.d, (int64_t)width * c.S, q.dtype == DGQ_F32);
    const AttnArgs a{q, c, table, lengths, out, static_cast<float *>(workspace), width, q.Hq / c.H, (int32_t)p.tiles, p.rows, p.splits, p.chunk};
    return q.dtype == DGQ_F32 ? launch<float>(a, p.kernel, st)
           : q.dtype == DGQ_F16 ? launch<_Float16>(a, p.kernel, st) : launch<__bf16>(a, p.kernel, st);
}

}  // namespace dgq
