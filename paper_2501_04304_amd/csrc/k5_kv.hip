// The 8-bit cache of text keys and values: block planning, writing and reading back.
//
// A prompt's K and V do not change over the denoising steps.  They are quantized once into blocks of S slots
// (S = 32, 64, 128) that all requests of a server share; a request names its blocks in a row of a table.  Every
// (block, head) has one scale for K and one for V:
//   s = max |x| * (1/127) over the block's rows,  code = clamp(rne(x * (1/s)), -127, 127),  stored byte = code + 128.
// The layout (dgq_internal.h, kv_*) is the attention's: a lane's 16-byte load is an operand of the matrix cores.
#include <algorithm>
#include <type_traits>

#include "dgq_internal.h"

namespace dgq {
namespace {

constexpr int kPlanArrays = 4;  // 32-bit words a request in LDS

// x of the lane that the DPP control names, 0 where there is none.
template <int CTRL, int ROWS = 15>
__device__ int64_t dpp(int64_t x) {
    const int lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 15, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 15, false);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}
// Inclusive sums over a wavefront: within rows of 16 lanes, then row 0 to 1 and 2 to 3, then the first half to the second.
__device__ int64_t wave_sums(int64_t x) {
    x += dpp<0x111>(x);
    x += dpp<0x112>(x);
    x += dpp<0x114>(x);
    x += dpp<0x118>(x);
    x += dpp<0x142, 0xa>(x);
    x += dpp<0x143, 0xc>(x);
    return x;
}
// Inclusive sums over the workgroup, and the total.  lds: an entry a wavefront, of this call's own.
template <int WAVES>
__device__ int64_t group_sums(int64_t x, int64_t &total, int64_t *lds) {
    const int wave = threadIdx.x >> 6;
    x = wave_sums(x);
    if ((threadIdx.x & 63) == 63) lds[wave] = x;
    __syncthreads();
    total = 0;
    int64_t before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    return x + before;
}

// First index in [0, n) whose entry is above x (n if none); `ends` ascending.
__device__ int first_above(const int32_t *ends, int n, int32_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

__device__ int32_t clamp31(int64_t x) { return (int32_t)min(x, (int64_t)INT32_MAX); }

// Every workgroup sums over all requests (PER to a thread, in registers) and writes its share of the runs, so nothing has to be
// passed between workgroups: the sums over some thousand requests take less than a second launch.  Bound by latency: one
// read of the requests, two sums, a search and a read of the free list for every run.
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void k_kv_plan(
    const int32_t *__restrict__ lengths, const int32_t *__restrict__ new_rows, int32_t B, int32_t shift_S, int64_t rows,
    int32_t *table, int32_t width, const int32_t *__restrict__ free_blocks, int32_t free_capacity,
    const int32_t *__restrict__ n_free_in, int32_t *__restrict__ lengths_out, int32_t *__restrict__ n_free_out,
    int32_t *__restrict__ row_offsets, int4 *__restrict__ runs, int32_t max_runs, int32_t *__restrict__ counts) {
    extern __shared__ int32_t request[];  // [kPlanArrays][B]
    __shared__ int64_t sums[4][THREADS / 64];
    int32_t *run_ends = request, *row0 = request + B, *take0 = request + 2 * B, *held = request + 3 * B;
    const int32_t S = 1 << shift_S, b0 = threadIdx.x * PER;
    int32_t old[PER], add[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        old[i] = b0 + i < B ? lengths[b0 + i] : 0;
        add[i] = b0 + i < B ? new_rows[b0 + i] : 0;
    }
    const int32_t n_free = min(max(*n_free_in, 0), free_capacity);

    // Rows of the packed tensors, and blocks asked for, in the order of the requests.  (A request whose rows end behind
    // `rows` counts here too: those before it, which is all that may be served, are not touched by that.)
    auto fits = [&](int i) { return old[i] >= 0 && add[i] >= 0 && (int64_t)old[i] + add[i] <= (int64_t)width << shift_S; };
    auto need = [&](int i) { return (((int64_t)old[i] + add[i] + S - 1) >> shift_S) - (((int64_t)old[i] + S - 1) >> shift_S); };
    int64_t my_rows = 0, my_blocks = 0, all_rows, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        my_rows += max(add[i], 0);
        if (fits(i)) my_blocks += need(i);
    }
    int64_t row = group_sums<THREADS / 64>(my_rows, all_rows, sums[0]) - my_rows, block = group_sums<THREADS / 64>(my_blocks, total, sums[1]) - my_blocks;

    // a request is served if the free blocks reach for it and for all before it
    int32_t served = 0;  // bits
    int64_t my_runs = 0, others = 0;  // others: blocks taken, and requests not served in the upper half
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int64_t first = block, end = row + max(add[i], 0);
        const bool ok = fits(i);
        if (ok) block += need(i);
        const bool yes = ok && end <= rows && (add[i] == 0 || block <= n_free);
        if (b0 + i < B) {
            row0[b0 + i] = clamp31(row);
            take0[b0 + i] = clamp31(first);
            held[b0 + i] = old[i];
            if (yes) served |= 1 << i;
            if (yes && add[i] > 0) my_runs += (((int64_t)old[i] + add[i] + S - 1) >> shift_S) - (old[i] >> shift_S), others += need(i);
            if (!yes) others += (int64_t)1 << 32;
            if (blockIdx.x == 0) {
                lengths_out[b0 + i] = yes ? old[i] + add[i] : old[i];
                row_offsets[b0 + i] = clamp31(row);
            }
        }
        row = end;
    }
    int64_t all_runs, all_others;
    int64_t run = group_sums<THREADS / 64>(my_runs, all_runs, sums[2]) - my_runs;
    group_sums<THREADS / 64>(others, all_others, sums[3]);
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (b0 + i < B) {
            if (served >> i & 1 && add[i] > 0) run += (((int64_t)old[i] + add[i] + S - 1) >> shift_S) - (old[i] >> shift_S);
            run_ends[b0 + i] = (int32_t)run;
        }
    __syncthreads();
    const int32_t n_runs = (int32_t)min(all_runs, (int64_t)max_runs), taken = (int32_t)all_others;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        row_offsets[B] = clamp31(all_rows);
        *n_free_out = n_free - taken;
        *reinterpret_cast<int4 *>(counts) = int4{n_runs, taken, (int32_t)(all_others >> 32), clamp31(all_rows)};
    }
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < max_runs; i += (int64_t)gridDim.x * THREADS) {
        int4 out{-1, 0, 0, 0};
        if (i < n_runs) {
            const int r = first_above(run_ends, B, (int32_t)i);
            const int32_t length = held[r], more = (r + 1 < B ? row0[r + 1] : (int32_t)all_rows) - row0[r];
            const int32_t have = (int32_t)(((int64_t)length + S - 1) >> shift_S);
            const int32_t col = (length >> shift_S) + (int32_t)(i - (r ? run_ends[r - 1] : 0));
            int32_t *entry = table + (int64_t)r * width + col;
            if (col >= have) {
                out.x = free_blocks[n_free - 1 - (take0[r] + (col - have))];
                *entry = out.x;
            } else {
                out.x = *entry;
            }
            const int64_t start = (int64_t)col << shift_S, first = max((int64_t)length, start);  // row of the request that starts the run
            out.y = (int32_t)(row0[r] + (first - length));
            out.z = (int32_t)(first - start);
            out.w = (int32_t)(min(start + S, (int64_t)length + more) - first);
        }
        runs[i] = out;
    }
}

// The blocks of finished requests go to the end of the free list, in the order of the requests.
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void k_kv_release(
    const uint8_t *__restrict__ done, const int32_t *__restrict__ lengths, const int32_t *__restrict__ table, int32_t B,
    int32_t width, int32_t shift_S, int32_t *__restrict__ free_blocks, int32_t free_capacity,
    const int32_t *__restrict__ n_free_in, int32_t *__restrict__ lengths_out, int32_t *__restrict__ n_free_out) {
    extern __shared__ int32_t ends[];  // [B]
    __shared__ int64_t sums[THREADS / 64];
    const int32_t b0 = threadIdx.x * PER;
    int32_t held[PER];
    int64_t mine = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        held[i] = 0;
        if (b0 + i >= B) continue;
        const int32_t length = lengths[b0 + i];
        const bool out = done[b0 + i];
        if (out) held[i] = (int32_t)min(((int64_t)max(length, 0) + (1 << shift_S) - 1) >> shift_S, (int64_t)width);
        if (blockIdx.x == 0) lengths_out[b0 + i] = out ? 0 : length;
        mine += held[i];
    }
    const int32_t n_free = min(max(*n_free_in, 0), free_capacity);
    const int64_t room = free_capacity - n_free;  // a list that would overflow drops what does not fit
    int64_t at = group_sums<THREADS / 64>(mine, total, sums) - mine;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        at += held[i];
        if (b0 + i < B) ends[b0 + i] = (int32_t)min(at, room);
    }
    __syncthreads();
    const int32_t n = (int32_t)min(total, room);
    if (blockIdx.x == 0 && threadIdx.x == 0) *n_free_out = n_free + n;
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS) {
        const int r = first_above(ends, B, (int32_t)i);
        free_blocks[n_free + i] = table[(int64_t)r * width + (i - (r ? ends[r - 1] : 0))];
    }
}

// ---- between rows and a tile's bytes ----------------------------------------------------------------------------------
// An item is 4 rows (slots 4 q .. 4 q + 3) by one 16-byte load of dims: V keeps 4 such slots of a dim in one word, K keeps the
// dims of a slot together, so an item's codes are whole words of either, and rows cross memory in whole lines.  The words
// meet in an image of the tile in LDS, which crosses memory in whole lines too.  16-byte units of the image change places so
// that the items of a wavefront, whose words lie 128 or 512 bytes apart, meet few banks twice.
template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

__host__ __device__ inline int k_unit(int unit) { return unit ^ ((unit >> 5) & 7); }  // [chunk][32 slots]
__host__ __device__ inline int v_unit(int unit) { return unit ^ ((unit >> 3) & 7); }  // [dim][2]
// words of the image: dims e .. e + 3 of a slot; slots 4 q .. 4 q + 3 of a dim (q < 8)
__device__ int k_word(int slot, int e) { return k_unit((e >> 4) * 32 + slot) * 4 + ((e >> 2) & 3); }
__device__ int v_word(int q, int e) { return v_unit(e * 2 + (q & 1)) * 4 + (q >> 1); }

template <class T>
__device__ void to_floats(const uint4 &w, float (&f)[kVec<T>]) {
    if constexpr (sizeof(T) == 4) {
        f[0] = __uint_as_float(w.x), f[1] = __uint_as_float(w.y), f[2] = __uint_as_float(w.z), f[3] = __uint_as_float(w.w);
    } else {
        const T *x = reinterpret_cast<const T *>(&w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)x[i];
    }
}

// code + 128 of a finite x
__device__ float code_of(float x, float inv) { return fminf(fmaxf(rintf(x * inv), -127.f), 127.f) + 128.f; }
__device__ float value_of(uint32_t word, int byte, float scale) { return ((float)((word >> (8 * byte)) & 255) - 128.f) * scale; }

// ---- writing ---------------------------------------------------------------------------------------------------------
// One workgroup per (run, head, K or V).  The run's rows are read once, into registers: max |x|, then the codes.  Bound by
// the bytes; I: items of a thread.
template <class T, int I>
__global__ __launch_bounds__(256) void k_kv_store(
    const T *__restrict__ k, const T *__restrict__ v, int64_t rows, int64_t k_row, int64_t k_head, int64_t v_row,
    int64_t v_head, const int4 *__restrict__ runs, KvCache c) {
    extern __shared__ uint32_t image[];  // [S / 32][e16 8 words]
    __shared__ uint32_t tops[4];
    constexpr int V = kVec<T>;
    const int4 run = runs[blockIdx.x];
    const int32_t block = run.x, slot0 = run.z, n = run.w, h = blockIdx.y, S = c.S, d = c.d, tid = threadIdx.x;
    const bool is_v = blockIdx.z;
    if (n < 1 || block < 0 || block >= c.n_blocks || slot0 < 0 || (int64_t)slot0 + n > S || run.y < 0 || (int64_t)run.y + n > rows)
        return;
    const int64_t stride = is_v ? v_row : k_row;
    const T *x = (is_v ? v + h * v_head : k + h * k_head) + (run.y - (int64_t)slot0) * stride;  // of slot 0, were it there
    const int groups = d / V, quad0 = slot0 / 4, items = ((slot0 + n - 1) / 4 - quad0 + 1) * groups;
    float *scale = c.scales + ((int64_t)block * c.H + h) * 2 + is_v;
    const float s_old = slot0 > 0 ? *scale : 0.f;

    uint4 w[I][4];
    uint32_t top = 0;  // |x| as bits: their order is the numbers', and NaN is above infinity
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int item = tid + 256 * i, quad = quad0 + item / groups, e = (item % groups) * V;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int slot = quad * 4 + r;
            w[i][r] = uint4{0, 0, 0, 0};
            if (item < items && slot >= slot0 && slot < slot0 + n) w[i][r] = *reinterpret_cast<const uint4 *>(x + slot * stride + e);
        }
    }
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float f[V];
            to_floats<T>(w[i][r], f);
#pragma unroll
            for (int o = 0; o < V; ++o) top = max(top, __float_as_uint(f[o]) & 0x7fffffffu);
        }
    for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();  // (every thread has read the old scale)
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    float s = __uint_as_float(top) * (1.f / 127.f);
    if (s < kKvLeastScale) s = 0.f;
    s = __uint_as_float(max(__float_as_uint(s), __float_as_uint(s_old)));  // as bits: NaN stays
    const float inv = s > 0.f ? 1.f / s : 0.f;
    if (tid == 0) *scale = s;

    const int e16 = kv_padded(d), units = e16 * 2, n_tiles = S / 32;  // units of 16 bytes of a tile's K or V
    uint4 *codes = reinterpret_cast<uint4 *>(c.codes + ((int64_t)block * c.H + h) * kv_slice_bytes(S, d)) + (is_v ? units : 0);
    // What the items leave open: rows in front (coded against the new scale), rows behind, dims from d on.
    if (slot0 > 0 || n < S || d < e16) {
        for (int u = tid; u < n_tiles * units; u += 256) {
            const int tile = u / units, at = u - tile * units;
            uint4 word{0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
            if (slot0 > tile * 32 && inv > 0.f) {
                word = codes[tile * 2 * units + at];
                uint32_t *b = reinterpret_cast<uint32_t *>(&word);
                for (int i = 0; i < 16; ++i) {
                    const int slot = tile * 32 + (is_v ? kv_slot(at & 1, i) : at & 31), e = is_v ? at >> 1 : (at >> 5) * 16 + i;
                    const uint32_t byte = slot < slot0 && e < d ? (uint32_t)code_of(value_of(b[i >> 2], i & 3, s_old), inv) : 128u;
                    b[i >> 2] = (b[i >> 2] & ~(255u << (8 * (i & 3)))) | byte << (8 * (i & 3));
                }
            }
            reinterpret_cast<uint4 *>(image)[tile * units + (is_v ? v_unit(at) : k_unit(at))] = word;
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int item = tid + 256 * i, quad = quad0 + item / groups, e = (item % groups) * V;
        if (item >= items) break;
        uint32_t *to = image + (quad >> 3) * units * 4;
        float f[4][V];
        uint32_t mask = 0;  // of the four slots, as bytes
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            to_floats<T>(w[i][r], f[r]);
            if (quad * 4 + r >= slot0 && quad * 4 + r < slot0 + n) mask |= 255u << (8 * r);
#pragma unroll
            for (int o = 0; o < V; ++o) f[r][o] = inv > 0.f ? code_of(f[r][o], inv) : 128.f;
        }
        if (is_v) {
#pragma unroll
            for (int o = 0; o < V; ++o) {
                uint32_t word = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) word |= (uint32_t)f[r][o] << (8 * r);
                uint32_t *p = to + v_word(quad & 7, e + o);
                *p = mask == 0xffffffffu ? word : (*p & ~mask) | (word & mask);  // no other thread has these bytes
            }
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (!(mask >> (8 * r) & 1)) continue;
#pragma unroll
                for (int o = 0; o < V; o += 4)
                    to[k_word((quad & 7) * 4 + r, e + o)] = (uint32_t)f[r][o] | (uint32_t)f[r][o + 1] << 8 | (uint32_t)f[r][o + 2] << 16 |
                                                            (uint32_t)f[r][o + 3] << 24;
            }
        }
    }
    __syncthreads();
    for (int u = tid; u < n_tiles * units; u += 256) {
        const int tile = u / units, at = u - tile * units;
        codes[tile * 2 * units + at] = reinterpret_cast<const uint4 *>(image)[tile * units + (is_v ? v_unit(at) : k_unit(at))];
    }
}

// ---- reading back ------------------------------------------------------------------------------------------------------
// One workgroup per (32 rows of a request, head), K and V.  Bound by the bytes written.
template <class T>
__global__ __launch_bounds__(256) void k_kv_load(KvCache c, const int32_t *__restrict__ table, int32_t width,
                                                 const int32_t *__restrict__ lengths, int32_t max_rows,
                                                 T *__restrict__ k, T *__restrict__ v) {
    extern __shared__ uint32_t image[];  // [K, V][e16 8 words]
    constexpr int V = kVec<T>;
    const int row0 = blockIdx.x * 32, h = blockIdx.y, b = blockIdx.z, S = c.S, d = c.d, units = kv_padded(d) * 2, tid = threadIdx.x;
    const int length = min(max(lengths[b], 0), width * S);
    int32_t block = -1;
    if (row0 < length) block = table[(int64_t)b * width + row0 / S];
    const bool there = block >= 0 && block < c.n_blocks;  // of the whole workgroup
    float2 scale{0.f, 0.f};
    if (there) {
        scale = reinterpret_cast<const float2 *>(c.scales)[(int64_t)block * c.H + h];
        const uint4 *codes = reinterpret_cast<const uint4 *>(c.codes + ((int64_t)block * c.H + h) * kv_slice_bytes(S, d)) +
                             (row0 % S / 32) * 2 * units;
        for (int u = tid; u < 2 * units; u += 256) {
            const int at = u < units ? k_unit(u) : units + v_unit(u - units);
            reinterpret_cast<uint4 *>(image)[at] = codes[u];
        }
        __syncthreads();
    }
    const int groups = d / V, most = min(length, max_rows);
    for (int item = tid; item < 16 * groups; item += 256) {
        const bool is_v = item >= 8 * groups;
        const int at = is_v ? item - 8 * groups : item, quad = at / groups, e = (at - quad * groups) * V;
        float f[4][V];
        if (!there) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int o = 0; o < V; ++o) f[r][o] = 0.f;
        } else if (is_v) {
#pragma unroll
            for (int o = 0; o < V; ++o) {
                const uint32_t word = image[units * 4 + v_word(quad, e + o)];
#pragma unroll
                for (int r = 0; r < 4; ++r) f[r][o] = value_of(word, r, scale.y);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int o = 0; o < V; o += 4) {
                    const uint32_t word = image[k_word(quad * 4 + r, e + o)];
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[r][o + j] = value_of(word, j, scale.x);
                }
        }
        T *to = (is_v ? v : k) + (((int64_t)b * max_rows + row0 + quad * 4) * c.H + h) * d + e;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = row0 + quad * 4 + r;
            if (row >= max_rows) break;
            typedef T vec __attribute__((ext_vector_type(V)));
            vec x;
#pragma unroll
            for (int o = 0; o < V; ++o) x[o] = (T)(row < most ? f[r][o] : 0.f);
            *reinterpret_cast<vec *>(to + (int64_t)r * c.H * d) = x;
        }
    }
}

}  // namespace

// Threads of a workgroup and requests to a thread: few of either where they cover B (16 requests: 3.0 us with 256 threads, 6.9
// with 1024), and no more than 4 to a thread, whose reads lie apart (2048 requests: 11.5 us with 16 to each of 256).
template <int T, int P>
struct PlanSize {
    static constexpr int threads = T, per = P;
};
template <class F>
static void by_requests(int32_t B, F go) {
    static_assert(kKvMaxRequests == 4 * 1024, "the last choice holds the most requests");
    if (B <= 256) go(PlanSize<256, 1>{});
    else if (B <= 1024) go(PlanSize<1024, 1>{});
    else go(PlanSize<1024, 4>{});
}

hipError_t launch_kv_plan(const int32_t *lengths, const int32_t *new_rows, int32_t B, int32_t S, int64_t rows,
                          int32_t *table, int32_t width, const int32_t *free_blocks, int32_t free_capacity,
                          const int32_t *n_free, int32_t *lengths_out, int32_t *n_free_out, int32_t *row_offsets,
                          int32_t *runs, int32_t max_runs, int32_t *counts, hipStream_t st) {
    hipError_t e = hipSuccess;
    by_requests(B, [&](auto size) {
        constexpr int T = decltype(size)::threads, P = decltype(size)::per;
        e = DGQ_ENSURE_LDS((k_kv_plan<T, P>), kPlanArrays * 4 * T * P);
        if (e == hipSuccess)
            k_kv_plan<T, P><<<std::min<int64_t>(256, ((int64_t)max_runs + T - 1) / T), T, kPlanArrays * 4 * B, st>>>(
                lengths, new_rows, B, __builtin_ctz(S), rows, table, width, free_blocks, free_capacity, n_free, lengths_out,
                n_free_out, row_offsets, reinterpret_cast<int4 *>(runs), max_runs, counts);
    });
    return e == hipSuccess ? hipGetLastError() : e;
}

hipError_t launch_kv_release(const uint8_t *done, const int32_t *lengths, const int32_t *table, int32_t B, int32_t width,
                             int32_t S, int32_t *free_blocks, int32_t free_capacity, const int32_t *n_free,
                             int32_t *lengths_out, int32_t *n_free_out, hipStream_t st) {
    const int64_t most = std::min((int64_t)B * width, (int64_t)free_capacity);
    by_requests(B, [&](auto size) {
        constexpr int T = decltype(size)::threads, P = decltype(size)::per;
        k_kv_release<T, P><<<std::max<int64_t>(1, std::min<int64_t>(64, (most + T - 1) / T)), T, 4 * B, st>>>(
            done, lengths, table, B, width, __builtin_ctz(S), free_blocks, free_capacity, n_free, lengths_out, n_free_out);
    });
    return hipGetLastError();
}

hipError_t launch_kv_store(const void *k, const void *v, int32_t dtype, int64_t rows, int64_t k_row, int64_t k_head,
                           int64_t v_row, int64_t v_head, const int32_t *runs, int32_t n_runs, const KvCache &c,
                           hipStream_t st) {
    const dim3 grid(n_runs, c.H, 2);
    const int bytes = c.S * kv_padded(c.d);  // at most 32 KiB
    auto go = [&](auto x) {
        using T = decltype(x);
        const T *kt = static_cast<const T *>(k), *vt = static_cast<const T *>(v);
        const int4 *r = reinterpret_cast<const int4 *>(runs);
        const int items = (c.S / 4 * (c.d / kVec<T>) + 255) / 256;  // at most 8 (fp32), 4
        if (items <= 1) k_kv_store<T, 1><<<grid, 256, bytes, st>>>(kt, vt, rows, k_row, k_head, v_row, v_head, r, c);
        else if (items <= 2) k_kv_store<T, 2><<<grid, 256, bytes, st>>>(kt, vt, rows, k_row, k_head, v_row, v_head, r, c);
        else if (items <= 4) k_kv_store<T, 4><<<grid, 256, bytes, st>>>(kt, vt, rows, k_row, k_head, v_row, v_head, r, c);
        else if constexpr (sizeof(T) == 4) k_kv_store<T, 8><<<grid, 256, bytes, st>>>(kt, vt, rows, k_row, k_head, v_row, v_head, r, c);
    };
    dtype == DGQ_F32 ? go(float{}) : dtype == DGQ_F16 ? go(_Float16{}) : go(__bf16{});
    return hipGetLastError();
}

hipError_t launch_kv_load(const KvCache &c, const int32_t *table, int32_t width, const int32_t *lengths, int32_t B,
                          int32_t max_rows, int32_t dtype, void *k, void *v, hipStream_t st) {
    const dim3 grid((max_rows + 31) / 32, c.H, B);
    auto go = [&](auto x) {
        using T = decltype(x);
        k_kv_load<T><<<grid, 256, 64 * kv_padded(c.d), st>>>(c, table, width, lengths, max_rows, static_cast<T *>(k), static_cast<T *>(v));
    };
    dtype == DGQ_F32 ? go(float{}) : dtype == DGQ_F16 ? go(_Float16{}) : go(__bf16{});
    return hipGetLastError();
}

}  // namespace dgq
