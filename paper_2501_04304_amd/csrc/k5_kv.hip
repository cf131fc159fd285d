// The 8-bit cache of text keys and values: block planning, writing and reading back.
//
// A prompt's K and V do not change over the denoising steps.  They are quantized once into blocks of S slots
// (S = 32, 64, 128) that all requests of a server share; a request names its blocks in a row of a table.  Every
// (block, head) has one scale for K and one for V:
//   s = max |x| * (1/127) over the block's rows,  code = clamp(rne(x * (1/s)), -127, 127),  stored byte = code + 128.
// The layout (dgq_internal.h, kv_*) is the attention's: a lane's 16-byte load is an operand of the matrix cores.
#include "dgq_internal.h"

namespace dgq {
namespace {

constexpr int kPlanThreads = 1024;

// Inclusive sums over the workgroup of two 64-bit values per thread; `total` of both for everyone.
struct Pair {
    int64_t a, b;
};
__device__ Pair scan_pair(Pair v, Pair &total, Pair *lds /* [kPlanThreads / 64] */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t a = __shfl_up(v.a, o), b = __shfl_up(v.b, o);
        if (lane >= o) v.a += a, v.b += b;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    Pair before{0, 0};
    total = {0, 0};
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        const Pair p = lds[w];
        if (w < wave) before.a += p.a, before.b += p.b;
        total.a += p.a, total.b += p.b;
    }
    return {v.a + before.a, v.b + before.b};
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

__device__ int64_t blocks_of(int64_t rows, int32_t S) { return (rows + S - 1) / S; }

// What one request asks for.
struct Ask {
    int64_t old, add, total, take;
    bool ok;
    __device__ Ask(int32_t length, int32_t more, int32_t S, int64_t width)
        : old(length), add(more), total(old + add), take(0), ok(old >= 0 && add >= 0 && total <= width * S) {
        if (ok) take = blocks_of(total, S) - blocks_of(old, S);
    }
};

// Every workgroup scans all requests (at most kKvMaxRequests: a few per thread) and writes its share of the runs, so
// nothing has to be passed between workgroups: the sums over some thousand requests take less than a second launch.
// Bound by latency: two scans and a search per run.  The prefixes that a run needs stay in LDS, 12 bytes a request.
__global__ __launch_bounds__(kPlanThreads) void k_kv_plan(
    const int32_t *__restrict__ lengths, const int32_t *__restrict__ new_rows, int32_t B, int32_t S, int64_t rows,
    int32_t *table, int32_t width, const int32_t *__restrict__ free_blocks, int32_t free_capacity,
    const int32_t *__restrict__ n_free_in, int32_t *__restrict__ lengths_out, int32_t *__restrict__ n_free_out,
    int32_t *__restrict__ row_offsets, int4 *__restrict__ runs, int32_t max_runs, int32_t *__restrict__ counts) {
    __shared__ int32_t run_ends[kKvMaxRequests], row0[kKvMaxRequests], take0[kKvMaxRequests];
    __shared__ Pair sums[kPlanThreads / 64];
    const int32_t n_free = min(max(*n_free_in, 0), free_capacity);
    const int per = (B + kPlanThreads - 1) / kPlanThreads;
    const int b0 = min((int)threadIdx.x * per, B), b1 = min(b0 + per, B);

    // rows of the packed tensors and blocks asked for, in the order of the requests
    Pair mine{0, 0}, total;
    for (int b = b0; b < b1; ++b) {
        mine.a += max(new_rows[b], 0);
    }
    Pair rows_before = scan_pair(mine, total, sums);
    const int64_t all_rows = total.a;
    int64_t at = rows_before.a - mine.a;
    Pair asked{0, 0};
    for (int b = b0; b < b1; ++b) {
        const Ask ask(lengths[b], new_rows[b], S, width);
        row0[b] = (int32_t)min(at, (int64_t)INT32_MAX);
        at += max(new_rows[b], 0);
        if (ask.ok && at <= rows) asked.a += ask.take;
    }
    Pair ends = scan_pair(asked, total, sums);
    int64_t blocks = ends.a - asked.a;

    // a request is served if the free blocks reach for it and for all before it
    at = rows_before.a - mine.a;
    Pair given{0, 0};  // runs, blocks
    int64_t refused = 0;
    for (int b = b0; b < b1; ++b) {
        const Ask ask(lengths[b], new_rows[b], S, width);
        at += max(new_rows[b], 0);
        const bool ok = ask.ok && at <= rows;
        take0[b] = (int32_t)min(blocks, (int64_t)INT32_MAX);
        if (ok) blocks += ask.take;
        const bool served = ok && (ask.add == 0 || blocks <= n_free);
        if (served && ask.add > 0) given.a += blocks_of(ask.total, S) - ask.old / S, given.b += ask.take;
        run_ends[b] = (int32_t)given.a;
        refused += !served;
        if (blockIdx.x == 0) {
            lengths_out[b] = served ? (int32_t)ask.total : lengths[b];
            row_offsets[b] = row0[b];
        }
    }
    ends = scan_pair(given, total, sums);
    const int32_t before = (int32_t)(ends.a - given.a);
    for (int b = b0; b < b1; ++b) run_ends[b] += before;
    const int32_t n_runs = (int32_t)min(total.a, (int64_t)max_runs);
    const int64_t taken = total.b;
    scan_pair({refused, 0}, total, sums);  // its barriers also publish run_ends
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        row_offsets[B] = (int32_t)min(all_rows, (int64_t)INT32_MAX);
        *n_free_out = n_free - (int32_t)taken;
        counts[0] = n_runs;
        counts[1] = (int32_t)taken;
        counts[2] = (int32_t)total.a;
        counts[3] = (int32_t)min(all_rows, (int64_t)INT32_MAX);
    }
    for (int64_t i = (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; i < max_runs; i += (int64_t)gridDim.x * kPlanThreads) {
        int4 run{-1, 0, 0, 0};
        if (i < n_runs) {
            const int r = first_above(run_ends, B, (int32_t)i);
            const int64_t old = lengths[r], total_r = old + new_rows[r], have = blocks_of(old, S);
            const int64_t col = old / S + (i - (r ? run_ends[r - 1] : 0));
            int32_t *entry = table + (int64_t)r * width + col;
            if (col >= have) {
                run.x = free_blocks[n_free - 1 - (int32_t)(take0[r] + (col - have))];
                *entry = run.x;
            } else {
                run.x = *entry;
            }
            const int64_t first = max(old, col * S);  // row of the request that starts the run
            run.y = (int32_t)(row0[r] + (first - old));
            run.z = (int32_t)(first - col * S);
            run.w = (int32_t)(min(col * S + S, total_r) - first);
        }
        runs[i] = run;
    }
}

// The blocks of finished requests go to the end of the free list, in the order of the requests.
__global__ __launch_bounds__(kPlanThreads) void k_kv_release(
    const uint8_t *__restrict__ done, const int32_t *__restrict__ lengths, const int32_t *__restrict__ table, int32_t B,
    int32_t width, int32_t S, int32_t *__restrict__ free_blocks, int32_t free_capacity,
    const int32_t *__restrict__ n_free_in, int32_t *__restrict__ lengths_out, int32_t *__restrict__ n_free_out) {
    __shared__ int32_t ends_lds[kKvMaxRequests];
    __shared__ Pair sums[kPlanThreads / 64];
    const int32_t n_free = min(max(*n_free_in, 0), free_capacity);
    const int per = (B + kPlanThreads - 1) / kPlanThreads;
    const int b0 = min((int)threadIdx.x * per, B), b1 = min(b0 + per, B);
    auto held = [&](int b) { return done[b] ? min(blocks_of(max(lengths[b], 0), S), (int64_t)width) : (int64_t)0; };
    const int64_t room = free_capacity - n_free;  // a list that would overflow drops what does not fit
    Pair mine{0, 0}, total;
    for (int b = b0; b < b1; ++b) mine.a += held(b);
    int64_t at = scan_pair(mine, total, sums).a - mine.a;
    for (int b = b0; b < b1; ++b) {
        at += held(b);
        ends_lds[b] = (int32_t)min(at, room);
        if (blockIdx.x == 0) lengths_out[b] = done[b] ? 0 : lengths[b];
    }
    __syncthreads();
    const int32_t n = (int32_t)min(total.a, room);
    if (blockIdx.x == 0 && threadIdx.x == 0) *n_free_out = n_free + n;
    for (int64_t i = (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kPlanThreads) {
        const int r = first_above(ends_lds, B, (int32_t)i);
        free_blocks[n_free + i] = table[(int64_t)r * width + (i - (r ? ends_lds[r - 1] : 0))];
    }
}

// ---- writing ---------------------------------------------------------------------------------------------------------

template <class T>
__device__ float as_float(T x) { return (float)x; }

__device__ uint32_t byte_of(float x, float inv) {
    const float r = rintf(x * inv);
    // NaN fails both comparisons and becomes 0
    return r >= 127.f ? 255u : r <= -127.f ? 1u : (uint32_t)((r == r ? (int)r : 0) + 128);
}

// One workgroup per (run, head, K or V).  Two passes over the run's rows: the first finds max |x|, the second, which
// finds them in the L2, makes the codes.  Rows that the block held before keep their values, coded against the new scale.
template <class T>
__global__ __launch_bounds__(256) void k_kv_store(
    const T *__restrict__ k, const T *__restrict__ v, int64_t rows, int64_t k_row, int64_t k_head, int64_t v_row,
    int64_t v_head, const int4 *__restrict__ runs, KvCache c) {
    const int4 run = runs[blockIdx.x];
    const int32_t block = run.x, slot0 = run.z, n = run.w, h = blockIdx.y, S = c.S, d = c.d;
    const bool is_v = blockIdx.z;
    if (n < 1 || block < 0 || block >= c.n_blocks || slot0 < 0 || (int64_t)slot0 + n > S || run.y < 0 || (int64_t)run.y + n > rows)
        return;
    const int64_t stride = is_v ? v_row : k_row;
    const T *x = (is_v ? v + h * v_head : k + h * k_head) + run.y * stride;

    uint32_t top = 0;  // |x| as bits: their order is the numbers', and NaN is above infinity
    for (int i = threadIdx.x; i < n * d; i += 256) {
        const int r = i / d, e = i - r * d;
        top = max(top, __float_as_uint(as_float(x[r * stride + e])) & 0x7fffffffu);
    }
    for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    __shared__ uint32_t tops[4];
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));

    float *scale = c.scales + ((int64_t)block * c.H + h) * 2 + is_v;
    const float s_old = slot0 > 0 ? *scale : 0.f;
    float s = __uint_as_float(top) * (1.f / 127.f);
    if (s < kKvLeastScale) s = 0.f;
    s = __uint_as_float(max(__float_as_uint(s), __float_as_uint(s_old)));  // as bits: NaN stays
    const float inv = s > 0.f ? 1.f / s : 0.f;
    __syncthreads();
    if (threadIdx.x == 0) *scale = s;

    const int e16 = kv_padded(d);
    uint8_t *codes = c.codes + ((int64_t)block * c.H + h) * kv_slice_bytes(S, d);
    // a thread makes 16 bytes: of K, 16 dims of one slot; of V, 16 slots of one dim
    for (int u = threadIdx.x; u < S * e16 / 16; u += 256) {
        const int tile = u / (2 * e16), w = u - tile * 2 * e16;
        uint8_t *to = codes + (int64_t)tile * 64 * e16 + (is_v ? 32 * e16 : 0) + w * 16;
        uint4 word = *reinterpret_cast<const uint4 *>(to);
        uint32_t *word32 = reinterpret_cast<uint32_t *>(&word);
        for (int i = 0; i < 16; ++i) {
            const int slot = tile * 32 + (is_v ? kv_slot(w & 1, i) : w & 31);
            const int e = is_v ? w >> 1 : (w >> 5) * 16 + i;
            uint32_t byte = 128;
            if (e < d && slot < slot0 + n) {
                const uint32_t was = (word32[i >> 2] >> (8 * (i & 3))) & 255;
                byte = slot >= slot0 ? byte_of(as_float(x[(slot - slot0) * stride + e]), inv)
                                     : byte_of((float)((int)was - 128) * s_old, inv);
            }
            word32[i >> 2] = (word32[i >> 2] & ~(255u << (8 * (i & 3)))) | byte << (8 * (i & 3));
        }
        *reinterpret_cast<uint4 *>(to) = word;
    }
}

// ---- reading back ------------------------------------------------------------------------------------------------------

template <class T>
__global__ __launch_bounds__(256) void k_kv_load(KvCache c, const int32_t *__restrict__ table, int32_t width,
                                                 const int32_t *__restrict__ lengths, int32_t max_rows,
                                                 T *__restrict__ k, T *__restrict__ v) {
    const int tile = blockIdx.x, h = blockIdx.y, b = blockIdx.z, S = c.S, d = c.d, e16 = kv_padded(d);
    const int64_t length = min((int64_t)max(lengths[b], 0), (int64_t)width * S);
    const int row0 = tile * 32;
    int32_t block = -1;
    if (row0 < length) block = table[(int64_t)b * width + row0 / S];
    const bool there = block >= 0 && block < c.n_blocks;
    float2 scale{0.f, 0.f};
    const uint8_t *codes = c.codes;
    if (there) {
        scale = reinterpret_cast<const float2 *>(c.scales)[(int64_t)block * c.H + h];
        codes += ((int64_t)block * c.H + h) * kv_slice_bytes(S, d) + (int64_t)(row0 % S / 32) * 64 * e16;
    }
    for (int i = threadIdx.x; i < 32 * d; i += 256) {
        const int slot = i / d, e = i - slot * d, row = row0 + slot;
        if (row >= max_rows) break;
        const int64_t to = (((int64_t)b * max_rows + row) * c.H + h) * d + e;
        float kx = 0.f, vx = 0.f;
        if (there && row < length) {
            kx = (float)((int)codes[kv_k_byte(slot, e)] - 128) * scale.x;
            vx = (float)((int)codes[32 * e16 + kv_v_byte(slot, e)] - 128) * scale.y;
        }
        k[to] = (T)kx;
        v[to] = (T)vx;
    }
}

}  // namespace

hipError_t launch_kv_plan(const int32_t *lengths, const int32_t *new_rows, int32_t B, int32_t S, int64_t rows,
                          int32_t *table, int32_t width, const int32_t *free_blocks, int32_t free_capacity,
                          const int32_t *n_free, int32_t *lengths_out, int32_t *n_free_out, int32_t *row_offsets,
                          int32_t *runs, int32_t max_runs, int32_t *counts, hipStream_t st) {
    const int grid = std::min(256, (max_runs + kPlanThreads - 1) / kPlanThreads);
    k_kv_plan<<<grid, kPlanThreads, 0, st>>>(lengths, new_rows, B, S, rows, table, width, free_blocks, free_capacity, n_free,
                                             lengths_out, n_free_out, row_offsets, reinterpret_cast<int4 *>(runs), max_runs,
                                             counts);
    return hipGetLastError();
}

hipError_t launch_kv_release(const uint8_t *done, const int32_t *lengths, const int32_t *table, int32_t B, int32_t width,
                             int32_t S, int32_t *free_blocks, int32_t free_capacity, const int32_t *n_free,
                             int32_t *lengths_out, int32_t *n_free_out, hipStream_t st) {
    const int64_t most = std::min((int64_t)B * width, (int64_t)free_capacity);
    const int grid = (int)std::min<int64_t>(64, (most + kPlanThreads - 1) / kPlanThreads);
    k_kv_release<<<std::max(grid, 1), kPlanThreads, 0, st>>>(done, lengths, table, B, width, S, free_blocks, free_capacity,
                                                             n_free, lengths_out, n_free_out);
    return hipGetLastError();
}

hipError_t launch_kv_store(const void *k, const void *v, int32_t dtype, int64_t rows, int64_t k_row, int64_t k_head,
                           int64_t v_row, int64_t v_head, const int32_t *runs, int32_t n_runs, const KvCache &c,
                           hipStream_t st) {
    const dim3 grid(n_runs, c.H, 2);
    auto go = [&](auto x) {
        using T = decltype(x);
        k_kv_store<T><<<grid, 256, 0, st>>>(static_cast<const T *>(k), static_cast<const T *>(v), rows, k_row, k_head, v_row,
                                            v_head, reinterpret_cast<const int4 *>(runs), c);
    };
    dtype == DGQ_F32 ? go(float{}) : dtype == DGQ_F16 ? go(_Float16{}) : go(__bf16{});
    return hipGetLastError();
}

hipError_t launch_kv_load(const KvCache &c, const int32_t *table, int32_t width, const int32_t *lengths, int32_t B,
                          int32_t max_rows, int32_t dtype, void *k, void *v, hipStream_t st) {
    const dim3 grid((max_rows + 31) / 32, c.H, B);
    auto go = [&](auto x) {
        using T = decltype(x);
        k_kv_load<T><<<grid, 256, 0, st>>>(c, table, width, lengths, max_rows, static_cast<T *>(k), static_cast<T *>(v));
    };
    dtype == DGQ_F32 ? go(float{}) : dtype == DGQ_F16 ? go(_Float16{}) : go(__bf16{});
    return hipGetLastError();
}

}  // namespace dgq
