// Group norm over [pixels, channels] rows, the map between a residual block's convolutions.
//
//   x'[n, c] = x[n, c] + add[b, c];  over the rows of image b and the C / G channels of a group
//   m = mean x',  v = mean (x' - m)^2,  r = 1 / sqrt(v + eps)
//   t = ((x' - m) r w[c] + beta[c]) (1 + scale[b, c]) + shift[b, c],   y = t  or  t / (1 + exp(-t))
//
// For every channel of an image three numbers of fp32,
//   p = (m - add) rounded,  a = r w (1 + scale),  q = ((p - (m - add)) r w + beta) (1 + scale) + shift,
// so that t = (x - p) a + q: x - p loses nothing where x is near the mean, however far that is from 0.  Sums, m, r and these three
// are computed in 64 bits: x and x^2 of 32-bit numbers are exact there (but for the sums' own last bits), so E[x^2] - m^2 keeps
// fp32's accuracy up to means of some thousand deviations, and partial sums combine by plain addition, in an order of the sizes
// alone.  (The three instructions a value hide behind its bytes: a read of 168 MB takes 28.8 us with 64-bit sums and 28.2 with
// 32-bit ones.)
//
// Maps whose groups fit a workgroup's registers: k_gn_one, x crosses memory once.  Others: k_gn_sums over chunks of rows, then
// k_gn_apply, whose workgroups first add up their image's chunks (or k_gn_tables between the two, where those are many); x is
// read twice.  2 x 64 x 1280 fp32 takes 5.1 us, 2 x 4096 x 320 13.8, 16 x 4096 x 640 82 (a copy of it 63) and 1048576 x 128 fp16 135
// (101).
#include <algorithm>

#include "vectors.h"

namespace dgq {
namespace {

constexpr int kMaxThreads = 512;

// Bounds of image b in the rows: [start, end).
struct Images {
    const int32_t *offsets;  // null: every image has n rows
    int64_t n, rows;         // rows: of all images (packed)
    int32_t B;
    __device__ int64_t at(int32_t i) const { return min(max((int64_t)offsets[i], (int64_t)0), rows); }
    __device__ int64_t start(int32_t b) const { return offsets ? at(b) : b * n; }
    __device__ int64_t end(int32_t b) const { return offsets ? at(b + 1) : (b + 1) * n; }
    // The first packed image that ends behind row r, B if none does: a wavefront tests 64 at a time, so that a search is one or
    // two reads after one another (three above 4096 images).
    __device__ int32_t image(int64_t r) const {
        int32_t lo = 0, n = B;
        for (;;) {
            const int32_t step = (n + 63) >> 6;
            const uint64_t behind = __ballot(at(lo + min(((int32_t)(threadIdx.x & 63) + 1) * step, n)) > r);
            if (!behind) return lo + n;
            const int32_t f = __builtin_ctzll(behind) * step;
            lo += f;
            if (step == 1) return lo;
            n = min(step, n - f);
        }
    }
};

// Rows pr, pr + high, .. of those from r0 on and below r1 (of all maps there are less than 2^31).
__device__ int rows_of(int64_t r0, int64_t r1, int pr, int high) {
    const int32_t left = (int32_t)(r1 - r0) - pr;
    return left > 0 ? (int)(((uint32_t)left + high - 1) / (uint32_t)high) : 0;
}

// Chunks of P rows, one to a workgroup.  Images of one size are cut one by one (`per` chunks each); packed ones are cut across, so
// that ragged ones keep all workgroups busy, and a chunk that several images meet in is worked on image by image.  Image b's part
// of chunk c has the number c (one size) or c + b (packed): no two parts share one, and an image's follow one another.
struct Chunks {
    int64_t P;
    int32_t count, per;
    __device__ int32_t first(const Images &im, int32_t b) const { return im.offsets ? (int32_t)((uint32_t)im.start(b) / (uint32_t)P) + b : b * per; }
    __device__ int32_t parts(const Images &im, int32_t b) const {
        if (!im.offsets) return per;
        const int64_t s = im.start(b), e = im.end(b);
        return e > s ? (int32_t)((uint32_t)(e - 1) / (uint32_t)P - (uint32_t)s / (uint32_t)P) + 1 : 0;
    }
    // f(image, part, first row, row behind the last) for the images of chunk c.  (Offsets that do not ascend give wrong rows, but
    // rows of x, images below B and parts below count + B.)
    template <class F>
    __device__ void each(const Images &im, int32_t c, F f) const {
        if (!im.offsets) {
            const int32_t b = c / per;
            const int64_t r = b * im.n + (int64_t)(c - b * per) * P;
            f(b, c, r, min(r + P, (b + 1) * im.n));
            return;
        }
        int64_t r = c * P;
        const int64_t r1 = min(r + P, im.rows);
        while (r < r1) {
            const int32_t lo = im.image(r);
            if (lo >= im.B) return;
            const int64_t from = max(r, im.start(lo)), to = min(im.end(lo), r1);
            if (to > from) f(lo, c + lo, from, to);
            const int64_t next = max(from, to);
            if (next == r) return;  // (offsets that do not ascend)
            r = next;
        }
    }
};

// Where row r of image b lies.
struct Rows {
    int64_t batch, row;  // strides in elements; packed: batch unused
    __device__ int64_t at(const Images &im, int32_t b, int64_t r) const {
        return im.offsets ? r * row : b * batch + (r - b * im.n) * row;
    }
};

// A workgroup's threads: `width` of them side by side over the channels, one vector each, over `high` rows; threads behind that idle.
struct Shape {
    int32_t threads, width, slices;  // slices of `width` vectors over the channels (blockIdx.y)
};

// A thread's vector of a slice: channels c0 .. c0 + V - 1.  The last vector of all ends with the channels, and the first `again`
// of its values are the vector before's; `have`: values of its own (0: no vector).  Fewer channels than V: `have` values, no more.
template <int V>
struct Place {
    int pr, high, c_slice, wide, c0, again, have;
    bool on;  // a row and a vector
    __device__ Place(const Shape &sh, int32_t C) {
        const int tid = threadIdx.x;
        high = sh.threads / sh.width, wide = sh.width * V;
        pr = tid / sh.width;
        c_slice = blockIdx.y * wide;
        const int c = c_slice + (tid - pr * sh.width) * V;
        have = max(min(V, C - c), 0);
        again = C >= V && have > 0 ? V - have : 0;
        c0 = c - again;
        on = pr < high && have > 0;
    }
};

// ---- sums ------------------------------------------------------------------------------------------------------------
__device__ double2 sum_of(double2 a, double2 b) { return {a.x + b.x, a.y + b.y}; }
// over `lanes` (a power of two) neighbouring lanes
__device__ double2 lane_sums(double2 s, int lanes) {
    for (int d = lanes >> 1; d; d >>= 1) s = sum_of(s, {__shfl_xor(s.x, d), __shfl_xor(s.y, d)});
    return s;
}

// Sum of n entries, each lane's from `from` on and `stride` apart, sixteen reads at a time; over `lanes` neighbours.
__device__ double2 strided_sum(const double2 *entries, int64_t n, int from, int stride, int lanes) {
    constexpr int AT_ONCE = 16;
    double2 s{0, 0};
    for (int64_t i = from; i < n; i += AT_ONCE * stride) {
        double2 e[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) e[u] = i + u * stride < n ? entries[i + u * stride] : double2{0, 0};
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) s = sum_of(s, e[u]);
    }
    return lane_sums(s, lanes);
}

// A thread's n rows, `step` elements apart: f(index of the row, values).  kAhead loads are on their way while as many rows are
// worked on (64 bytes of them).  PAST: past the caches.
template <class T, int V, bool PAST>
struct RowsOf {
    static constexpr int kAhead = 4 * kVec<T> / V;
    using Vec = loose<T, V>;
    const T *row;
    int64_t step;
    int n, few;  // few: values to a row, where they fill no vector
    Vec now[kAhead];
    __device__ RowsOf(const T *first, int64_t step_, int n_, int few_) : row(first), step(step_), n(n_), few(few_) {
        if (!few) fetch(now, 0);
    }
    __device__ void fetch(Vec (&to)[kAhead], int i) const {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < n) {
                const Vec *from = reinterpret_cast<const Vec *>(row + (i + u) * step);
                to[u] = PAST ? load_past(from) : *from;
            }
    }
    template <class F>
    __device__ void each(F f) {
        float x[V];
        if (!few) {
            for (int i = 0; i < n; i += kAhead) {
                Vec next[kAhead];
                fetch(next, i + kAhead);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (i + u < n) {
#pragma unroll
                        for (int e = 0; e < V; ++e) x[e] = (float)now[u][e];
                        f(i + u, x);
                    }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) now[u] = next[u];
            }
        } else {
            for (int i = 0; i < n; ++i) {
                load_vector(row + i * step, few, x);
                f(i, x);
            }
        }
    }
};

// Bound by the bytes of x, and for small maps by the way from the kernel's arguments over x and LDS to the sums (4.7 us for 2 x
// 4096 x 320, of which the rows take 2.5).  add enters per channel: sum x' = sum x + n add, sum x'^2 = sum x^2 + 2 add sum x + n
// add^2. 16 x 4096 x 640 fp32: 30 us, 5.6 TB/s.  sums: [G][parts][met] double2, met: slices that a group's channels may lie in,
// that of its first channel first, 0 for those that they do not.
template <class T>
__global__ __launch_bounds__(kMaxThreads) void k_gn_sums(const T *__restrict__ x, Images im, Rows xs, Chunks ch, Shape sh, int32_t C,
                                                         int32_t G, const float *__restrict__ add, int64_t add_row,
                                                         double2 *__restrict__ sums, int32_t parts, int32_t met) {
    constexpr int V = kVec<T>;
    extern __shared__ double2 entries[];  // [values of a vector, or 1 where vectors end with their groups][high][width]
    const int tid = threadIdx.x;
    const Place<V> at(sh, C);
    const int high = at.high, c_slice = at.c_slice, c_end = min(c_slice + at.wide, C), Cg = C / G, each = Cg % V ? 1 : V;  // channels of an entry
    const int g_first = sh.slices > 1 ? c_slice / Cg : 0, g_end = sh.slices > 1 ? (c_end - 1) / Cg + 1 : G;  // groups of the slice
    // neighbouring lanes that share a group's entries
    int lanes = 64;
    while (lanes > 1 && lanes * (g_end - g_first) > sh.threads) lanes >>= 1;
    ch.each(im, blockIdx.x, [&](int32_t b, int32_t part, int64_t r0, int64_t r1) {
        double s[V] = {}, ss[V] = {};
        if (at.on) {
            const int n = rows_of(r0, r1, at.pr, high);
            RowsOf<T, V, false>(x + xs.at(im, b, r0 + at.pr) + at.c0, high * xs.row, n, C < V ? at.have : 0).each([&](int, const float (&f)[V]) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    s[i] += (double)f[i];
                    ss[i] = fma((double)f[i], (double)f[i], ss[i]);
                }
            });
            if (add)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const double d = j < at.again + at.have ? add[b * add_row + at.c0 + j] : 0.f;
                    ss[j] += d * (2 * s[j] + n * d);
                    s[j] += n * d;
                }
        }
        __syncthreads();
        if (each == 1) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i >= at.again) entries[(i - at.again) * sh.threads + tid] = {s[i], ss[i]};  // (none reads what that leaves out)
        } else {
            double2 sum{0, 0};
#pragma unroll
            for (int i = 0; i < V; ++i) sum = sum_of(sum, {s[i], ss[i]});
            entries[tid] = sum;
        }
        __syncthreads();
        // over the rows, into the first of them
        for (int e = tid; e < sh.width * (V / each); e += sh.threads) {
            const int i = e / sh.width;
            double2 *column = entries + i * sh.threads + (e - i * sh.width);
            double2 sum = column[0];
#pragma unroll 4
            for (int p = 1; p < high; ++p) sum = sum_of(sum, column[p * sh.width]);
            column[0] = sum;
        }
        __syncthreads();
        for (int g = g_first + tid / lanes; g < g_end; g += sh.threads / lanes) {
            const int lo = (max(g * Cg, c_slice) - c_slice) / each, end = (min((g + 1) * Cg, c_end) - c_slice) / each;
            double2 sum{0, 0};
            for (int e = lo + (tid & (lanes - 1)); e < end; e += lanes)
                sum = sum_of(sum, each == 1 ? entries[e % V * sh.threads + e / V] : entries[e]);
            sum = lane_sums(sum, lanes);
            if ((tid & (lanes - 1)) == 0) {
                double2 *to = sums + ((int64_t)g * parts + part) * met;
                if (met > 1) {
                    const int from = g * Cg / at.wide, n = ((g + 1) * Cg - 1) / at.wide + 1 - from;
                    if ((int)blockIdx.y == from)
                        for (int i = n; i < met; ++i) to[i] = {0, 0};
                    to += (int)blockIdx.y - from;
                }
                *to = sum;
            }
        }
    });
}

// What an image's channel is given,
struct Terms {
    float weight, bias, add, scale, shift;
    __device__ static Terms of(const NormTerms &t, const float *weight, const float *bias, int32_t b, int32_t c) {
        return {weight ? weight[c] : 1.f, bias ? bias[c] : 0.f, t.add ? t.add[b * t.add_row + c] : 0.f,
                t.scale ? t.scale[b * t.scale_row + c] : 0.f, t.shift ? t.shift[b * t.shift_row + c] : 0.f};
    }
};
// and its line, from the sums over its group's n values.
struct Line {
    float p, a, q;
};
struct Group {
    double m, r;
    Group() = default;
    __device__ Group(double2 s, double per, float eps) : m(s.x * per) {  // per: 1 / n
        double v = s.y * per - m * m;
        if (v < 0) v = 0;  // (not NaN)
        r = rsqrt(v + (double)eps);
    }
    __device__ Line line(const Terms &t) const {
        const double mean = m - (double)t.add;
        const float p = (float)mean;
        const double rw = r * (double)t.weight, one = 1 + (double)t.scale;
        return {p, (float)(rw * one), (float)((((double)p - mean) * rw + (double)t.bias) * one + (double)t.shift)};
    }
};

// ---- tables ----------------------------------------------------------------------------------------------------------
// One workgroup per (group, image), where an image has too many sums for all to add up.  Bound by latency (5 us).  tables: fp32
// [B][p, a, q][C].
__global__ __launch_bounds__(256) void k_gn_tables(const double2 *__restrict__ sums, int32_t parts, Images im, Chunks ch, int32_t met,
                                                   int32_t C, int32_t G, const float *__restrict__ weight, const float *__restrict__ bias,
                                                   float eps, NormTerms terms, float *__restrict__ tables) {
    __shared__ double2 wave_sums[4];
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, Cg = C / G;
    const int64_t first = ((int64_t)g * parts + ch.first(im, b)) * met, n_parts = (int64_t)ch.parts(im, b) * met;
    double2 s = strided_sum(sums + first, n_parts, tid, 256, 64);
    if ((tid & 63) == 0) wave_sums[tid >> 6] = s;
    __syncthreads();
    s = wave_sums[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) s = sum_of(s, wave_sums[w]);
    const Group group(s, 1 / ((double)(im.end(b) - im.start(b)) * Cg), eps);
    for (int c = g * Cg + tid; c < (g + 1) * Cg; c += 256) {
        const Line line = group.line(Terms::of(terms, weight, bias, b, c));
        float *t = tables + (int64_t)b * 3 * C + c;
        t[0] = line.p;
        t[C] = line.a;
        t[2 * (int64_t)C] = line.q;
    }
}

// ---- values ----------------------------------------------------------------------------------------------------------
// Bound by the bytes of x and y.  x and y may be one buffer.  tables null: every workgroup adds up its image's sums itself, its
// first rows on their way meanwhile: 2.7 us at 128 sums of 32 groups, and a launch less.  The second read of x and the writes of y
// go past the caches, so that more of x is still there: 16 x 4096 x 640 fp32 82 us for both kernels, 93 with writes alone, 108 with
// neither, and 113, 115 and 123 with a kernel behind that reads y.  Such a write wants whole lines: a vector is 16 bytes of y (8 bf16
// values to 32 bytes of fp32, 16 x up to 4096 x 640 packed: 62, by the 4 here 47).
template <class T, class Y>
__global__ __launch_bounds__(kMaxThreads) void k_gn_apply(const T *x, Images im, Rows xs, Chunks ch, Shape sh, int32_t C, int32_t G,
                                                          const float *__restrict__ tables, const double2 *__restrict__ sums,
                                                          int32_t parts, int32_t met, const float *__restrict__ weight,
                                                          const float *__restrict__ bias, float eps, NormTerms terms, int32_t silu_on,
                                                          Y *y) {
    constexpr int V = kVec<Y>;
    extern __shared__ float lines[];  // the groups' m and r, [p, a, q][width V + V]
    const int tid = threadIdx.x, Cg = C / G;
    const Place<V> at(sh, C);
    const int high = at.high, c_slice = at.c_slice, wide = at.wide;
    const bool same = static_cast<const void *>(x) == y;
    int lanes = 64;
    while (lanes > 1 && lanes * G > sh.threads) lanes >>= 1;
    ch.each(im, blockIdx.x, [&](int32_t b, int32_t, int64_t r0, int64_t r1) {
        float p[V], a[V], q[V];
        const float *from;
        int64_t stride;
        RowsOf<T, V, true> rows(x + xs.at(im, b, r0 + at.pr) + at.c0, high * xs.row, at.on ? rows_of(r0, r1, at.pr, high) : 0,
                       C < V ? at.have : 0);
        if (tables) {
            from = tables + (int64_t)b * 3 * C + at.c0;
            stride = C;
        } else {
            Group *groups = reinterpret_cast<Group *>(lines);
            float *to = lines + G * (sizeof(Group) / sizeof(float));
            const int64_t first = ch.first(im, b), n_parts = (int64_t)ch.parts(im, b) * met;
            const double per = 1 / ((double)(im.end(b) - im.start(b)) * Cg);
            // (the last vector of all may begin in front of its slice)
            const int c_first = max(c_slice - V, 0), c_end = min(c_slice + wide, C), room = wide + V;
            Terms mine{};
            if (c_first + tid < c_end) mine = Terms::of(terms, weight, bias, b, c_first + tid);
            __syncthreads();
            for (int g = tid / lanes; g < G; g += sh.threads / lanes) {
                const double2 s = strided_sum(sums + ((int64_t)g * parts + first) * met, n_parts, tid & (lanes - 1), lanes, lanes);
                if ((tid & (lanes - 1)) == 0) groups[g] = Group(s, per, eps);
            }
            __syncthreads();
            for (int c = c_first + tid; c < c_end; c += sh.threads) {
                const Line line = groups[c / Cg].line(c == c_first + tid ? mine : Terms::of(terms, weight, bias, b, c));
                float *t = to + c - c_first;
                t[0] = line.p, t[room] = line.a, t[2 * room] = line.q;
            }
            __syncthreads();
            from = to + at.c0 - c_first;
            stride = room;
        }
        if (!at.on) return;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < at.again + at.have) p[i] = from[i], a[i] = from[stride + i], q[i] = from[2 * stride + i];
            else p[i] = a[i] = q[i] = 0.f;
        Y *to = y + (r0 + at.pr) * C + at.c0;
        rows.each([&](int r, const float (&f)[V]) {
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = fmaf(f[i] - p[i], a[i], q[i]);
            if (silu_on)
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = silu(v[i]);
            Y *row = to + (int64_t)r * high * C;
            if (same && at.again) {  // what two vectors share is written by the first; the second may have read it anew
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i >= at.again) row[i] = (Y)v[i];
            } else {
                store_past(row, at.again + at.have, v);
            }
        });
    });
}

// ---- all in one ------------------------------------------------------------------------------------------------------
// One workgroup per (image, group) keeps its part of the map in registers, so that x crosses memory once: HELD vectors of a
// thread, `width` threads side by side over the group's channels (the last vector ends with the group, and what it shares with
// the one before counts there) and threads / width rows at a time.  Rows that do not fit are read twice.  A group is a stripe of
// the rows, cut inside lines of memory: an XCD gets neighbouring groups, so that its cache puts the lines together.
// Bound by latency where maps are small (2 x 64 x 1280 fp32 4 us on the GPU), by the longest image's 32 workgroups in 8 packed
// images of up to 4096 x 960 bf16 (37.5 us; a copy of the bytes 18), by lines that two XCDs write (25 % more than there are) above.
// Its stripes share lines, whose parts must meet in the caches: past them 16 x 4096 x 320 fp32 takes 120 us instead of 63.
template <class T, class Y, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void k_gn_one(const T *x, Images im, Rows xs, int32_t C, int32_t G, int32_t width,
                                                    const float *__restrict__ weight, const float *__restrict__ bias, float eps,
                                                    NormTerms terms, int32_t silu_on, Y *y) {
    constexpr int V = kVec<T>;
    using Vec = loose<T, V>;
    extern __shared__ float lines[];  // [p, a, q][C / G]
    __shared__ double2 wave_sums[THREADS / 64];
    const int n_all = im.B * G, each = (n_all + 7) / 8, id = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
    if (id >= n_all || (int)(blockIdx.x >> 3) >= each) return;
    // one size: the groups of an image on one XCD; packed: some groups of all images, whose sizes differ
    const int b = im.offsets ? id % im.B : id / G, g = im.offsets ? id / im.B : id % G;
    const int Cg = C / G, tid = threadIdx.x, pr = tid / width, v = tid - pr * width, high = THREADS / width;
    const int c = min(v * V, Cg - V), again = v * V - c, c0 = g * Cg + c;  // again: values that the vector before has too
    const int64_t r0 = im.start(b), r1 = im.end(b);
    if (r1 <= r0) return;
    const int n = pr < high ? rows_of(r0, r1, pr, high) : 0;  // rows of this thread
    const int64_t step = high * xs.row;
    const T *from = x + xs.at(im, b, r0 + pr) + c0;
    const double per = 1 / ((double)(r1 - r0) * Cg);

    Vec held[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (i < n) held[i] = *reinterpret_cast<const Vec *>(from + i * step);
    Terms mine{};
    if (tid < Cg) mine = Terms::of(terms, weight, bias, b, g * Cg + tid);
    double2 s{0, 0};
    // first pass over a thread's rows; PLAIN: nothing is added, no value counts elsewhere
    auto first = [&](auto plain) {
        float shift[V];
#pragma unroll
        for (int i = 0; i < V; ++i) shift[i] = terms.add ? terms.add[b * terms.add_row + c0 + i] : 0.f;
        auto count = [&](const Vec &w) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                double d = (double)(float)w[i];
                if constexpr (!decltype(plain)::value) {
                    d += (double)shift[i];
                    if (i < again) d = 0;
                }
                s.x += d;
                s.y = fma(d, d, s.y);
            }
        };
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < n) count(held[i]);
        for (int i = HELD; i < n; ++i) count(*reinterpret_cast<const Vec *>(from + i * step));
    };
    if (!terms.add && Cg % V == 0) first(std::true_type{});
    else first(std::false_type{});
    s = lane_sums(s, 64);
    if ((tid & 63) == 0) wave_sums[tid >> 6] = s;
    __syncthreads();
    s = wave_sums[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) s = sum_of(s, wave_sums[w]);
    const Group group(s, per, eps);
    for (int i = tid; i < Cg; i += THREADS) {
        const Line l = group.line(i == tid ? mine : Terms::of(terms, weight, bias, b, g * Cg + i));
        lines[i] = l.p, lines[Cg + i] = l.a, lines[2 * Cg + i] = l.q;
    }
    __syncthreads();
    if (n == 0) return;
    float p[V], a[V], q[V];
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = lines[c + e], a[e] = lines[Cg + c + e], q[e] = lines[2 * Cg + c + e];
    Y *to = y + (r0 + pr) * C + c0;
    auto value = [&](const Vec &w, float (&f)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = fmaf((float)w[e] - p[e], a[e], q[e]);
        if (silu_on)
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = silu(f[e]);
    };
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (i < n) {
            float f[V];
            value(held[i], f);
            store_vector(to + (int64_t)i * high * C, V, f);
        }
    for (int i = HELD; i < n; ++i) {  // y may be x: what two vectors share is written by the first, the second may have read it anew
        float f[V];
        value(*reinterpret_cast<const Vec *>(from + i * step), f);
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e >= again) to[(int64_t)i * high * C + e] = (Y)f[e];
    }
}

// ---- launches --------------------------------------------------------------------------------------------------------

// Of workgroups of half to all of `most` threads, the one with most threads that have a vector of their own, as long as few idle.
Shape shape_for(int32_t C, int V, int32_t most) {
    const int32_t vectors = (C + V - 1) / V, slices = (vectors + most - 1) / most, width = (vectors + slices - 1) / slices;
    int32_t best = 0, threads = most;
    for (int32_t t = most / 2; t <= most; t += 64) {
        const int32_t used = t / width * width;
        if (used > best && 8 * used >= 7 * t) best = used, threads = t;
    }
    return {threads, width, slices};
}

constexpr int64_t kChunks = 256;  // workgroups of the two streaming kernels, one to a CU: more add their own beginnings and ends
Chunks chunks_for(const NormCall &n, const Shape &sh) {
    const int64_t rows = n.rows(), high = sh.threads / sh.width;
    auto up = [&](int64_t r) { return (r + high - 1) / high * high; };
    if (n.offsets) {
        const int64_t P = up((rows + kChunks - 1) / kChunks);
        return {P, (int32_t)((rows + P - 1) / P), 0};
    }
    // chunks of an image alike, in the number of rounds that costs least: a round takes its rows and some 5 us, 100 KB of them
    const int64_t extra = 100000 / ((int64_t)n.C * (n.dtype == DGQ_F32 ? 4 : 2));
    int64_t per = 1, least = INT64_MAX;
    for (int64_t rounds = 1; rounds <= 4; ++rounds) {
        const int64_t p = std::min(std::max<int64_t>(kChunks * rounds / n.B, 1), (n.N + high - 1) / high);
        const int64_t cost = (p * n.B + kChunks - 1) / kChunks * (up((n.N + p - 1) / p) + extra);
        if (cost < least) least = cost, per = p;
    }
    const int64_t P = up((n.N + per - 1) / per);
    per = (n.N + P - 1) / P;
    return {P, (int32_t)(per * n.B), (int32_t)per};
}

constexpr int64_t kMaxFolded = 16384;  // sums of an image that every workgroup may read

// Whether a workgroup can hold an image's group, and how: threads and vectors of each (0: it cannot, or is slower).  Many values
// keep its vector pipes busy and need most CUs to keep up: 2 x 1024 x 1280 fp32 10.7 us, 14.1 with sums of chunks, but 2 x 4096
// x 320 16.7 and 13.9, 4 x 4096 x 320 18.3 and 16.8.  A group's stripe of the rows touches lines of memory that others touch
// too, and no access of it can go past the caches: large maps of stripes below a line or two are faster in chunks (16 x 4096 x
// 320 fp32 63 and 44, 16 x 4096 x 640 bf16 67 and 49, 32 x 1024 x 320 bf16 22.8 and 19.7; 16 x 1024 x 640 fp32 22 and 25, 32 x
// 1024 x 1280 83 and 90).  Of packed images the host knows the rows of all, so a long one is taken to have 1.5 times the mean's;
// what a thread does not hold it reads twice, and a much longer image keeps 32 workgroups busy while the others are done (8
// images x 960 bf16, 16384 rows: even ones 37.5 us, nearly all in one 298; in chunks 39 and 60.  But chunks take some 10 us for
// every image in them: 16 x 1024 x 1280 fp32 40 and 52, 65535 images x 16 rows x 64 channels in one group 183 and 1794).  A
// launch has fewer than 2^32 threads: what needs more (2^24 groups of 256 threads, 2^22 of 1024) is cut in chunks too.
struct Hold {
    int32_t threads = 0, held = 0, width = 0;
};
int64_t one_grid(const NormCall &n) { return 8 * (((int64_t)n.B * n.G + 7) / 8); }  // workgroups: as many to every XCD
Hold hold_for(const NormCall &n) {
    const int32_t V = n.dtype == DGQ_F32 ? 4 : 8, Cg = n.C / n.G, width = (Cg + V - 1) / V;
    if (Cg < V || width > 256) return {};
    const int64_t rows = n.offsets ? n.N / n.B * 3 / 2 : n.N;  // of a long image
    if ((rows > 2048 || rows * Cg > 65536) && (int64_t)n.B * n.G < 192) return {};
    const int64_t stripe = Cg * (16 / V), bytes = n.rows() * n.C * (16 / V);
    if ((stripe < 128 && bytes >= 44000000) || (stripe < 32 && bytes >= 20000000)) return {};
    const Hold ways[] = {{256, 4, width}, {1024, 4, width}, {1024, 8, width}, {1024, 16, width}};
    for (const Hold &h : ways)
        if (rows <= (int64_t)h.held * (h.threads / width))
            return one_grid(n) * h.threads <= (int64_t)UINT32_MAX ? h : Hold{};  // (wider ways ask for more)
    return {};
}

struct NormPlan {
    Hold hold;
    Shape shape;
    Chunks chunks;
    int32_t parts = 0, met = 1;  // met: slices that a group's channels may lie in
    size_t sums_bytes = 0, tables_bytes = 0;  // tables_bytes 0: the last kernel makes them itself
    explicit NormPlan(const NormCall &n) : hold(hold_for(n)), shape(shape_for(n.C, n.dtype == DGQ_F32 ? 4 : 8, kMaxThreads)), chunks(chunks_for(n, shape)) {
        if (hold.held) return;
        parts = chunks.count + (n.offsets ? n.B : 0);
        const int32_t Cg = n.C / n.G, wide = shape.width * (n.dtype == DGQ_F32 ? 4 : 8);
        if (wide % Cg) met = std::min(shape.slices, Cg % wide ? (Cg - 1) / wide + 2 : Cg / wide);
        sums_bytes = (size_t)n.G * parts * met * sizeof(double2);
        if (n.G > 2048 || (int64_t)n.G * shape.slices * (n.offsets ? parts : chunks.per) > kMaxFolded) tables_bytes = (size_t)n.B * 3 * n.C * sizeof(float);
    }
};

template <class T, class Y>
hipError_t launch_one(const NormCall &n, const Hold &h, const Images &im, const Rows &xs, hipStream_t st) {
    const T *x = static_cast<const T *>(n.x);
    Y *y = static_cast<Y *>(n.out);
    const unsigned grid = (unsigned)one_grid(n);
    hipError_t e = hipSuccess;
    auto go = [&](auto threads, auto held) {
        constexpr int THREADS = decltype(threads)::value;
        constexpr int HELD = decltype(held)::value;
        const int bytes = 3 * (n.C / n.G) * (int)sizeof(float);
        e = DGQ_ENSURE_LDS((k_gn_one<T, Y, THREADS, HELD>), bytes);
        if (e == hipSuccess)
            k_gn_one<T, Y, THREADS, HELD><<<grid, THREADS, bytes, st>>>(x, im, xs, n.C, n.G, h.width, n.weight, n.bias, n.eps,
                                                                        n.terms, n.act == DGQ_ACT_SILU, y);
    };
    constexpr std::integral_constant<int, 1024> all{};
    if (h.threads == 256) go(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
    else if (h.held == 4) go(all, std::integral_constant<int, 4>{});
    else if (h.held == 8) go(all, std::integral_constant<int, 8>{});
    else go(all, std::integral_constant<int, 16>{});
    return e;
}

}  // namespace

size_t groupnorm_workspace_bytes(const NormCall &n) {
    const NormPlan p(n);
    return p.sums_bytes + p.tables_bytes;
}

int groupnorm_kernel(const NormCall &n) {
    const NormPlan p(n);
    if (!p.hold.held) return p.tables_bytes ? 1 : 0;
    return p.hold.threads == 256 ? 10 : p.hold.held == 4 ? 11 : p.hold.held == 8 ? 12 : 13;
}

hipError_t launch_groupnorm(const NormCall &n, void *workspace, hipStream_t st) {
    const NormPlan p(n);
    const Images im{n.offsets, n.N, n.rows(), n.B};
    const Rows xs{n.x_batch, n.x_row};
    double2 *sums = static_cast<double2 *>(workspace);
    float *tables = p.tables_bytes ? reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + p.sums_bytes) : nullptr;
    const dim3 grid(p.chunks.count, p.shape.slices);
    hipError_t e = hipSuccess;
    by_dtype(n.dtype, [&](auto xt) {
        using T = decltype(xt);
        const T *x = static_cast<const T *>(n.x);
        if (!p.hold.held) {
            const int bytes = p.shape.threads * (int)sizeof(double2) * (n.C / n.G % kVec<T> ? kVec<T> : 1);
            e = DGQ_ENSURE_LDS(k_gn_sums<T>, bytes);
            if (e != hipSuccess) return;
            k_gn_sums<T><<<grid, p.shape.threads, bytes, st>>>(x, im, xs, p.chunks, p.shape, n.C, n.G, n.terms.add, n.terms.add_row,
                                                               sums, p.parts, p.met);
            if (tables)
                k_gn_tables<<<dim3(n.G, n.B), 256, 0, st>>>(sums, p.parts, im, p.chunks, p.met, n.C, n.G, n.weight, n.bias,
                                                            n.eps, n.terms, tables);
        }
        by_output<T>(n.out_dtype, [&](auto yt) {
            using Y = decltype(yt);
            Y *y = static_cast<Y *>(n.out);
            if (p.hold.held) {
                e = launch_one<T, Y>(n, p.hold, im, xs, st);
                return;
            }
            const Shape shape = shape_for(n.C, kVec<Y>, kMaxThreads);
            const int bytes = tables ? 0 : n.G * (int)sizeof(Group) + 3 * (shape.width + 1) * kVec<Y> * (int)sizeof(float);
            e = DGQ_ENSURE_LDS((k_gn_apply<T, Y>), bytes);
            if (e == hipSuccess)
                k_gn_apply<T, Y><<<dim3(p.chunks.count, shape.slices), shape.threads, bytes, st>>>(
                    x, im, xs, p.chunks, shape, n.C, n.G, tables, sums, p.parts, p.met, n.weight, n.bias, n.eps, n.terms,
                    n.act == DGQ_ACT_SILU, y);
        });
    });
    return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace dgq
