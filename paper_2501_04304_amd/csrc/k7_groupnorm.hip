// Group norm over [pixels, channels] rows, the map between a residual block's convolutions.
//
//   x'[n, c] = x[n, c] + add[b, c];  over the rows of image b and the C / G channels of a group
//   m = mean x',  v = mean (x' - m)^2,  r = 1 / sqrt(v + eps)
//   t = ((x' - m) r w[c] + beta[c]) (1 + scale[b, c]) + shift[b, c],   y = t  or  t / (1 + exp(-t))
//
// Three launches.  k_gn_sums: sum and sum of squares of every group over chunks of rows.  k_gn_tables: an image's chunks summed in
// order, and for every channel three numbers of fp32,
//   p = (m - add) rounded,  a = r w (1 + scale),  q = ((p - (m - add)) r w + beta) (1 + scale) + shift,
// so that t = (x - p) a + q: x - p loses nothing where x is near the mean, however far that is from 0.  k_gn_apply: that line and
// the activation for every value.  Sums and tables are in 64 bits: x and x^2 of 32-bit numbers are exact there (but for the
// sums' own last bits), so E[x^2] - m^2 keeps fp32's accuracy up to means of some thousand standard deviations, and partial sums
// combine by plain addition.  add enters the sums per channel: sum x' = sum x + n add, sum x'^2 = sum x^2 + 2 add sum x + n add^2.
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
};

// Chunks of P rows, one to a workgroup.  Images of one size are cut one by one (`per` chunks each); packed ones are cut across, so
// that ragged ones keep all workgroups busy, and a chunk that several images meet in is worked on image by image.  Image b's part
// of chunk c has the number c (one size) or c + b (packed): no two parts share one, and an image's follow one another.
struct Chunks {
    int64_t P;
    int32_t count, per;
    __device__ int32_t first(const Images &im, int32_t b) const { return im.offsets ? (int32_t)(im.start(b) / P) + b : b * per; }
    __device__ int32_t parts(const Images &im, int32_t b) const {
        if (!im.offsets) return per;
        const int64_t s = im.start(b), e = im.end(b);
        return e > s ? (int32_t)((e - 1) / P - s / P) + 1 : 0;
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
            int32_t lo = 0, hi = im.B;
            while (lo < hi) {
                const int32_t mid = (lo + hi) >> 1;
                if (im.at(mid + 1) > r) hi = mid; else lo = mid + 1;
            }
            if (lo == im.B) return;
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

// ---- sums ------------------------------------------------------------------------------------------------------------
// Bound by the bytes of x.  sums: [G][parts][slices] double2.
template <class T>
__global__ __launch_bounds__(kMaxThreads) void k_gn_sums(const T *__restrict__ x, Images im, Rows xs, Chunks ch, Shape sh, int32_t C,
                                                         int32_t G, const float *__restrict__ add, int64_t add_row,
                                                         double2 *__restrict__ sums, int32_t parts) {
    constexpr int V = kVec<T>;
    extern __shared__ double channel[];  // [high][width V]
    const int tid = threadIdx.x, lane = tid & 63, high = sh.threads / sh.width, wide = sh.width * V;
    const int pr = tid / sh.width, c_slice = blockIdx.y * wide, c0 = c_slice + (tid - pr * sh.width) * V, have = min(V, C - c0);
    const bool on = pr < high && have > 0;
    const int Cg = C / G, c_end = min(c_slice + wide, C);
    ch.each(im, blockIdx.x, [&](int32_t b, int32_t part, int64_t r0, int64_t r1) {
        double s[V] = {}, ss[V] = {};
        int64_t n = 0;
        if (on) {
            const T *row = x + xs.at(im, b, r0 + pr) + c0;
            for (int64_t r = r0 + pr; r < r1; r += high, row += high * xs.row) {
                float f[V];
                load_vector(row, have, f);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    s[i] += (double)f[i];
                    ss[i] = fma((double)f[i], (double)f[i], ss[i]);
                }
                ++n;
            }
            if (add)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const double d = i < have ? add[b * add_row + c0 + i] : 0.f;
                    ss[i] += d * (2 * s[i] + n * d);
                    s[i] += n * d;
                }
        }
        double sum = 0;
        for (int pass = 0; pass < 2; ++pass) {
            __syncthreads();
            if (pr < high)
#pragma unroll
                for (int i = 0; i < V; ++i) channel[tid * V + i] = pass ? ss[i] : s[i];
            __syncthreads();
            // a wavefront per group
            for (int g = tid >> 6; g < G; g += sh.threads >> 6) {
                const int lo = max(g * Cg, c_slice), n_here = min((g + 1) * Cg, c_end) - lo;
                sum = 0;
                for (int e = lane; e < n_here * high; e += 64) sum += channel[e / n_here * wide + (lo - c_slice) + e % n_here];
#pragma unroll
                for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
                if (lane == 0) {
                    double *to = reinterpret_cast<double *>(sums + ((int64_t)g * parts + part) * sh.slices + blockIdx.y);
                    to[pass] = sum;
                }
            }
        }
    });
}

// ---- tables ----------------------------------------------------------------------------------------------------------
// One workgroup per (group, image).  Bound by latency.  tables: fp32 [B][p, a, q][C].
__global__ __launch_bounds__(256) void k_gn_tables(const double2 *__restrict__ sums, int32_t parts, Images im, Chunks ch, int32_t slices,
                                                   int32_t C, int32_t G, const float *__restrict__ weight, const float *__restrict__ bias,
                                                   float eps, NormTerms terms, float *__restrict__ tables) {
    __shared__ double2 wave_sums[4];
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, Cg = C / G;
    const int64_t first = ((int64_t)g * parts + ch.first(im, b)) * slices, n_parts = (int64_t)ch.parts(im, b) * slices;
    double2 s{0, 0};
    for (int64_t i = tid; i < n_parts; i += 256) {
        const double2 p = sums[first + i];
        s.x += p.x, s.y += p.y;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) s.x += __shfl_xor(s.x, d), s.y += __shfl_xor(s.y, d);
    if ((tid & 63) == 0) wave_sums[tid >> 6] = s;
    __syncthreads();
    s = wave_sums[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) s.x += wave_sums[w].x, s.y += wave_sums[w].y;
    const double n = (double)(im.end(b) - im.start(b)) * Cg, m = s.x / n;
    double v = s.y / n - m * m;
    if (v < 0) v = 0;  // (not NaN)
    const double r = 1 / sqrt(v + (double)eps);
    for (int c = g * Cg + tid; c < (g + 1) * Cg; c += 256) {
        const double mean = terms.add ? m - (double)terms.add[b * terms.add_row + c] : m;
        const float p = (float)mean;
        const double rw = weight ? r * (double)weight[c] : r, one = terms.scale ? 1 + (double)terms.scale[b * terms.scale_row + c] : 1.0;
        const double q = (((double)p - mean) * rw + (bias ? (double)bias[c] : 0.0)) * one;
        float *t = tables + (int64_t)b * 3 * C + c;
        t[0] = p;
        t[C] = (float)(rw * one);
        t[2 * (int64_t)C] = (float)(terms.shift ? q + (double)terms.shift[b * terms.shift_row + c] : q);
    }
}

// ---- values ----------------------------------------------------------------------------------------------------------
// Bound by the bytes of x and y.  x and y may be one buffer: a thread writes what it alone has read.
template <class T, class Y, bool SILU>
__global__ __launch_bounds__(kMaxThreads) void k_gn_apply(const T *x, Images im, Rows xs, Chunks ch, Shape sh, int32_t C,
                                                          const float *__restrict__ tables, Y *y) {
    constexpr int V = kVec<T>;
    const int tid = threadIdx.x, high = sh.threads / sh.width, pr = tid / sh.width;
    const int c0 = (blockIdx.y * sh.width + tid - pr * sh.width) * V, have = min(V, C - c0);
    if (pr >= high || have <= 0) return;
    ch.each(im, blockIdx.x, [&](int32_t b, int32_t, int64_t r0, int64_t r1) {
        float p[V], a[V], q[V];
        const float *t = tables + (int64_t)b * 3 * C + c0;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < have) p[i] = t[i], a[i] = t[C + i], q[i] = t[2 * (int64_t)C + i];
            else p[i] = a[i] = q[i] = 0.f;
        const T *from = x + xs.at(im, b, r0 + pr) + c0;
        Y *to = y + (r0 + pr) * C + c0;
        for (int64_t r = r0 + pr; r < r1; r += high, from += high * xs.row, to += (int64_t)high * C) {
            float f[V];
            load_vector(from, have, f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[i] = fmaf(f[i] - p[i], a[i], q[i]);
                if (SILU) f[i] = silu(f[i]);
            }
            store_vector(to, have, f);
        }
    });
}

// ---- launches --------------------------------------------------------------------------------------------------------

// Most threads that have a vector of their own, of workgroups of 4 to 8 wavefronts.
Shape shape_for(int32_t C, int V) {
    const int32_t vectors = (C + V - 1) / V, slices = (vectors + kMaxThreads - 1) / kMaxThreads, width = (vectors + slices - 1) / slices;
    int32_t best = 0, threads = 0;
    for (int32_t t = 256; t <= kMaxThreads; t += 64) {
        const int32_t used = 1024 * (t / width * width) / t;  // share in use
        if (used > best) best = used, threads = t;
    }
    return {threads, width, slices};
}

Chunks chunks_for(const NormCall &n, const Shape &sh, int64_t most) {
    const int64_t rows = n.rows(), high = sh.threads / sh.width;
    int64_t P = (rows + most - 1) / most;
    P = (P + high - 1) / high * high;
    if (n.offsets) return {P, (int32_t)((rows + P - 1) / P), 0};
    const int64_t per = (n.N + P - 1) / P;
    P = ((n.N + per - 1) / per + high - 1) / high * high;  // the chunks of an image alike
    return {P, (int32_t)(per * n.B), (int32_t)per};
}

constexpr int64_t kChunks = 1024;

struct NormPlan {
    Shape shape;
    Chunks chunks;
    int32_t parts;
    size_t sums_bytes, tables_bytes;
    explicit NormPlan(const NormCall &n) : shape(shape_for(n.C, n.dtype == DGQ_F32 ? 4 : 8)), chunks(chunks_for(n, shape, kChunks)) {
        parts = chunks.count + (n.offsets ? n.B : 0);
        sums_bytes = (size_t)n.G * parts * shape.slices * sizeof(double2);
        tables_bytes = (size_t)n.B * 3 * n.C * sizeof(float);
    }
};

}  // namespace

size_t groupnorm_workspace_bytes(const NormCall &n) {
    const NormPlan p(n);
    return p.sums_bytes + p.tables_bytes;
}

hipError_t launch_groupnorm(const NormCall &n, void *workspace, hipStream_t st) {
    const NormPlan p(n);
    const Images im{n.offsets, n.N, n.rows(), n.B};
    const Rows xs{n.x_batch, n.x_row};
    double2 *sums = static_cast<double2 *>(workspace);
    float *tables = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + p.sums_bytes);
    const dim3 grid(p.chunks.count, p.shape.slices);
    by_dtype(n.dtype, [&](auto xt) {
        using T = decltype(xt);
        const T *x = static_cast<const T *>(n.x);
        k_gn_sums<T><<<grid, p.shape.threads, p.shape.threads * kVec<T> * sizeof(double), st>>>(
            x, im, xs, p.chunks, p.shape, n.C, n.G, n.terms.add, n.terms.add_row, sums, p.parts);
        k_gn_tables<<<dim3(n.G, n.B), 256, 0, st>>>(sums, p.parts, im, p.chunks, p.shape.slices, n.C, n.G, n.weight, n.bias, n.eps,
                                                    n.terms, tables);
        by_output<T>(n.out_dtype, [&](auto yt) {
            using Y = decltype(yt);
            Y *y = static_cast<Y *>(n.out);
            if (n.act == DGQ_ACT_SILU)
                k_gn_apply<T, Y, true><<<grid, p.shape.threads, 0, st>>>(x, im, xs, p.chunks, p.shape, n.C, tables, y);
            else
                k_gn_apply<T, Y, false><<<grid, p.shape.threads, 0, st>>>(x, im, xs, p.chunks, p.shape, n.C, tables, y);
        });
    });
    return hipGetLastError();
}

}  // namespace dgq
