// Group norm with an activation, channels last: y = act(gamma (x - mean) / sqrt(var + eps) + beta), mean and var over the
// P pixels and D channels of a group of one image.
#include "norm_common.h"

namespace gspc {

// Where block (n, chunk, slab) leaves its part of group g: a group that a slab's end cuts has a part in either, and
// consecutive slabs' parts do not meet in g + slab.
__host__ __device__ __forceinline__ size_t norm_parts(const NormShape &h, const NormGrid &g) { return (size_t)h.groups + g.slabs - 1; }

// Mean and sum of squared deviations of each group over a block's rows.  A thread sums x - x0 and its square, x0 its first value
// of the channel, so that an offset of the channel does not cancel; the threads' means and deviations are joined as such
// (total deviation = sum of the parts' own + sum of count * (part's mean - mean)^2), never as sums of squares.
template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void norm_stats_kernel(NormShape h, NormGrid g, const T *__restrict__ x, size_t ldx,
                                                                  float2 *__restrict__ parts, int lanes) {
    __shared__ float s_mean[kNormThreads * V], s_dev[kNormThreads * V];
    const NormBlock b = norm_block(h, g, blockIdx.x);
    const int width = b.c1 - b.c0;
    if (b.active) {
        const T *p = x + ((size_t)b.n * h.P + b.r0) * ldx + b.at;
        float first[V], sum[V] = {}, sq[V] = {};
        int count = 0;
        for (int r = b.ty; r < b.r1 - b.r0; r += 4 * g.TY) {
            Raw<T, V> raw[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (r + k * g.TY < b.r1 - b.r0) raw[k] = fetch<V>(p + (size_t)(r + k * g.TY) * ldx);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (r + k * g.TY < b.r1 - b.r0) {
                    float v[V];
                    widen(raw[k], v);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if (count == 0) first[e] = v[e];
                        const float d = v[e] - first[e];
                        sum[e] += d;
                        sq[e] = fmaf(d, d, sq[e]);
                    }
                    ++count;
                }
        }
        const float inv = 1.f / (float)count;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = b.at + e - b.c0;
            const float m = sum[e] * inv;
            if (c >= 0 && count) {
                s_mean[b.ty * width + c] = first[e] + m;
                s_dev[b.ty * width + c] = fmaxf(sq[e] - sum[e] * m, 0.f);
            }
        }
    }
    __syncthreads();
    const int rows = b.r1 - b.r0, TY = min(g.TY, rows);
    const int g0 = b.c0 / h.D, g1 = (b.c1 - 1) / h.D, lane = threadIdx.x & (lanes - 1);
    for (int k = g0 + threadIdx.x / lanes; k <= g1; k += blockDim.x / lanes) {
        const int lo = max(k * h.D, b.c0) - b.c0, hi = min((k + 1) * h.D, b.c1) - b.c0, n = (hi - lo) * TY;
        // (the rows of thread ty: all have rows / TY, the first rows % TY one more)
        const int each = rows / TY, more = rows - each * TY;
        float mean = 0.f, dev = 0.f;
        for (int i = lane; i < n; i += lanes) {
            const int ty = i / (hi - lo), c = lo + i - ty * (hi - lo);
            mean += s_mean[ty * width + c] * (float)(each + (ty < more));
        }
        mean = lanes_sum(mean, lanes) / ((float)rows * (float)(hi - lo));
        for (int i = lane; i < n; i += lanes) {
            const int ty = i / (hi - lo), c = lo + i - ty * (hi - lo);
            const float d = s_mean[ty * width + c] - mean;
            dev += s_dev[ty * width + c] + d * d * (float)(each + (ty < more));
        }
        dev = lanes_sum(dev, lanes);
        if (lane == 0)
            parts[((size_t)b.n * g.chunks + b.chunk) * norm_parts(h, g) + k + b.c0 / kSlab] = make_float2(mean, dev);
    }
}

// The blocks' parts joined: stats[n][g] = mean, 1 / sqrt(var + eps).  16 lanes for a group of an image.
__global__ __launch_bounds__(256) void norm_join_kernel(NormShape h, NormGrid g, const float2 *__restrict__ parts, float eps,
                                                        float2 *__restrict__ stats) {
    const unsigned pair = (blockIdx.x * 256 + threadIdx.x) / 16, lane = threadIdx.x & 15;
    if (pair >= (unsigned)h.N * h.groups) return;
    const int n = pair / h.groups, k = pair - n * h.groups;
    const int s0 = (k * h.D) / kSlab, s1 = ((k + 1) * h.D - 1) / kSlab, count = (s1 - s0 + 1) * g.chunks;
    const float2 *p = parts + (size_t)n * g.chunks * norm_parts(h, g) + k;
    const auto weight = [&](int s, int chunk) {
        const int channels = min((k + 1) * h.D, (s + 1) * kSlab) - max(k * h.D, s * kSlab);
        return (float)channels * (float)(min(h.P - chunk * g.rows, g.rows));
    };
    const float total = (float)h.P * (float)h.D;
    float mean = 0.f, dev = 0.f;
    for (int i = lane; i < count; i += 16) {
        const int s = s0 + i / g.chunks, chunk = i % g.chunks;
        mean += p[chunk * norm_parts(h, g) + s].x * weight(s, chunk);
    }
    mean = lanes_sum(mean, 16) / total;
    for (int i = lane; i < count; i += 16) {
        const int s = s0 + i / g.chunks, chunk = i % g.chunks;
        const float2 v = p[chunk * norm_parts(h, g) + s];
        const float d = v.x - mean;
        dev += v.y + d * d * weight(s, chunk);
    }
    dev = lanes_sum(dev, 16);
    if (lane == 0) stats[pair] = make_float2(mean, 1.f / sqrtf(dev / total + eps));
}

// What a channel's values are multiplied with: z = (x - mean) a + b, a = gamma / sqrt(var + eps).  (x a + (b - mean a) would
// save an operation and lose what mean a has more than z.)
template <int V> struct Affine {
    float mean[V], a[V], b[V];
};
template <int V>
__device__ __forceinline__ void load_affine(const NormShape &h, const float2 *__restrict__ stats, const float *__restrict__ gamma,
                                            const float *__restrict__ beta, int n, int at, Affine<V> &f) {
    const float2 *st = stats + (size_t)n * h.groups;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float2 s = st[(at + e) / h.D];
        f.mean[e] = s.x;
        f.a[e] = s.y * (gamma ? gamma[at + e] : 1.f);
        f.b[e] = beta ? beta[at + e] : 0.f;
    }
}
template <int V> __device__ __forceinline__ void apply_affine(const Affine<V> &f, int act, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = fmaf(v[e] - f.mean[e], f.a[e], f.b[e]);
    activate_all(act, v);
}

// y as fp32 or bf16: threads keep their channels' coefficients and walk down the rows.
template <typename TX, typename TY, int V>
__global__ __launch_bounds__(kNormThreads) void norm_apply_kernel(NormShape h, NormGrid g, const TX *__restrict__ x, size_t ldx,
                                                                  const float2 *__restrict__ stats, const float *__restrict__ gamma,
                                                                  const float *__restrict__ beta, TY *__restrict__ y, size_t ldy) {
    const NormBlock b = norm_block(h, g, blockIdx.x);
    if (!b.active) return;
    Affine<V> f;
    load_affine<V>(h, stats, gamma, beta, b.n, b.at, f);
    const size_t row0 = (size_t)b.n * h.P + b.r0;
    const TX *p = x + row0 * ldx + b.at;
    TY *q = y + row0 * ldy + b.at;
    for (int r = b.ty; r < b.r1 - b.r0; r += 4 * g.TY) {
        Raw<TX, V> raw[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (r + k * g.TY < b.r1 - b.r0) raw[k] = fetch<V>(p + (size_t)(r + k * g.TY) * ldx);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (r + k * g.TY < b.r1 - b.r0) {
                float v[V];
                widen(raw[k], v);
                apply_affine<V>(f, h.act, v);
                store(q + (size_t)(r + k * g.TY) * ldy, v);
            }
    }
}

// Outputs in 8-bit rows need all of a row's channels: `width` lanes hold one row, HELD vectors each with their coefficients, and
// walk down the rows of an image (HELD = 0: rows of any length, read and computed twice).  TY = int8_t: y is 8-bit rows;
// SAVE: x is written as 8-bit rows too.
template <typename TX, typename TY, int V, int HELD, bool SAVE>
__global__ __launch_bounds__(256) void norm_rows_kernel(NormShape h, int width, int blocks, int rows, unsigned m_blocks,
                                                        const TX *__restrict__ x, size_t ldx, const float2 *__restrict__ stats,
                                                        const float *__restrict__ gamma, const float *__restrict__ beta,
                                                        TY *__restrict__ y, size_t ldy, float *__restrict__ y_scale,
                                                        int8_t *__restrict__ saved, float *__restrict__ saved_scale) {
    constexpr bool CODES = sizeof(TY) == 1;
    constexpr int H = HELD ? HELD : 1;
    const int n = fast_div_any(blockIdx.x, blocks, m_blocks), lane = threadIdx.x & (width - 1);
    const int r0 = ((int)blockIdx.x - n * blocks) * rows, r1 = min(r0 + rows, h.P);
    const int nv = vectors_of<V>(h.C), pitch = rows8_pitch(h.C);
    Affine<V> f[H];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (lane + k * width < nv) load_affine<V>(h, stats, gamma, beta, n, vector_start<V>(lane + k * width, h.C), f[k]);
    }
    for (int r = r0 + threadIdx.x / width; r < r1; r += 256 / width) {
        const size_t row = (size_t)n * h.P + r;
        const TX *p = x + row * ldx;
        unsigned top_x = 0, top_y = 0;
        float v[H][V];
        const auto each = [&](auto body) {       // body(first channel, its values, its coefficients, loop count)
            if constexpr (HELD > 0) {
#pragma unroll
                for (int k = 0; k < HELD; ++k)
                    if (lane + k * width < nv) body(vector_start<V>(lane + k * width, h.C), v[k], f[k]);
            } else {
                for (int i = lane; i < nv; i += width) {
                    const int at = vector_start<V>(i, h.C);
                    widen(fetch<V>(p + at), v[0]);
                    load_affine<V>(h, stats, gamma, beta, n, at, f[0]);
                    body(at, v[0], f[0]);
                }
            }
        };
        if constexpr (HELD > 0) {
            Raw<TX, V> raw[H];
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (lane + k * width < nv) raw[k] = fetch<V>(p + vector_start<V>(lane + k * width, h.C));
#pragma unroll
            for (int k = 0; k < HELD; ++k)
                if (lane + k * width < nv) widen(raw[k], v[k]);
        }
        if constexpr (SAVE) {
            each([&](int, float (&t)[V], Affine<V> &) {
#pragma unroll
                for (int e = 0; e < V; ++e) top_x = max(top_x, magnitude(t[e]));
            });
            const RowCode c = row_code(lanes_umax(top_x, width));
            each([&](int at, float (&t)[V], Affine<V> &) { store_codes(saved + row * pitch + at, t, c); });
            for (int i = h.C + lane; i < pitch; i += width) saved[row * pitch + i] = 0;
            if (lane == 0) saved_scale[row] = c.scale;
        }
        if constexpr (CODES) {
            each([&](int, float (&t)[V], Affine<V> &fk) {
                apply_affine<V>(fk, h.act, t);
#pragma unroll
                for (int e = 0; e < V; ++e) top_y = max(top_y, magnitude(t[e]));
            });
            const RowCode c = row_code(lanes_umax(top_y, width));
            each([&](int at, float (&t)[V], Affine<V> &fk) {
                if constexpr (HELD == 0) apply_affine<V>(fk, h.act, t);
                store_codes(reinterpret_cast<int8_t *>(y) + row * pitch + at, t, c);
            });
            for (int i = h.C + lane; i < pitch; i += width) reinterpret_cast<int8_t *>(y)[row * pitch + i] = 0;
            if (lane == 0) y_scale[row] = c.scale;
        } else {
            each([&](int at, float (&t)[V], Affine<V> &fk) {
                apply_affine<V>(fk, h.act, t);
                store(y + row * ldy + at, t);
            });
        }
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
static size_t forward_bytes(const NormShape &h, const NormGrid &g) {
    return (size_t)h.N * g.chunks * norm_parts(h, g) * sizeof(float2) + (size_t)h.N * h.groups * sizeof(float2);
}

size_t norm_forward_bytes(const NormShape &h) { return forward_bytes(h, norm_grid(h, 2048)); }

template <typename TX, typename TY, int V, bool SAVE>
static void launch_rows(const NormShape &h, const NormForward &f, const float2 *stats, hipStream_t s) {
    const int nv = vectors_of<V>(h.C);
    int width = 1;
    while (width < nv && width < kWave) width *= 2;
    const int each = (nv + width - 1) / width;
    const auto kern = V == 1 || each <= 1 ? norm_rows_kernel<TX, TY, V, 1, SAVE>
                    : each <= 2 ? norm_rows_kernel<TX, TY, V, 2, SAVE>
                    : each <= 4 ? norm_rows_kernel<TX, TY, V, 4, SAVE> : norm_rows_kernel<TX, TY, V, 0, SAVE>;
    const int at_once = 256 / width;
    long blocks = 2048 / h.N + 1;
    const long most = (h.P + 4L * at_once - 1) / (4L * at_once);
    if (blocks > most) blocks = most;
    const int rows = (int)((h.P + blocks - 1) / blocks);
    blocks = (h.P + rows - 1) / rows;
    hipLaunchKernelGGL(kern, dim3((unsigned)(blocks * h.N)), dim3(256), 0, s, h, width, (int)blocks, rows, div_magic((unsigned)blocks),
                       static_cast<const TX *>(f.x), f.ldx, stats, f.gamma, f.beta, static_cast<TY *>(f.y), f.ldy, f.y_scale, f.saved,
                       f.saved_scale);
}

template <typename TX, int V>
static hipError_t forward(const NormShape &h, const NormForward &f, void *ws, hipStream_t s, const char **name) {
    const NormGrid g = norm_grid(h, 2048);
    const TX *x = static_cast<const TX *>(f.x);
    float2 *parts = static_cast<float2 *>(ws);
    float2 *stats = f.stats ? reinterpret_cast<float2 *>(f.stats) : parts + (size_t)h.N * g.chunks * norm_parts(h, g);
    const dim3 grid((unsigned)((size_t)h.N * g.chunks * g.slabs));
    hipLaunchKernelGGL((norm_stats_kernel<TX, V>), grid, dim3(g.threads), 0, s, h, g, x, f.ldx, parts, group_lanes(g.TY * (h.D < kSlab ? h.D : kSlab)));
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(((size_t)h.N * h.groups * 16 + 255) / 256)), dim3(256), 0, s, h, g, parts, f.eps, stats);
    if (f.y_dtype == GSPC_I8) {
        *name = "norm_rows<i8>";
        if (f.saved) launch_rows<TX, int8_t, V, true>(h, f, stats, s);
        else launch_rows<TX, int8_t, V, false>(h, f, stats, s);
    } else if (f.saved) {
        *name = "norm_rows<saved>";
        if (f.y_dtype == GSPC_F32) launch_rows<TX, float, V, true>(h, f, stats, s);
        else launch_rows<TX, uint16_t, V, true>(h, f, stats, s);
    } else {
        *name = "norm_apply";
        if (f.y_dtype == GSPC_F32)
            hipLaunchKernelGGL((norm_apply_kernel<TX, float, V>), grid, dim3(g.threads), 0, s, h, g, x, f.ldx, stats, f.gamma, f.beta,
                               static_cast<float *>(f.y), f.ldy);
        else
            hipLaunchKernelGGL((norm_apply_kernel<TX, uint16_t, V>), grid, dim3(g.threads), 0, s, h, g, x, f.ldx, stats, f.gamma, f.beta,
                               static_cast<uint16_t *>(f.y), f.ldy);
    }
    return hipGetLastError();
}

hipError_t launch_norm_forward(const NormShape &h, const NormForward &f, void *ws, hipStream_t s, const char **name) {
    if (f.x_dtype == GSPC_F32) return h.C >= 8 ? forward<float, 8>(h, f, ws, s, name) : forward<float, 1>(h, f, ws, s, name);
    return h.C >= 8 ? forward<uint16_t, 8>(h, f, ws, s, name) : forward<uint16_t, 1>(h, f, ws, s, name);
}

}  // namespace gspc
