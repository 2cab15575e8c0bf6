// Group norm with an activation, channels last: y = act(gamma (x - mean) / sqrt(var + eps) + beta), mean and var over the
// P pixels and D channels of a group of one image.
#include "norm_common.h"

namespace gspc {

// Where block (n, chunk, slab) leaves its part of group g: a group that a slab's end cuts has a part in either, and
// consecutive slabs' parts do not meet in g + slab.
__host__ __device__ __forceinline__ size_t norm_parts(const NormShape &h, const NormGrid &g) { return (size_t)h.groups + g.slabs - 1; }

// Mean and sum of squared deviations of each group over a block's rows.  A thread sums x - x0 and its square, x0 its first value
// (of the channel, or of the vector where all its channels are of one group: ONE), so that an offset does not cancel; the threads'
// means and deviations are joined as such (total deviation = sum of the parts' own + sum of count * (part's mean - mean)^2), never
// as sums of squares.  Bound by memory: 64 images of 56x56, 256 channels in bf16, 18.4 us, 5.6 TB/s (43 with sums across lanes
// through LDS).
template <typename T, int V, bool ONE>
__global__ __launch_bounds__(kNormThreads) void norm_stats_kernel(NormShape h, NormGrid g, const T *__restrict__ x, size_t ldx,
                                                                  float2 *__restrict__ parts, int lanes) {
    constexpr int E = ONE ? 1 : V, DEEP = sizeof(T) == 4 ? 4 : 8;
    __shared__ float s_mean[kNormThreads * E], s_dev[kNormThreads * E];
    const NormBlock b = norm_block(h, g, blockIdx.x);
    const int width = ONE ? b.nv : b.c1 - b.c0, rows = b.r1 - b.r0;
    if (b.active) {
        const T *p = x + ((size_t)b.n * h.P + b.r0 + b.ty) * ldx + b.at;
        const size_t step = g.TY * ldx;
        float first[E], sum[E] = {}, sq[E] = {};
        int count = 0;
        for (int r = b.ty; r < rows; r += DEEP * g.TY) {
            Raw<T, V> raw[DEEP];
#pragma unroll
            for (int k = 0; k < DEEP; ++k, p += step)
                if (r + k * g.TY < rows) raw[k] = fetch<V>(p);
#pragma unroll
            for (int k = 0; k < DEEP; ++k)
                if (r + k * g.TY < rows) {
                    float v[V];
                    widen(raw[k], v);
                    if (k == 0 && count == 0) {
#pragma unroll
                        for (int e = 0; e < E; ++e) first[e] = v[e];
                    }
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int f = ONE ? 0 : e;
                        const float d = v[e] - first[f];
                        sum[f] += d;
                        sq[f] = fmaf(d, d, sq[f]);
                    }
                    ++count;
                }
        }
        const float inv = 1.f / (float)(count * (V / E));
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = ONE ? b.tx : b.at + e - b.c0;
            const float m = sum[e] * inv;
            if (c >= 0 && count) {
                s_mean[b.ty * width + c] = first[e] + m;
                s_dev[b.ty * width + c] = fmaxf(sq[e] - sum[e] * m, 0.f);
            }
        }
    }
    __syncthreads();
    constexpr int U = V / E;                        // channels behind one of these
    const int TY = min(g.TY, rows), each = rows / TY, more = rows - each * TY;   // thread ty had each + (ty < more) rows
    const int g0 = group_of(h, b.c0), g1 = group_of(h, b.c1 - 1), lane = threadIdx.x & (lanes - 1);
    for (int k = g0 + threadIdx.x / lanes; k <= g1; k += blockDim.x / lanes) {
        const int lo = (max(k * h.D, b.c0) - b.c0) / U, hi = (min((k + 1) * h.D, b.c1) - b.c0) / U, wide = hi - lo;
        const unsigned mul = div_magic(wide);
        float mean = 0.f, dev = 0.f;
        for (int i = lane; i < wide * TY; i += lanes) {
            const int ty = fast_div(i, mul);
            mean += s_mean[ty * width + lo + i - ty * wide] * (float)(each + (ty < more));
        }
        mean = lanes_sum(mean, lanes) / ((float)rows * (float)wide);
        for (int i = lane; i < wide * TY; i += lanes) {
            const int ty = fast_div(i, mul), at = ty * width + lo + i - ty * wide;
            const float d = s_mean[at] - mean;
            dev += s_dev[at] + d * d * (float)((each + (ty < more)) * U);
        }
        dev = lanes_sum(dev, lanes);
        if (lane == 0)
            parts[((size_t)b.n * g.chunks + b.chunk) * norm_parts(h, g) + k + b.c0 / kSlab] = make_float2(mean, dev);
    }
}

// The blocks' parts of group k of image n joined by kJoinLanes lanes (always as many: the same statistics, whoever joins them): mean,
// 1 / sqrt(var + eps).
constexpr int kJoinLanes = kWave;
__device__ __forceinline__ float2 join_parts(const NormShape &h, const NormGrid &g, const float2 *__restrict__ parts, int n, int k, float eps,
                                             int lane) {
    constexpr int lanes = kJoinLanes;
    const int s0 = (k * h.D) / kSlab, s1 = ((k + 1) * h.D - 1) / kSlab, count = (s1 - s0 + 1) * g.chunks;
    const float2 *p = parts + (size_t)n * g.chunks * norm_parts(h, g) + k;
    const auto weight = [&](int s, int chunk) {
        const int channels = min((k + 1) * h.D, (s + 1) * kSlab) - max(k * h.D, s * kSlab);
        return (float)channels * (float)(min(h.P - chunk * g.rows, g.rows));
    };
    const float total = (float)h.P * (float)h.D;
    const auto part = [&](int i, float &w) {
        const int s = fast_div_any(i, g.chunks, g.m_chunks), chunk = i - s * g.chunks;
        w = weight(s0 + s, chunk);
        return p[chunk * norm_parts(h, g) + s0 + s];
    };
    constexpr int HELD = 4;                         // parts that a lane loads once, all at the same time
    float2 v[HELD];
    float w[HELD], mean = 0.f, dev = 0.f;
#pragma unroll
    for (int j = 0; j < HELD; ++j)
        if (lane + j * lanes < count) v[j] = part(lane + j * lanes, w[j]);
#pragma unroll
    for (int j = 0; j < HELD; ++j)
        if (lane + j * lanes < count) mean += v[j].x * w[j];
    for (int i = lane + HELD * lanes; i < count; i += lanes) {
        float wi;
        const float2 vi = part(i, wi);
        mean += vi.x * wi;
    }
    mean = lanes_sum(mean, lanes) / total;
#pragma unroll
    for (int j = 0; j < HELD; ++j)
        if (lane + j * lanes < count) dev += v[j].y + (v[j].x - mean) * (v[j].x - mean) * w[j];
    for (int i = lane + HELD * lanes; i < count; i += lanes) {
        float wi;
        const float2 vi = part(i, wi);
        dev += vi.y + (vi.x - mean) * (vi.x - mean) * wi;
    }
    dev = lanes_sum(dev, lanes);
    return make_float2(mean, 1.f / sqrtf(dev / total + eps));
}

__global__ __launch_bounds__(256) void norm_join_kernel(NormShape h, NormGrid g, const float2 *__restrict__ parts, float eps,
                                                        float2 *__restrict__ stats) {
    const unsigned pair = (blockIdx.x * 256 + threadIdx.x) / kJoinLanes, lane = threadIdx.x % kJoinLanes;
    if (pair >= (unsigned)h.N * h.groups) return;
    const float2 s = join_parts(h, g, parts, pair / h.groups, pair % h.groups, eps, lane);
    if (lane == 0) stats[pair] = s;
}

// An image's groups that a block of norm_apply_kernel joins itself instead, and the parts behind them: in small launches, where a
// third one costs more (in 2048 blocks, 64 images of 56x56, 256 channels: 10 us).
constexpr int kFoldGroups = 64, kFoldParts = 1024, kFoldBlocks = 512;

// What a channel's values are multiplied with: z = (x - mean) a + b, a = gamma / sqrt(var + eps).  (x a + (b - mean a) would
// save an operation and lose what mean a has more than z.)
template <int V> struct Affine {
    float mean[V], a[V], b[V];
};
template <int V>
__device__ __forceinline__ void load_affine(const NormShape &h, const float2 *__restrict__ stats, const float *__restrict__ gamma,
                                            const float *__restrict__ beta, int at, Affine<V> &f) {
    load_params<V>(gamma, at, 1.f, f.a);
    load_params<V>(beta, at, 0.f, f.b);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float2 s = stats[group_of(h, at + e)];
        f.mean[e] = s.x;
        f.a[e] *= s.y;
    }
}
template <int V> __device__ __forceinline__ void apply_affine(const Affine<V> &f, int act, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = fmaf(v[e] - f.mean[e], f.a[e], f.b[e]);
    activate_all(act, v);
}

// y as fp32 or bf16: threads keep their channels' coefficients and walk down the rows, one batch of loads ahead of the values that
// they multiply (and ahead of the coefficients' own loads: those are a second trip to memory; with them first an image of 7x7 took 6.8 us).
// 64 images of 56x56, 256 channels in bf16 with SiLU: 31.6 us, x partly from the cache that the
// statistics left it in.  SiLU is 58 clocks for 64 values (16 each for the exponential and the reciprocal): 22 us of that.
// FOLD: the block joins the parts of its image's groups itself; stats, where asked for, are then an output.
template <typename TX, typename TY, int V, bool FOLD>
__global__ __launch_bounds__(kNormThreads) void norm_apply_kernel(NormShape h, NormGrid g, const TX *__restrict__ x, size_t ldx,
                                                                  const float2 *__restrict__ parts, float eps, float2 *__restrict__ stats,
                                                                  const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                  TY *__restrict__ y, size_t ldy, int past) {
    constexpr int DEEP = 4;
    __shared__ float2 s_stats[FOLD ? kFoldGroups : 1];
    const NormBlock b = norm_block(h, g, blockIdx.x);
    const size_t row0 = (size_t)b.n * h.P + b.r0 + b.ty;
    const int rows = b.r1 - b.r0;
    const TX *p = x + row0 * ldx + b.at;
    TY *q = y + row0 * ldy + b.at;
    Raw<TX, V> raw[DEEP], next[DEEP];
    const auto load = [&](int r, Raw<TX, V> (&to)[DEEP]) {
#pragma unroll
        for (int k = 0; k < DEEP; ++k, p += g.TY * ldx)
            if (r + k * g.TY < rows) to[k] = fetch<V>(p);
    };
    if (b.active) load(b.ty, raw);
    if constexpr (FOLD) {
        const int lane = threadIdx.x % kJoinLanes;
        for (int k = threadIdx.x / kJoinLanes; k < h.groups; k += g.threads / kJoinLanes) {
            const float2 s = join_parts(h, g, parts, b.n, k, eps, lane);
            if (lane == 0) {
                s_stats[k] = s;
                if (stats && b.chunk == 0 && b.c0 == 0) stats[(size_t)b.n * h.groups + k] = s;
            }
        }
        __syncthreads();
    }
    if (!b.active) return;
    Affine<V> f;
    load_affine<V>(h, FOLD ? s_stats : stats + (size_t)b.n * h.groups, gamma, beta, b.at, f);
    for (int r = b.ty; r < rows; r += DEEP * g.TY) {
        load(r + DEEP * g.TY, next);
#pragma unroll
        for (int k = 0; k < DEEP; ++k, q += g.TY * ldy)
            if (r + k * g.TY < rows) {
                float v[V];
                widen(raw[k], v);
                apply_affine<V>(f, h.act, v);
                store(q, v, past);
            }
#pragma unroll
        for (int k = 0; k < DEEP; ++k) raw[k] = next[k];
    }
}

// Outputs in 8-bit rows need all of a row's channels: `width` lanes hold one row, HELD vectors each with their coefficients, and
// walk down the rows of an image, several at a time so that their loads are in flight together (HELD = 0: rows of any length,
// read and computed twice).  TY = int8_t: y is 8-bit rows; SAVE: x is written as 8-bit rows too.  64 images of 14x14, 512 channels
// to 8-bit rows 9.3 us, half of it arithmetic; 256 of 28x28, 128 channels with SAVE 24.9 us, 128 MB.
template <typename TX, typename TY, int V, int HELD, bool SAVE>
__global__ __launch_bounds__(256) void norm_rows_kernel(NormShape h, int log_width, int blocks, int rows, unsigned m_blocks,
                                                        const TX *__restrict__ x, size_t ldx, const float2 *__restrict__ stats,
                                                        const float *__restrict__ gamma, const float *__restrict__ beta,
                                                        TY *__restrict__ y, size_t ldy, float *__restrict__ y_scale,
                                                        int8_t *__restrict__ saved, float *__restrict__ saved_scale, int past) {
    constexpr bool CODES = sizeof(TY) == 1;
    constexpr int H = HELD ? HELD : 1, DEEP = HELD == 1 ? 2 : 1;
    const int n = fast_div_any(blockIdx.x, blocks, m_blocks), width = 1 << log_width, lane = threadIdx.x & (width - 1);
    const int r0 = ((int)blockIdx.x - n * blocks) * rows, count = min(rows, h.P - r0), slots = 256 >> log_width;
    const int nv = vectors_of<V>(h.C), pitch = rows8_pitch(h.C);
    const size_t row0 = (size_t)n * h.P + r0;
    stats += (size_t)n * h.groups;
    Raw<TX, V> raw[DEEP][H], next[DEEP][H];
    const auto load = [&](int r, Raw<TX, V> (&to)[DEEP][H]) {
        if constexpr (HELD > 0) {
#pragma unroll
            for (int d = 0; d < DEEP; ++d)
#pragma unroll
                for (int k = 0; k < HELD; ++k)
                    if (r + d * slots < count && lane + k * width < nv)
                        to[d][k] = fetch<V>(x + (row0 + r + d * slots) * ldx + vector_start<V>(lane + k * width, h.C));
        }
    };
    load(threadIdx.x >> log_width, raw);
    Affine<V> f[H];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (lane + k * width < nv) load_affine<V>(h, stats, gamma, beta, vector_start<V>(lane + k * width, h.C), f[k]);
    }
    for (int r = threadIdx.x >> log_width; r < count; r += DEEP * slots) {
        load(r + DEEP * slots, next);
#pragma unroll
        for (int d = 0; d < DEEP; ++d) {
            if (r + d * slots >= count) continue;
            const size_t row = row0 + r + d * slots;
            float v[H][V];
            const auto each = [&](auto body) {       // body(first channel, its values, its coefficients)
                if constexpr (HELD > 0) {
#pragma unroll
                    for (int k = 0; k < HELD; ++k)
                        if (lane + k * width < nv) body(vector_start<V>(lane + k * width, h.C), v[k], f[k]);
                } else {
                    for (int i = lane; i < nv; i += width) {
                        const int at = vector_start<V>(i, h.C);
                        widen(fetch<V>(x + row * ldx + at), v[0]);
                        load_affine<V>(h, stats, gamma, beta, at, f[0]);
                        body(at, v[0], f[0]);
                    }
                }
            };
            if constexpr (HELD > 0) {
#pragma unroll
                for (int k = 0; k < HELD; ++k)
                    if (lane + k * width < nv) widen(raw[d][k], v[k]);
            }
            if constexpr (SAVE) {
                unsigned top = 0;
                each([&](int, float (&t)[V], Affine<V> &) {
#pragma unroll
                    for (int e = 0; e < V; ++e) top = max(top, magnitude(t[e]));
                });
                const RowCode c = row_code(lanes_umax(top, width));
                each([&](int at, float (&t)[V], Affine<V> &) { store_codes(saved + row * pitch + at, t, c); });
                for (int i = h.C + lane; i < pitch; i += width) saved[row * pitch + i] = 0;
                if (lane == 0) saved_scale[row] = c.scale;
            }
            if constexpr (CODES) {
                unsigned top = 0;
                each([&](int, float (&t)[V], Affine<V> &fk) {
                    apply_affine<V>(fk, h.act, t);
#pragma unroll
                    for (int e = 0; e < V; ++e) top = max(top, magnitude(t[e]));
                });
                const RowCode c = row_code(lanes_umax(top, width));
                each([&](int at, float (&t)[V], Affine<V> &fk) {
                    if constexpr (HELD == 0) apply_affine<V>(fk, h.act, t);
                    store_codes(reinterpret_cast<int8_t *>(y) + row * pitch + at, t, c);
                });
                for (int i = h.C + lane; i < pitch; i += width) reinterpret_cast<int8_t *>(y)[row * pitch + i] = 0;
                if (lane == 0) y_scale[row] = c.scale;
            } else {
                each([&](int at, float (&t)[V], Affine<V> &fk) {
                    apply_affine<V>(fk, h.act, t);
                    store(y + row * ldy + at, t, past);
                });
            }
        }
        if constexpr (HELD > 0) {
#pragma unroll
            for (int d = 0; d < DEEP; ++d)
#pragma unroll
                for (int k = 0; k < HELD; ++k) raw[d][k] = next[d][k];
        }
    }
}

// All of it in one launch, x read once: a block holds its channels of an image in registers, HELD vectors a thread, takes the
// mean, then the squared deviations from it, then writes y (TY = void: only the statistics).  ONE: a vector's channels are of
// one group (D a multiple of 8).  Bound by memory where it fills the chip: 256 images of 28x28, 128 channels in bf16 with SiLU
// 20 us, 5.1 TB/s (65 in two passes as they were first written, 39 as they are); one image of 7x7, 512 channels 3.7 us, a launch.
template <typename TX, typename TY, int V, int HELD, bool ONE>
__global__ __launch_bounds__(512) void norm_held_kernel(NormShape h, HeldGrid g, const TX *__restrict__ x, size_t ldx,
                                                        const float *__restrict__ gamma, const float *__restrict__ beta, float eps,
                                                        float2 *__restrict__ stats, TY *__restrict__ y, size_t ldy, int past) {
    constexpr int E = ONE ? 1 : V;                  // groups, and sums, of a vector
    extern __shared__ float part[];                 // [slots][seg / unit], then the groups' results
    const unsigned block = held_block(g, blockIdx.x), n = fast_div_any(block, g.segs, g.m_segs);
    const int c0 = (block - n * g.segs) * g.seg, groups = ONE ? g.seg / 8 / g.units : g.seg / h.D;
    const int lane = threadIdx.x & ((1 << g.log_width) - 1), slot = threadIdx.x >> g.log_width;
    const int nv = vectors_of<V>(g.seg), row = ONE ? nv : g.seg, at = vector_start<V>(lane, g.seg);
    const bool on = lane < nv;
    float *group_mean = part + g.slots * row, *group_rstd = group_mean + groups;

    const size_t token = (size_t)n * h.P + slot;
    Raw<TX, V> raw[HELD];
    {
        const TX *p = x + token * ldx + c0 + at;
#pragma unroll
        for (int k = 0; k < HELD; ++k, p += g.slots * ldx)
            if (slot + k * g.slots < h.P && on) raw[k] = fetch<V>(p);
    }
    float a[V], b[V];
    if constexpr (!std::is_void<TY>::value) {
        load_params<V>(gamma, c0 + (on ? at : 0), 1.f, a);
        load_params<V>(beta, c0 + (on ? at : 0), 0.f, b);
    }
    int group[E];
#pragma unroll
    for (int e = 0; e < E; ++e) group[e] = on ? fast_div(ONE ? lane : at + e, g.m_units) : 0;

    const auto each = [&](auto body) {
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (slot + k * g.slots < h.P && on) {
                float v[V];
                hold(raw[k]);
                widen(raw[k], v);
                body(v);
            }
            __builtin_amdgcn_sched_barrier(0);      // one token's values at a time: the raw ones fill the registers
        }
    };
    const auto leave = [&](const float (&sum)[E]) {
        if (on) {
#pragma unroll
            for (int e = 0; e < E; ++e) part[slot * row + (ONE ? lane : at) + e] = sum[e];   // (shared channels: the same sum twice)
        }
        __syncthreads();
    };
    const float m = (float)h.P * (float)h.D;
    float mean[E];
    {
        float sum[E] = {};
        each([&](float (&v)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) sum[ONE ? 0 : e] += v[e];
        });
        leave(sum);
        held_group_sums(g, part, row, groups, [&](int k, float s) { group_mean[k] = s / m; });
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) mean[e] = group_mean[group[e]];
    }
    {
        float sum[E] = {};
        each([&](float (&v)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = v[e] - mean[ONE ? 0 : e];
                sum[ONE ? 0 : e] = fmaf(d, d, sum[ONE ? 0 : e]);
            }
        });
        leave(sum);
        held_group_sums(g, part, row, groups, [&](int k, float s) {
            const float r = 1.f / sqrtf(s / m + eps);
            group_rstd[k] = r;
            if (stats) stats[(size_t)n * h.groups + group_of(h, c0) + k] = make_float2(group_mean[k], r);
        });
    }
    if constexpr (!std::is_void<TY>::value) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) a[e] *= group_rstd[group[ONE ? 0 : e]];
        TY *q = y + token * ldy + c0 + at;
        each([&](float (&v)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = fmaf(v[e] - mean[ONE ? 0 : e], a[e], b[e]);
            activate_all(h.act, v);
            store(q, v, past);
            q += g.slots * ldy;
        });
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
constexpr int kForwardBlocks = 2048, kForwardChunks = 256;

template <typename TX, typename TY, int V, bool SAVE>
static void launch_rows(const NormShape &h, const NormForward &f, const float2 *stats, hipStream_t s) {
    const int nv = vectors_of<V>(h.C);
    int log_width = 0;
    while ((1 << log_width) < nv && log_width < 6) ++log_width;
    const int width = 1 << log_width, each = (nv + width - 1) / width;
    const auto kern = V == 1 || each <= 1 ? norm_rows_kernel<TX, TY, V, 1, SAVE>
                    : each <= 2 ? norm_rows_kernel<TX, TY, V, 2, SAVE>
                    : each <= 4 ? norm_rows_kernel<TX, TY, V, 4, SAVE> : norm_rows_kernel<TX, TY, V, 0, SAVE>;
    const int at_once = 256 / width;
    // (blocks of two rows a lane: with four and a quarter as many blocks 64 images of 14x14, 512 channels took 9.8 us instead of 8.8)
    long blocks = 8192 / h.N + 1;
    const long most = (h.P + 2L * at_once - 1) / (2L * at_once);
    if (blocks > most) blocks = most;
    const int rows = (int)((h.P + blocks - 1) / blocks);
    blocks = (h.P - 1) / rows + 1;
    hipLaunchKernelGGL(kern, dim3((unsigned)(blocks * h.N)), dim3(256), 0, s, h, log_width, (int)blocks, rows, div_magic((unsigned)blocks),
                       static_cast<const TX *>(f.x), f.ldx, stats, f.gamma, f.beta, static_cast<TY *>(f.y), f.ldy, f.y_scale, f.saved,
                       f.saved_scale, f.past);
}

// Vectors that a thread of norm_held_kernel holds at most: 64 registers of raw values.
template <typename TX> constexpr int held_most() { return sizeof(TX) == 4 ? 8 : 16; }

template <typename TX, typename TY, int V, bool ONE>
static void launch_held(const NormShape &h, const HeldGrid &g, const NormForward &f, float2 *stats, hipStream_t s) {
    constexpr int MOST = held_most<TX>();
    const int held = (h.P - 1) / g.slots + 1, row = ONE ? g.seg / 8 : g.seg;
    const auto kern = held <= 2 ? norm_held_kernel<TX, TY, V, 2, ONE>
                    : held <= MOST / 2 ? norm_held_kernel<TX, TY, V, MOST / 2, ONE> : norm_held_kernel<TX, TY, V, MOST, ONE>;
    const size_t lds = ((size_t)g.slots * row + 2 * (g.seg / h.D)) * sizeof(float);
    hipLaunchKernelGGL(kern, dim3((unsigned)((size_t)h.N * g.segs)), dim3(g.threads), lds, s, h, g, static_cast<const TX *>(f.x), f.ldx,
                       f.gamma, f.beta, f.eps, stats, static_cast<TY *>(f.y), f.ldy, f.past);
}
template <typename TX, typename TY, int V>
static void run_held(const NormShape &h, const HeldGrid &g, const NormForward &f, float2 *stats, hipStream_t s) {
    if constexpr (V == 8) {
        if (g.unit == 8) return launch_held<TX, TY, V, true>(h, g, f, stats, s);
    }
    launch_held<TX, TY, V, false>(h, g, f, stats, s);
}

// Statistics of images too large to be held: parts, and with `join` a second launch.
template <typename TX, int V>
static void launch_stats(const NormShape &h, const NormGrid &g, const NormForward &f, float2 *parts, float2 *stats, bool join, hipStream_t s) {
    const dim3 grid((unsigned)((size_t)h.N * g.chunks * g.slabs));
    const TX *x = static_cast<const TX *>(f.x);
    const int units = V == 8 && h.D % 8 == 0 ? h.D / 8 : h.D;      // of a group in one row of a block's sums
    const int lanes = group_lanes(g.TY * (units < kSlab ? units : kSlab), (h.C < kSlab ? h.C : kSlab) / h.D + 1, g.threads);
    if constexpr (V == 8) {
        const auto kern = h.D % 8 == 0 ? norm_stats_kernel<TX, V, true> : norm_stats_kernel<TX, V, false>;
        hipLaunchKernelGGL(kern, grid, dim3(g.threads), 0, s, h, g, x, f.ldx, parts, lanes);
    } else
        hipLaunchKernelGGL((norm_stats_kernel<TX, V, false>), grid, dim3(g.threads), 0, s, h, g, x, f.ldx, parts, lanes);
    if (join) hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(((size_t)h.N * h.groups * kJoinLanes + 255) / 256)), dim3(256), 0, s, h, g, parts, f.eps, stats);
}

// Statistics of the caller's that it did not ask for, and the parts of two-launch ones.
size_t norm_forward_bytes(const NormShape &h, int x_dtype, bool rows8, bool given) {
    HeldGrid held;
    const bool hold = x_dtype == GSPC_F32 ? plan_held(h, 4, held_most<float>(), 512, &held) : plan_held(h, 2, held_most<uint16_t>(), 512, &held);
    if (hold && !rows8) return 0;
    const size_t stats = given ? 0 : (size_t)h.N * h.groups * sizeof(float2);
    if (hold) return stats;
    const NormGrid g = norm_grid(h, kForwardBlocks, kForwardChunks);
    return stats + (size_t)h.N * g.chunks * norm_parts(h, g) * sizeof(float2);
}

// The call's tensors from image n on.
static NormForward from_image(const NormShape &h, NormForward f, size_t n) {
    const size_t row = n * h.P, pitch = rows8_pitch(h.C);
    const auto size = [](int dtype) { return dtype == GSPC_F32 ? 4u : 2u; };
    f.x = static_cast<const char *>(f.x) + row * f.ldx * size(f.x_dtype);
    f.y = static_cast<char *>(f.y) + row * (f.y_dtype == GSPC_I8 ? pitch : f.ldy * size(f.y_dtype));
    if (f.y_scale) f.y_scale += row;
    if (f.stats) f.stats += n * h.groups * 2;
    if (f.saved) f.saved += row * pitch, f.saved_scale += row;
    return f;
}

template <typename TX, int V>
static hipError_t forward(const NormShape &h, NormForward f, void *ws, hipStream_t s, const char **name) {
    const NormGrid g = norm_grid(h, kForwardBlocks, kForwardChunks);
    float2 *stats = f.stats ? reinterpret_cast<float2 *>(f.stats) : static_cast<float2 *>(ws);
    float2 *parts = static_cast<float2 *>(ws) + (f.stats ? 0 : (size_t)h.N * h.groups);
    f.past = f.y_dtype == GSPC_BF16 && (size_t)h.N * h.P * h.C * 2 >= kPastCaches &&
             (f.ldy == (size_t)h.C || whole_pieces(f.y, (size_t)h.C * 2, f.ldy * 2));
    HeldGrid held;
    const bool hold = plan_held(h, sizeof(TX), held_most<TX>(), 512, &held);
    if (f.y_dtype != GSPC_I8 && !f.saved && hold) {
        *name = "norm_held";
        if (f.y_dtype == GSPC_F32) run_held<TX, float, V>(h, held, f, reinterpret_cast<float2 *>(f.stats), s);
        else run_held<TX, uint16_t, V>(h, held, f, reinterpret_cast<float2 *>(f.stats), s);
        return hipGetLastError();
    }
    const bool rows8 = f.y_dtype == GSPC_I8 || f.saved, fold = !rows8 && h.groups <= kFoldGroups && h.groups * g.chunks <= kFoldParts &&
                      (long)h.N * g.chunks * g.slabs <= kFoldBlocks;
    *name = f.y_dtype == GSPC_I8 ? "norm_rows<i8>" : f.saved ? "norm_rows<saved>" : "norm_apply";
    if (hold) run_held<TX, void, V>(h, held, f, stats, s);
    const long step = norm_images(g);
    for (long n = 0; n < h.N; n += step) {          // (an image that is held has fewer companions than that)
        NormShape some = h;
        some.N = (int)(h.N - n < step ? h.N - n : step);
        const NormForward p = from_image(h, f, n);
        float2 *const st = stats + n * h.groups, *const pt = parts + n * g.chunks * norm_parts(h, g);
        if (!hold) launch_stats<TX, V>(some, g, p, pt, st, !fold, s);
        if (f.y_dtype == GSPC_I8) {
            if (f.saved) launch_rows<TX, int8_t, V, true>(some, p, st, s);
            else launch_rows<TX, int8_t, V, false>(some, p, st, s);
        } else if (f.saved) {
            if (f.y_dtype == GSPC_F32) launch_rows<TX, float, V, true>(some, p, st, s);
            else launch_rows<TX, uint16_t, V, true>(some, p, st, s);
        } else {
            const dim3 grid((unsigned)((size_t)some.N * g.chunks * g.slabs));
            const auto run = [&](auto kern, auto *y) {
                hipLaunchKernelGGL(kern, grid, dim3(g.threads), 0, s, some, g, static_cast<const TX *>(p.x), p.ldx, pt, p.eps,
                                   fold ? reinterpret_cast<float2 *>(p.stats) : st, p.gamma, p.beta, y, p.ldy, p.past);
            };
            if (f.y_dtype == GSPC_F32)
                run(fold ? norm_apply_kernel<TX, float, V, true> : norm_apply_kernel<TX, float, V, false>, static_cast<float *>(p.y));
            else
                run(fold ? norm_apply_kernel<TX, uint16_t, V, true> : norm_apply_kernel<TX, uint16_t, V, false>, static_cast<uint16_t *>(p.y));
        }
    }
    return hipGetLastError();
}

hipError_t launch_norm_forward(const NormShape &h, const NormForward &f, void *ws, hipStream_t s, const char **name) {
    if (f.x_dtype == GSPC_F32) return h.C >= 8 ? forward<float, 8>(h, f, ws, s, name) : forward<float, 1>(h, f, ws, s, name);
    return h.C >= 8 ? forward<uint16_t, 8>(h, f, ws, s, name) : forward<uint16_t, 1>(h, f, ws, s, name);
}

}  // namespace gspc
