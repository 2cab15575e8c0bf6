// Gradient of group norm with an activation, channels last.  With xh = (x - mean) rstd, z = gamma xh + beta, dz = dy act'(z):
//   dbeta = sum dz, dgamma = sum dz xh over images and pixels,
//   dx = rstd (gamma dz - (A + xh B) / m), A and B the sums of gamma dz and gamma dz xh over the m = P D values of the group.
#include "norm_common.h"

namespace gspc {

// With d = x - mean and a = gamma rstd: z = a d + beta; dgamma is rstd times the sum of dz d; dx = a dz + kappa d - lambda with
// kappa = - rstd^2 B / m, lambda = rstd A / m.  A vector's V channels are of E groups (V: any), V / E side by side in each.
template <int V, int E> struct GradAffine {
    float mean[E], rstd[E], a[V], beta[V];
};
template <int V, int E>
__device__ __forceinline__ void load_grad_affine(const NormShape &h, const float2 *__restrict__ stats, const float *__restrict__ gamma,
                                                 const float *__restrict__ beta, int n, int at, GradAffine<V, E> &f) {
    load_params<V>(gamma, at, 1.f, f.a);
    load_params<V>(beta, at, 0.f, f.beta);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float2 s = stats[(size_t)n * h.groups + group_of(h, at + e * (V / E))];
        f.mean[e] = s.x;
        f.rstd[e] = s.y;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) f.a[e] *= f.rstd[e * E / V];
}

// dy -> dz
template <int V, int E> __device__ __forceinline__ void to_dz(const GradAffine<V, E> &f, int act, const float (&d)[V], float (&dy)[V]) {
    if (act == kActRelu) {
#pragma unroll
        for (int e = 0; e < V; ++e) dy[e] *= slope<kActRelu>(fmaf(d[e], f.a[e], f.beta[e]));
    } else if (act == kActSilu) {
#pragma unroll
        for (int e = 0; e < V; ++e) dy[e] *= slope<kActSilu>(fmaf(d[e], f.a[e], f.beta[e]));
    }
}
// dz -> dx
template <int E> struct GradGroups {
    float kappa[E], lambda[E];
};
template <int V, int E> __device__ __forceinline__ void set_group(const GradAffine<V, E> &f, int e, float2 ab, GradGroups<E> &s) {
    s.kappa[e] = -f.rstd[e] * f.rstd[e] * ab.y;
    s.lambda[e] = f.rstd[e] * ab.x;
}
template <int V, int E>
__device__ __forceinline__ void to_dx(const GradAffine<V, E> &f, const GradGroups<E> &s, const float (&d)[V], float (&dz)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) dz[e] = fmaf(f.a[e], dz[e], fmaf(d[e], s.kappa[e * E / V], -s.lambda[e * E / V]));
}
// x -> d.  x of an 8-bit row is q * scale: with u = q + 128 (an unsigned byte converts to fp32 in one instruction)
// d = u scale - (128 scale + mean), off by 2^-24 of 128 scale + |mean|: 2^-17 of a step of the row's, and where the mean is far larger than the row as
// much as x - mean is rounded by.
template <typename TX, int V, int E>
__device__ __forceinline__ void widen_d(const GradAffine<V, E> &f, const Raw<TX, V> &r, float scale, float (&d)[V]) {
    if constexpr (sizeof(TX) == 1 && V == 8) {
        float shift[E];
#pragma unroll
        for (int e = 0; e < E; ++e) shift[e] = fmaf(-128.f, scale, -f.mean[e]);
        const u32x2 u = r.a ^ 0x80808080u;
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] = fmaf((float)(u[e / 4] >> (e % 4 * 8) & 0xffu), scale, shift[e * E / V]);
    } else {
        widen(r, d);
#pragma unroll
        for (int e = 0; e < V; ++e) d[e] = (sizeof(TX) == 1 ? d[e] * scale : d[e]) - f.mean[e * E / V];
    }
}

// A batch of rows of x and dy in flight.
template <typename TX, typename TG, int V> struct GradBatch {
    static constexpr int DEEP = 4;
    Raw<TX, V> x[DEEP];
    Raw<TG, V> g[DEEP];
    float scale[DEEP];
    __device__ __forceinline__ void load(const TX *px, size_t ldx, const TG *pg, size_t ldg, const float *ps, int r, int rows, int TY) {
#pragma unroll
        for (int k = 0; k < DEEP; ++k)
            if (r + k * TY < rows) {
                x[k] = fetch<V>(px + (size_t)(r + k * TY) * ldx);
                g[k] = fetch<V>(pg + (size_t)(r + k * TY) * ldg);
                if constexpr (sizeof(TX) == 1) scale[k] = ps[r + k * TY];
            }
    }
};

// Per channel and block: sums of dz and of dz xh over the block's rows, parts [n][chunk][2][C].  5 images of 29x37, 60 channels in fp32:
// 5.6 us, and 6.0 for dx, latency.  (64 images of 56x56, 256 channels in bf16: 97 us together, 515 MB with what is read
// twice, 5.3 TB/s; over batches of images whose x and dy fit the memory-side cache 135.)
template <typename TX, typename TG, int V, int E>
__global__ __launch_bounds__(kNormThreads) void norm_grad_sums_kernel(NormShape h, NormGrid g, const TG *__restrict__ dy, size_t lddy,
                                                                      const TX *__restrict__ x, size_t ldx,
                                                                      const float *__restrict__ x_scale, const float2 *__restrict__ stats,
                                                                      const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                      float *__restrict__ parts) {
    typedef GradBatch<TX, TG, V> Batch;
    __shared__ float s_dz[kNormThreads * V], s_dx[kNormThreads * V];
    const NormBlock b = norm_block(h, g, blockIdx.x);
    const int width = b.c1 - b.c0, rows = b.r1 - b.r0;
    if (b.active) {
        const size_t row0 = (size_t)b.n * h.P + b.r0;
        const TX *px = x + row0 * ldx + b.at;
        const TG *pg = dy + row0 * lddy + b.at;
        const float *ps = sizeof(TX) == 1 ? x_scale + row0 : nullptr;
        Batch now, next;
        now.load(px, ldx, pg, lddy, ps, b.ty, rows, g.TY);
        GradAffine<V, E> f;
        load_grad_affine<V, E>(h, stats, gamma, beta, b.n, b.at, f);
        float sz[V] = {}, sx[V] = {};
        for (int r = b.ty; r < rows; r += Batch::DEEP * g.TY) {
            next.load(px, ldx, pg, lddy, ps, r + Batch::DEEP * g.TY, rows, g.TY);
#pragma unroll
            for (int k = 0; k < Batch::DEEP; ++k)
                if (r + k * g.TY < rows) {
                    float d[V], dz[V];
                    widen_d<TX, V, E>(f, now.x[k], now.scale[k], d);
                    widen(now.g[k], dz);
                    to_dz<V, E>(f, h.act, d, dz);
#pragma unroll
                    for (int e = 0; e < V; ++e) sz[e] += dz[e], sx[e] = fmaf(dz[e], d[e], sx[e]);
                }
            now = next;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = b.at + e - b.c0;
            if (c >= 0) s_dz[b.ty * width + c] = sz[e], s_dx[b.ty * width + c] = sx[e] * f.rstd[e * E / V];
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += blockDim.x) {
        float sz = 0.f, sx = 0.f;
#pragma unroll 4
        for (int ty = 0; ty < g.TY; ++ty) sz += s_dz[ty * width + c], sx += s_dx[ty * width + c];
        float *p = parts + ((size_t)b.n * g.chunks + b.chunk) * 2 * h.C + b.c0 + c;
        p[0] = sz;
        p[h.C] = sx;
    }
}

// The blocks' parts joined: sums[n][2][C] of an image, and A / m, B / m of each group.  A wave has a group of an image: 2^log_lanes
// lanes its channels (in turn, where there are more), and as many times as these fit a wave the chunks between them.
__global__ __launch_bounds__(256) void norm_grad_join_kernel(NormShape h, int chunks, int log_lanes, const float *__restrict__ parts,
                                                             const float *__restrict__ gamma, float *__restrict__ sums,
                                                             float2 *__restrict__ ab) {
    const unsigned pair = (blockIdx.x * 256 + threadIdx.x) / kWave;
    if (pair >= (unsigned)h.N * h.groups) return;
    const int lanes = 1 << log_lanes, lane = threadIdx.x % kWave, own = lane & (lanes - 1), share = lane >> log_lanes, shares = kWave >> log_lanes;
    const int n = pair / h.groups, k = pair - n * h.groups;
    float a = 0.f, b = 0.f;
    for (int i = own; i - own < h.D; i += lanes) {
        const int c = k * h.D + min(i, h.D - 1);
        const float *p = parts + (size_t)n * chunks * 2 * h.C + c;
        float sz = 0.f, sx = 0.f;
#pragma unroll 8
        for (int j = share; j < chunks; j += shares) sz += p[(size_t)j * 2 * h.C], sx += p[((size_t)j * 2 + 1) * h.C];
        for (int d = lanes; d < kWave; d *= 2) sz += __shfl_xor(sz, d), sx += __shfl_xor(sx, d);
        if (i < h.D) {
            if (share == 0) {
                sums[(size_t)n * 2 * h.C + c] = sz;
                sums[((size_t)n * 2 + 1) * h.C + c] = sx;
            }
            const float w = gamma ? gamma[c] : 1.f;
            a = fmaf(w, sz, a);
            b = fmaf(w, sx, b);
        }
    }
    a = lanes_sum(a, lanes);
    b = lanes_sum(b, lanes);
    const float m = (float)h.P * (float)h.D;
    if (lane == 0) ab[pair] = make_float2(a / m, b / m);
}

// dgamma and dbeta: `blocks` blocks take 64 channels at a time, in turn, and their waves (MOST at most) the rows of sums ([rows][2][C]: of
// images, or of their parts).  In 64 bits: millions of images added up in 32 lose what is small against their sum (17 million of one
// pixel each: 5 % of dgamma).
template <int MOST>
__device__ __forceinline__ void sum_params(int C, unsigned block, unsigned blocks, int rows, const float *__restrict__ sums,
                                           float *__restrict__ dgamma, float *__restrict__ dbeta) {
    __shared__ double s_sum[2][MOST][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    for (unsigned c = block * kWave + lane; c - lane < (unsigned)C; c += blocks * kWave) {
        double sz = 0., sx = 0.;
        if (c < (unsigned)C) {
#pragma unroll 8
            for (int n = wave; n < rows; n += waves) sz += sums[(size_t)n * 2 * C + c], sx += sums[((size_t)n * 2 + 1) * C + c];
        }
        s_sum[0][wave][lane] = sz;
        s_sum[1][wave][lane] = sx;
        __syncthreads();
        for (int which = wave; which < 2; which += waves) {
            if (c >= (unsigned)C) continue;
            double sum = 0.;
            for (int w = 0; w < waves; ++w) sum += s_sum[which][w][lane];
            if (which == 0 && dbeta) dbeta[c] = (float)sum;
            if (which == 1 && dgamma) dgamma[c] = (float)sum;
        }
        __syncthreads();
    }
}

constexpr int kParamWaves = 16;
constexpr int kParamBlocks = 1 << 16;
static unsigned param_blocks(int C) { return C > kParamBlocks * kWave ? kParamBlocks : (C + kWave - 1) / kWave; }
__global__ __launch_bounds__(kParamWaves * kWave) void norm_grad_params_kernel(int C, int rows, const float *__restrict__ sums,
                                                                               float *__restrict__ dgamma, float *__restrict__ dbeta) {
    sum_params<kParamWaves>(C, blockIdx.x, gridDim.x, rows, sums, dgamma, dbeta);
}

// An image's groups whose A and B a block of norm_grad_apply_kernel takes from the parts itself, and the channels' sums behind them: in
// small launches, where a third one costs more.
constexpr int kFoldGroups = 64, kFoldSums = 4096, kFoldBlocks = 512;

// The first param_blocks blocks sum the parameters' gradients, the others write dx.  FOLD: sums are the blocks' parts, and a block
// takes its image's A and B from them (ab is not read).
template <typename TX, typename TG, int V, int E, bool FOLD>
__global__ __launch_bounds__(kNormThreads) void norm_grad_apply_kernel(NormShape h, NormGrid g, const TG *__restrict__ dy, size_t lddy,
                                                                       const TX *__restrict__ x, size_t ldx,
                                                                       const float *__restrict__ x_scale, const float2 *__restrict__ stats,
                                                                       const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                       const float2 *__restrict__ ab, TG *__restrict__ dx, size_t lddx,
                                                                       int past, int param_blocks, int param_rows,
                                                                       const float *__restrict__ sums, float *__restrict__ dgamma,
                                                                       float *__restrict__ dbeta) {
    typedef GradBatch<TX, TG, V> Batch;
    __shared__ float2 s_ab[FOLD ? kFoldGroups : 1];
    if ((int)blockIdx.x < param_blocks) return sum_params<kNormThreads / kWave>(h.C, blockIdx.x, param_blocks, param_rows, sums, dgamma, dbeta);
    const NormBlock b = norm_block(h, g, blockIdx.x - param_blocks);
    const size_t row0 = (size_t)b.n * h.P + b.r0;
    const TX *px = x + row0 * ldx + b.at;
    const TG *pg = dy + row0 * lddy + b.at;
    const float *ps = sizeof(TX) == 1 ? x_scale + row0 : nullptr;
    TG *pd = dx + row0 * lddx + b.at;
    const int rows = b.r1 - b.r0;
    Batch now, next;
    if (b.active) now.load(px, ldx, pg, lddy, ps, b.ty, rows, g.TY);
    if constexpr (FOLD) {
        const int lane = threadIdx.x % kWave;
        const float m = (float)h.P * (float)h.D, *part = sums + (size_t)b.n * g.chunks * 2 * h.C;
        for (int k = threadIdx.x / kWave; k < h.groups; k += g.threads / kWave) {
            float a = 0.f, bb = 0.f;
            for (int j = lane; j < g.chunks * h.D; j += kWave) {
                const int chunk = group_of(h, j), c = k * h.D + j - chunk * h.D;
                const float w = gamma ? gamma[c] : 1.f, *p = part + (size_t)chunk * 2 * h.C + c;
                a = fmaf(w, p[0], a);
                bb = fmaf(w, p[h.C], bb);
            }
            a = lanes_sum(a, kWave);
            bb = lanes_sum(bb, kWave);
            if (lane == 0) s_ab[k] = make_float2(a / m, bb / m);
        }
        __syncthreads();
    }
    if (!b.active) return;
    GradAffine<V, E> f;
    load_grad_affine<V, E>(h, stats, gamma, beta, b.n, b.at, f);
    GradGroups<E> s;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int k = group_of(h, b.at + e * (V / E));
        set_group(f, e, FOLD ? s_ab[k] : ab[(size_t)b.n * h.groups + k], s);
    }
    for (int r = b.ty; r < rows; r += Batch::DEEP * g.TY) {
        next.load(px, ldx, pg, lddy, ps, r + Batch::DEEP * g.TY, rows, g.TY);
#pragma unroll
        for (int k = 0; k < Batch::DEEP; ++k)
            if (r + k * g.TY < rows) {
                float d[V], dz[V];
                widen_d<TX, V, E>(f, now.x[k], now.scale[k], d);
                widen(now.g[k], dz);
                to_dz<V, E>(f, h.act, d, dz);
                to_dx<V, E>(f, s, d, dz);
                store(pd + (size_t)(r + k * g.TY) * lddx, dz, past);
            }
        now = next;
    }
}

// All but the sum over images in one launch, x and dy read once: a block holds its channels of an image, x as it came and dz in fp32,
// so that the activation's slope is computed once (256 images of 14x14, 512 channels in bf16 with SiLU: 36 us; with x and dy held as
// they came and it computed twice 44).  Four vectors a thread: with eight dz spills (69 us on 28x28, 128 channels from 8-bit rows; four in
// 1024 threads 41.6, 48 where the rows are not in the caches: loads, arithmetic and stores of the one block that a compute unit has room for follow
// one another; x and dy as they came, eight vectors in 512 threads and the slope computed twice, 38).
// sums: [n][2][C] for the parameters' gradients, or where there is one image these themselves.
template <typename TX, typename TG, int V, int E, int HELD>
__global__ __launch_bounds__(1024) void norm_grad_held_kernel(NormShape h, HeldGrid g, const TG *__restrict__ dy, size_t lddy,
                                                             const TX *__restrict__ x, size_t ldx, const float *__restrict__ x_scale,
                                                             const float2 *__restrict__ stats, const float *__restrict__ gamma,
                                                             const float *__restrict__ beta, float *__restrict__ sum_dz,
                                                             float *__restrict__ sum_dx, size_t ld_sums, TG *__restrict__ dx, size_t lddx,
                                                             int past) {
    extern __shared__ float part[];                 // [2][slots][row], then [2][seg] of the channels, [groups][2] of the groups
    const unsigned block = held_block(g, blockIdx.x), n = fast_div_any(block, g.segs, g.m_segs);
    const int c0 = (block - n * g.segs) * g.seg, row = g.seg + 1;      // (an odd pitch: sums over slots read one column)
    const int lane = threadIdx.x & ((1 << g.log_width) - 1), slot = threadIdx.x >> g.log_width;
    const int nv = vectors_of<V>(g.seg);
    const bool on = lane < nv;
    const int at = vector_start<V>(min(lane, nv - 1), g.seg);
    float *channel = part + 2 * g.slots * row;
    float2 *group_ab = reinterpret_cast<float2 *>(channel + 2 * g.seg);

    // No branch on a lane's own account from here to the sums: lanes past the last vector repeat it and are left out of the sums,
    // slots past the last token repeat that with dy = 0.
    const size_t token0 = (size_t)n * h.P;
    Raw<TX, V> rx[HELD];
    Raw<TG, V> rg[HELD];
    float scale[HELD];
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        if (k * g.slots < h.P) {
            const int p = slot + k * g.slots;
            const size_t token = token0 + min(p, h.P - 1);
            rx[k] = fetch<V>(x + token * ldx + c0 + at);
            rg[k] = fetch<V>(dy + token * lddy + c0 + at);
            if constexpr (sizeof(TX) == 1) scale[k] = x_scale[token];
        }
    GradAffine<V, E> f;
    load_grad_affine<V, E>(h, stats, gamma, beta, n, c0 + at, f);
    // Eight groups a vector and four vectors of fp32: d takes the place of x at once, and 1 / deviation is fetched where sums are complete, so that
    // neither has registers during the passes below (kept as for the others, they spilled).
    constexpr bool CENTRED = E == 8 && HELD == 4 && sizeof(TX) == 4;
    if constexpr (CENTRED) {
#pragma unroll
        for (int k = 0; k < HELD; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) rx[k].a[e] -= f.mean[e], rx[k].b[e] -= f.mean[4 + e];
    }
    const auto to_d = [&](int k, float (&d)[V]) {
        if constexpr (CENTRED) widen(rx[k], d);
        else widen_d<TX, V, E>(f, rx[k], scale[k], d);
    };
    float dz[HELD][V];
    {
        float sz[V] = {}, sx[V] = {};
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (k * g.slots < h.P) {
                float d[V];
                hold(rx[k]);
                hold(rg[k]);
                if ((k + 1) * g.slots > h.P) keep_if(rg[k], slot + k * g.slots < h.P);
                to_d(k, d);
                widen(rg[k], dz[k]);
                to_dz<V, E>(f, h.act, d, dz[k]);
#pragma unroll
                for (int e = 0; e < V; ++e) sz[e] += dz[k][e], sx[e] = fmaf(dz[k][e], d[e], sx[e]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (on) {
#pragma unroll
            for (int e = 0; e < V; ++e) part[slot * row + at + e] = sz[e], part[(g.slots + slot) * row + at + e] = CENTRED ? sx[e] : sx[e] * f.rstd[e * E / V];
        }
    }
    __syncthreads();
    // sums over the slots: `lanes` lanes for each of the 2 seg columns
    const int lanes = 1 << g.log_lanes;
    for (int i = threadIdx.x >> g.log_lanes; i < 2 * g.seg; i += g.threads >> g.log_lanes) {
        const int which = i >= g.seg, c = i - which * g.seg;
        float sum = 0.f;
        for (int j = threadIdx.x & (lanes - 1); j < g.slots; j += lanes) sum += part[(which * g.slots + j) * row + c];
        sum = lanes_sum(sum, lanes);
        if ((threadIdx.x & (lanes - 1)) == 0) {
            if (CENTRED && which) sum *= stats[(size_t)n * h.groups + group_of(h, c0 + c)].y;
            channel[i] = sum;
            float *to = which ? sum_dx : sum_dz;
            if (to) to[n * ld_sums + c0 + c] = sum;
        }
    }
    __syncthreads();
    const float m = (float)h.P * (float)h.D;
    const int groups = g.seg / h.D, wave_lane = threadIdx.x % kWave;
    for (int k = threadIdx.x / kWave; k < groups; k += g.threads / kWave) {
        float a = 0.f, b = 0.f;
        for (int j = wave_lane; j < h.D; j += kWave) {
            const float w = gamma ? gamma[c0 + k * h.D + j] : 1.f;
            a = fmaf(w, channel[k * h.D + j], a);
            b = fmaf(w, channel[g.seg + k * h.D + j], b);
        }
        a = lanes_sum(a, kWave);
        b = lanes_sum(b, kWave);
        if (wave_lane == 0) {
            group_ab[k] = make_float2(a / m, b / m);
            if constexpr (CENTRED) {
                const float r = stats[(size_t)n * h.groups + group_of(h, c0) + k].y;
                group_ab[k] = make_float2(r * (a / m), -r * r * (b / m));
            }
        }
    }
    __syncthreads();
    GradGroups<E> s;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float2 ab = group_ab[group_of(h, at + e * (V / E))];
        if constexpr (CENTRED) s.lambda[e] = ab.x, s.kappa[e] = ab.y;
        else set_group(f, e, ab, s);
    }
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
        if (k * g.slots < h.P) {
            const int p = slot + k * g.slots;
            float d[V];
            hold(rx[k]);
            to_d(k, d);
            to_dx<V, E>(f, s, d, dz[k]);
            if (on && p < h.P) store(dx + (token0 + p) * lddx + c0 + at, dz[k], past);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
constexpr int kBackwardBlocks = 2048, kBackwardChunks = 256;

// Up to 512 threads where four vectors each hold the channels; 1024 leave one block a compute unit and are taken where 512 do not.
static bool plan_grad_held(const NormShape &h, int size, HeldGrid *g) { return plan_held(h, size, 4, 512, g) || plan_held(h, size, 4, 1024, g); }

size_t norm_backward_bytes(const NormShape &h, int dy_dtype) {
    HeldGrid held;
    const bool hold = plan_grad_held(h, dy_dtype == GSPC_F32 ? 4 : 2, &held);
    if (hold && h.N == 1) return 0;
    const size_t sums = (size_t)h.N * 2 * h.C * sizeof(float);
    if (hold) return sums;
    return sums + ((size_t)h.N * norm_grid(h, kBackwardBlocks, kBackwardChunks).chunks * 2 * h.C + (size_t)h.N * h.groups * 2) * sizeof(float);
}

template <typename TX, typename TG, int V, int E>
static hipError_t launch_grad_held(const NormShape &h, HeldGrid g, const NormBackward &b, float *sums, hipStream_t s) {
    const int held = (h.P - 1) / g.slots + 1;
    const auto kern = held <= 1 ? norm_grad_held_kernel<TX, TG, V, E, 1> : held <= 2 ? norm_grad_held_kernel<TX, TG, V, E, 2>
                                                                          : norm_grad_held_kernel<TX, TG, V, E, 4>;
    g.log_lanes = 0;
    while ((1 << g.log_lanes) < g.slots && g.log_lanes < 6 && (4 * g.seg << g.log_lanes) <= g.threads) ++g.log_lanes;
    const size_t lds = (2 * (size_t)g.slots * (g.seg + 1) + 2 * g.seg + 2 * (g.seg / h.D) + 1) * sizeof(float);
    const bool one = h.N == 1;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)((size_t)h.N * g.segs)), dim3(g.threads), lds, s, h, g, static_cast<const TG *>(b.dy), b.lddy,
                       static_cast<const TX *>(b.x), b.ldx, b.x_scale, reinterpret_cast<const float2 *>(b.stats), b.gamma, b.beta,
                       one ? b.dbeta : sums, one ? b.dgamma : sums + h.C, (size_t)2 * h.C, static_cast<TG *>(b.dx), b.lddx, b.past);
    return hipSuccess;
}

// The call's tensors from image n on.
template <typename TX, typename TG> static NormBackward from_image(const NormShape &h, NormBackward b, size_t n) {
    const size_t row = n * h.P;
    b.dy = static_cast<const TG *>(b.dy) + row * b.lddy;
    b.x = static_cast<const TX *>(b.x) + row * b.ldx;
    if (b.x_scale) b.x_scale += row;
    b.stats += n * h.groups * 2;
    b.dx = static_cast<TG *>(b.dx) + row * b.lddx;
    return b;
}

template <typename TX, typename TG, int V, int E>
static void launch_grad(const NormShape &h, const NormGrid &g, const NormBackward &b, float *parts, float *sums, float2 *ab, hipStream_t s) {
    const unsigned params = b.dgamma || b.dbeta ? param_blocks(h.C) : 0;
    const bool fold = h.groups <= kFoldGroups && (long)g.chunks * 2 * h.C <= kFoldSums && (long)h.N * g.chunks * g.slabs <= kFoldBlocks;
    // f(images, their shape, tensors, blocks) for the images of each launch
    const auto launches = [&](const auto &f) {
        const long step = norm_images(g) - kParamBlocks / (g.chunks * g.slabs) - 1;
        for (long n = 0; n < h.N; n += step) {
            NormShape some = h;
            some.N = (int)(h.N - n < step ? h.N - n : step);
            f((size_t)n, some, from_image<TX, TG>(h, b, n), (unsigned)((size_t)some.N * g.chunks * g.slabs));
        }
    };
    launches([&](size_t n, const NormShape &some, const NormBackward &p, unsigned blocks) {
        hipLaunchKernelGGL((norm_grad_sums_kernel<TX, TG, V, E>), dim3(blocks), dim3(g.threads), 0, s, some, g, static_cast<const TG *>(p.dy), p.lddy,
                           static_cast<const TX *>(p.x), p.ldx, p.x_scale, reinterpret_cast<const float2 *>(p.stats), p.gamma, p.beta,
                           parts + n * g.chunks * 2 * h.C);
    });
    const auto apply = [&](auto kern, int rows, const float *from) {
        launches([&](size_t n, const NormShape &some, const NormBackward &p, unsigned blocks) {
            const unsigned own = n == 0 ? params : 0;
            hipLaunchKernelGGL(kern, dim3(blocks + own), dim3(g.threads), 0, s, some, g, static_cast<const TG *>(p.dy), p.lddy,
                               static_cast<const TX *>(p.x), p.ldx, p.x_scale, reinterpret_cast<const float2 *>(p.stats), p.gamma, p.beta,
                               ab + n * h.groups, static_cast<TG *>(p.dx), p.lddx, p.past, (int)own, rows, from, p.dgamma, p.dbeta);
        });
    };
    if (fold) return apply(norm_grad_apply_kernel<TX, TG, V, E, true>, h.N * g.chunks, parts);
    int log_lanes = 0;
    while ((1 << log_lanes) < h.D && log_lanes < 6) ++log_lanes;
    hipLaunchKernelGGL(norm_grad_join_kernel, dim3((unsigned)(((size_t)h.N * h.groups * kWave + 255) / 256)), dim3(256), 0, s, h, g.chunks,
                       log_lanes, parts, b.gamma, sums, ab);
    apply(norm_grad_apply_kernel<TX, TG, V, E, false>, h.N, sums);
}

template <typename TX, typename TG, int V>
static hipError_t backward(const NormShape &h, NormBackward b, void *ws, hipStream_t s, const char **name) {
    const dim3 params_grid(param_blocks(h.C));
    const bool params = b.dgamma || b.dbeta;
    if ((long)h.N * h.P == 0) {                     // no tokens: zeros
        *name = "norm_grad_params";
        if (params)
            hipLaunchKernelGGL(norm_grad_params_kernel, params_grid, dim3(kParamWaves * kWave), 0, s, h.C, 0, (const float *)nullptr, b.dgamma, b.dbeta);
        return hipGetLastError();
    }
    const NormGrid g = norm_grid(h, kBackwardBlocks, kBackwardChunks);
    float *sums = static_cast<float *>(ws);
    float2 *ab = reinterpret_cast<float2 *>(sums + (size_t)h.N * 2 * h.C);
    float *parts = reinterpret_cast<float *>(ab + (size_t)h.N * h.groups);
    // (and rows of 512 bytes and more, however they lie: 64 images of 56x56, 256 of 258 channels 104.7 us through the caches, 98.9 past them; 100 of
    // 102 level)
    b.past = sizeof(TG) == 2 && (size_t)h.N * h.P * h.C * 2 >= kPastCaches &&
             (h.C >= 256 || b.lddx == (size_t)h.C || whole_pieces(b.dx, (size_t)h.C * 2, b.lddx * 2));
    HeldGrid held;
    const bool hold = plan_grad_held(h, sizeof(TG), &held);
    *name = hold ? "norm_grad_held" : "norm_grad_apply";
    const auto run = [&](auto e) {
        constexpr int E = decltype(e)::value;
        if (hold) return launch_grad_held<TX, TG, V, E>(h, held, b, sums, s);
        launch_grad<TX, TG, V, E>(h, g, b, parts, sums, ab, s);
        return hipSuccess;
    };
    hipError_t e;
    if (V == 8 && h.D % 8 == 0) e = run(std::integral_constant<int, 1>{});
    else if (V == 8 && h.D % 4 == 0) e = run(std::integral_constant<int, V == 8 ? 2 : 1>{});
    else e = run(std::integral_constant<int, V>{});
    if (e != hipSuccess) return e;
    if (params && hold && h.N > 1)
        hipLaunchKernelGGL(norm_grad_params_kernel, params_grid, dim3(kParamWaves * kWave), 0, s, h.C, h.N, sums, b.dgamma, b.dbeta);
    return hipGetLastError();
}

template <typename TG, int V>
static hipError_t backward_of(const NormShape &h, const NormBackward &b, void *ws, hipStream_t s, const char **name) {
    return b.x_dtype == GSPC_F32 ? backward<float, TG, V>(h, b, ws, s, name)
         : b.x_dtype == GSPC_BF16 ? backward<uint16_t, TG, V>(h, b, ws, s, name) : backward<int8_t, TG, V>(h, b, ws, s, name);
}

hipError_t launch_norm_backward(const NormShape &h, const NormBackward &b, void *ws, hipStream_t s, const char **name) {
    if (b.dy_dtype == GSPC_F32)
        return h.C >= 8 ? backward_of<float, 8>(h, b, ws, s, name) : backward_of<float, 1>(h, b, ws, s, name);
    return h.C >= 8 ? backward_of<uint16_t, 8>(h, b, ws, s, name) : backward_of<uint16_t, 1>(h, b, ws, s, name);
}

}  // namespace gspc
