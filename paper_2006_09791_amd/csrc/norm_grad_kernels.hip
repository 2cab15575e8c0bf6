// Gradient of group norm with an activation, channels last.  With xh = (x - mean) rstd, z = gamma xh + beta, dz = dy act'(z):
//   dbeta = sum dz, dgamma = sum dz xh over images and pixels,
//   dx = rstd (gamma dz - (A + xh B) / m), A and B the sums of gamma dz and gamma dz xh over the m = P D values of the group.
#include "norm_common.h"

namespace gspc {

template <int V> struct GradAffine {
    float mean[V], rstd[V], gamma[V], beta[V];
};
template <int V>
__device__ __forceinline__ void load_grad_affine(const NormShape &h, const float2 *__restrict__ stats, const float *__restrict__ gamma,
                                                 const float *__restrict__ beta, int n, int at, GradAffine<V> &f) {
    const float2 *st = stats + (size_t)n * h.groups;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float2 s = st[(at + e) / h.D];
        f.mean[e] = s.x;
        f.rstd[e] = s.y;
        f.gamma[e] = gamma ? gamma[at + e] : 1.f;
        f.beta[e] = beta ? beta[at + e] : 0.f;
    }
}

// x -> xh, dy -> dz
template <int V> __device__ __forceinline__ void to_grad(const GradAffine<V> &f, int act, float scale, float (&x)[V], float (&dy)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = (x[e] * scale - f.mean[e]) * f.rstd[e];
    if (act == kActRelu) {
#pragma unroll
        for (int e = 0; e < V; ++e) dy[e] *= slope<kActRelu>(fmaf(x[e], f.gamma[e], f.beta[e]));
    } else if (act == kActSilu) {
#pragma unroll
        for (int e = 0; e < V; ++e) dy[e] *= slope<kActSilu>(fmaf(x[e], f.gamma[e], f.beta[e]));
    }
}

// Per channel and block: sums of dz and of dz xh over the block's rows, parts [n][chunk][2][C].
template <typename TX, typename TG, int V>
__global__ __launch_bounds__(kNormThreads) void norm_grad_sums_kernel(NormShape h, NormGrid g, const TG *__restrict__ dy, size_t lddy,
                                                                      const TX *__restrict__ x, size_t ldx,
                                                                      const float *__restrict__ x_scale, const float2 *__restrict__ stats,
                                                                      const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                      float *__restrict__ parts) {
    __shared__ float s_dz[kNormThreads * V], s_dx[kNormThreads * V];
    const NormBlock b = norm_block(h, g, blockIdx.x);
    const int width = b.c1 - b.c0, rows = b.r1 - b.r0;
    if (b.active) {
        GradAffine<V> f;
        load_grad_affine<V>(h, stats, gamma, beta, b.n, b.at, f);
        const size_t row0 = (size_t)b.n * h.P + b.r0;
        const TX *px = x + row0 * ldx + b.at;
        const TG *pg = dy + row0 * lddy + b.at;
        float sz[V] = {}, sx[V] = {};
        for (int r = b.ty; r < rows; r += 2 * g.TY) {
            Raw<TX, V> rx[2];
            Raw<TG, V> rg[2];
            float scale[2] = {1.f, 1.f};
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (r + k * g.TY < rows) {
                    rx[k] = fetch<V>(px + (size_t)(r + k * g.TY) * ldx);
                    rg[k] = fetch<V>(pg + (size_t)(r + k * g.TY) * lddy);
                    if (sizeof(TX) == 1) scale[k] = x_scale[row0 + r + k * g.TY];
                }
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (r + k * g.TY < rows) {
                    float vx[V], vg[V];
                    widen(rx[k], vx);
                    widen(rg[k], vg);
                    to_grad<V>(f, h.act, scale[k], vx, vg);
#pragma unroll
                    for (int e = 0; e < V; ++e) sz[e] += vg[e], sx[e] = fmaf(vg[e], vx[e], sx[e]);
                }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = b.at + e - b.c0;
            if (c >= 0) s_dz[b.ty * width + c] = sz[e], s_dx[b.ty * width + c] = sx[e];
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += blockDim.x) {
        float sz = 0.f, sx = 0.f;
        for (int ty = 0; ty < g.TY; ++ty) sz += s_dz[ty * width + c], sx += s_dx[ty * width + c];
        float *p = parts + ((size_t)b.n * g.chunks + b.chunk) * 2 * h.C + b.c0 + c;
        p[0] = sz;
        p[h.C] = sx;
    }
}

// The blocks' parts joined: sums[n][2][C] of an image, and A / m, B / m of each group.  `lanes` lanes for a group of an image.
__global__ __launch_bounds__(256) void norm_grad_join_kernel(NormShape h, int chunks, int lanes, const float *__restrict__ parts,
                                                             const float *__restrict__ gamma, float *__restrict__ sums,
                                                             float2 *__restrict__ ab) {
    const unsigned pair = (blockIdx.x * 256 + threadIdx.x) / lanes, lane = threadIdx.x & (lanes - 1);
    if (pair >= (unsigned)h.N * h.groups) return;
    const int n = pair / h.groups, k = pair - n * h.groups;
    float a = 0.f, b = 0.f;
    for (int i = lane; i < h.D; i += lanes) {
        const int c = k * h.D + i;
        const float *p = parts + (size_t)n * chunks * 2 * h.C + c;
        float sz = 0.f, sx = 0.f;
#pragma unroll 4
        for (int j = 0; j < chunks; ++j) sz += p[(size_t)j * 2 * h.C], sx += p[((size_t)j * 2 + 1) * h.C];
        sums[(size_t)n * 2 * h.C + c] = sz;
        sums[((size_t)n * 2 + 1) * h.C + c] = sx;
        const float w = gamma ? gamma[c] : 1.f;
        a = fmaf(w, sz, a);
        b = fmaf(w, sx, b);
    }
    a = lanes_sum(a, lanes);
    b = lanes_sum(b, lanes);
    const float m = (float)h.P * (float)h.D;
    if (lane == 0) ab[pair] = make_float2(a / m, b / m);
}

// dgamma and dbeta: 64 channels a block, its waves take the images in turn.
__global__ __launch_bounds__(256) void norm_grad_params_kernel(NormShape h, const float *__restrict__ sums, float *__restrict__ dgamma,
                                                               float *__restrict__ dbeta) {
    __shared__ float s_sum[2][4][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    float sz = 0.f, sx = 0.f;
    if (c < h.C) {
#pragma unroll 8
        for (int n = wave; n < h.N; n += 4) sz += sums[(size_t)n * 2 * h.C + c], sx += sums[((size_t)n * 2 + 1) * h.C + c];
    }
    s_sum[0][wave][lane] = sz;
    s_sum[1][wave][lane] = sx;
    __syncthreads();
    if (wave == 0 && c < h.C) {
        if (dbeta) dbeta[c] = (s_sum[0][0][lane] + s_sum[0][1][lane]) + (s_sum[0][2][lane] + s_sum[0][3][lane]);
        if (dgamma) dgamma[c] = (s_sum[1][0][lane] + s_sum[1][1][lane]) + (s_sum[1][2][lane] + s_sum[1][3][lane]);
    }
}

template <typename TX, typename TG, int V>
__global__ __launch_bounds__(kNormThreads) void norm_grad_apply_kernel(NormShape h, NormGrid g, const TG *__restrict__ dy, size_t lddy,
                                                                       const TX *__restrict__ x, size_t ldx,
                                                                       const float *__restrict__ x_scale, const float2 *__restrict__ stats,
                                                                       const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                       const float2 *__restrict__ ab, TG *__restrict__ dx, size_t lddx) {
    const NormBlock b = norm_block(h, g, blockIdx.x);
    if (!b.active) return;
    GradAffine<V> f;
    load_grad_affine<V>(h, stats, gamma, beta, b.n, b.at, f);
    float2 s[V];
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = ab[(size_t)b.n * h.groups + (b.at + e) / h.D];
    const size_t row0 = (size_t)b.n * h.P + b.r0;
    const TX *px = x + row0 * ldx + b.at;
    const TG *pg = dy + row0 * lddy + b.at;
    TG *pd = dx + row0 * lddx + b.at;
    const int rows = b.r1 - b.r0;
    for (int r = b.ty; r < rows; r += 2 * g.TY) {
        Raw<TX, V> rx[2];
        Raw<TG, V> rg[2];
        float scale[2] = {1.f, 1.f};
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (r + k * g.TY < rows) {
                rx[k] = fetch<V>(px + (size_t)(r + k * g.TY) * ldx);
                rg[k] = fetch<V>(pg + (size_t)(r + k * g.TY) * lddy);
                if (sizeof(TX) == 1) scale[k] = x_scale[row0 + r + k * g.TY];
            }
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (r + k * g.TY < rows) {
                float vx[V], vg[V];
                widen(rx[k], vx);
                widen(rg[k], vg);
                to_grad<V>(f, h.act, scale[k], vx, vg);
                // (the product gamma dz is rounded on its own, as in A: of a group of one value nothing is left)
#pragma unroll
                for (int e = 0; e < V; ++e) vg[e] = f.rstd[e] * (__fmul_rn(f.gamma[e], vg[e]) - fmaf(vx[e], s[e].y, s[e].x));
                store(pd + (size_t)(r + k * g.TY) * lddx, vg);
            }
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------
size_t norm_backward_bytes(const NormShape &h) {
    const NormGrid g = norm_grid(h, 2048);
    return ((size_t)h.N * g.chunks * 2 * h.C + (size_t)h.N * 2 * h.C + (size_t)h.N * h.groups * 2) * sizeof(float);
}

template <typename TX, typename TG, int V>
static hipError_t backward(const NormShape &h, const NormBackward &b, void *ws, hipStream_t s, const char **name) {
    const unsigned param_blocks = (h.C + kWave - 1) / kWave;
    if ((long)h.N * h.P == 0) {
        if (b.dgamma || b.dbeta)
            hipLaunchKernelGGL(norm_grad_params_kernel, dim3(param_blocks), dim3(256), 0, s, NormShape{0, 0, h.C, h.groups, h.D, 0},
                               (const float *)nullptr, b.dgamma, b.dbeta);
        *name = "norm_grad_params";
        return hipGetLastError();
    }
    const NormGrid g = norm_grid(h, 2048);
    float *parts = static_cast<float *>(ws), *sums = parts + (size_t)h.N * g.chunks * 2 * h.C;
    float2 *ab = reinterpret_cast<float2 *>(sums + (size_t)h.N * 2 * h.C);
    const TX *x = static_cast<const TX *>(b.x);
    const TG *dy = static_cast<const TG *>(b.dy);
    const float2 *stats = reinterpret_cast<const float2 *>(b.stats);
    const dim3 grid((unsigned)((size_t)h.N * g.chunks * g.slabs));
    const int lanes = group_lanes(h.D);
    hipLaunchKernelGGL((norm_grad_sums_kernel<TX, TG, V>), grid, dim3(g.threads), 0, s, h, g, dy, b.lddy, x, b.ldx, b.x_scale, stats,
                       b.gamma, b.beta, parts);
    hipLaunchKernelGGL(norm_grad_join_kernel, dim3((unsigned)(((size_t)h.N * h.groups * lanes + 255) / 256)), dim3(256), 0, s, h, g.chunks,
                       lanes, parts, b.gamma, sums, ab);
    if (b.dgamma || b.dbeta)
        hipLaunchKernelGGL(norm_grad_params_kernel, dim3(param_blocks), dim3(256), 0, s, h, sums, b.dgamma, b.dbeta);
    hipLaunchKernelGGL((norm_grad_apply_kernel<TX, TG, V>), grid, dim3(g.threads), 0, s, h, g, dy, b.lddy, x, b.ldx, b.x_scale, stats,
                       b.gamma, b.beta, ab, static_cast<TG *>(b.dx), b.lddx);
    *name = "norm_grad_apply";
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
