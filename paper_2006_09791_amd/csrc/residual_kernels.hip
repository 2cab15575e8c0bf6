// x' = scale x + gate drop(post(h)), z = act(pre(x')): a block's output normalised, gated and added to the residual stream, and the stream normalised
// for the next block, in one pass.
#include "residual_common.h"

namespace gspc {

// A team keeps its parameters and walks down consecutive tokens; the next token's values are on their way while this one's are worked on.  Bound by
// memory where there are many tokens: x and h in, x' and z out.
template <typename TX, typename TH>
__global__ __launch_bounds__(kMaxTeam) void residual_norm_kernel(Residual a, ResidualForward f, int team, unsigned each, unsigned m_gate) {
    __shared__ float2 s_place[2][kMaxTeam / kWave];
    TeamSums sums{s_place, 0};
    const int lane = threadIdx.x & (team - 1), seg = lane / kWave, at = lane * 8, n = max(0, min(8, a.cols - at));
    const unsigned first = ((size_t)blockIdx.x * (blockDim.x / team) + threadIdx.x / team) * each;
    const unsigned last = min(first + each, a.rows);            // (fewer than 2^32)
    const TX *x = static_cast<const TX *>(f.x) + at;
    const TH *h = static_cast<const TH *>(f.h) + at;
    float g1[8], b1[8], g2[8], b2[8], gate[8];
    some_params(a.post_gamma, at, n, 1.f, g1);
    some_params(a.post_beta, at, n, 0.f, b1);
    some_params(a.pre_gamma, at, n, 1.f, g2);
    some_params(a.pre_beta, at, n, 0.f, b2);
    unsigned gate_row = ~0u;
    if (!a.gate) some_params(nullptr, 0, 0, 1.f, gate);
    const uint64_t call = a.drop.offset + (a.drop.step ? *a.drop.step : 0);
    Raw<TX, 8> rx{};
    Raw<TH, 8> rh{};
    if (first < last) {
        rx = fetch_some(x + first * f.ldx, n);
        if (f.h) rh = fetch_some(h + first * f.ldh, n);
    }
    for (unsigned k = 0; k < each; ++k) {                       // as often in every team: there are barriers
        const unsigned row = first + k;
        const bool there = row < last;
        float v[8];
        float2 st1 = make_float2(0.f, 1.f), st2 = make_float2(0.f, 1.f);
        widen(rx, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        if (f.h) {
            float u[8];
            widen(rh, u);
            if (a.post != kNormNone) {
                st1 = team_stats(u, n, a.cols, a.post, a.eps, team, seg, sums);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = fmaf((u[e] - st1.x) * st1.y, g1[e], b1[e]);
            }
            if (a.gate) {
                const unsigned now = fast_div_any(min(row, a.rows - 1), a.gate_rows, m_gate);
                if (now != gate_row) some_params(a.gate + (size_t)now * a.cols, at, n, 1.f, gate), gate_row = now;
            }
            if (a.drop.limit) {
                float m[8];
                dropout_factors(a.drop, call, row, lane, m);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = m[e] != 0.f ? u[e] * m[e] : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(gate[e], u[e], v[e]);
        }
        if (k + 1 < each && row + 1 < last) {
            rx = fetch_some(x + (row + 1) * f.ldx, n);
            if (f.h) rh = fetch_some(h + (row + 1) * f.ldh, n);
        }
        if (there && f.xo) store_some(static_cast<TX *>(f.xo) + row * f.ldxo + at, v, n, f.past);
        if (a.pre != kNormNone) {
            st2 = team_stats(v, n, a.cols, a.pre, a.eps, team, seg, sums);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - st2.x) * st2.y, g2[e], b2[e]);
            activate_all(a.act, v);
            if (f.z_dtype == GSPC_F8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = e < n ? v[e] : 0.f;
                const unsigned code = block_code(lanes_umax(top_of(v), 16));
                const int pitch = f8_pitch(a.cols), s_pitch = f8_scale_pitch(a.cols);
                if (there && at < pitch) {
                    *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(f.z) + (size_t)row * pitch + at) = f8_codes(v, block_up(code));
                    uint8_t *s = f.z_scale + (size_t)row * s_pitch + lane / 16;
                    if (lane % 16 == 0) *s = (uint8_t)code;
                    else if (lane / 16 == pitch / kBlock8 - 1 && lane / 16 + lane % 16 < s_pitch) s[lane % 16] = 0;
                }
            } else if (there && f.z) {
                if (f.z_dtype == GSPC_F32) store_some(static_cast<float *>(f.z) + row * f.ldz + at, v, n);
                else store_some(static_cast<uint16_t *>(f.z) + row * f.ldz + at, v, n, f.past);
            }
        }
        if (there && f.stats && lane == 0) *reinterpret_cast<float4 *>(f.stats + (size_t)row * 4) = make_float4(st1.x, st1.y, st2.x, st2.y);
    }
}

hipError_t launch_residual_norm(const Residual &a, ResidualForward f, hipStream_t s) {
    const TeamGrid g = team_grid(a.cols, 16);
    // tokens of a team: as few as keep 2048 blocks
    const size_t teams = (size_t)2048 * g.teams;
    const unsigned each = (unsigned)((a.rows + teams - 1) / teams), of_block = each * g.teams;
    const unsigned blocks = (a.rows - 1) / of_block + 1;
    f.past = (size_t)a.rows * a.cols * 2 >= kPastCaches && (!f.xo || f.x_dtype == GSPC_F32 || whole_pieces(f.xo, a.cols * 2, f.ldxo * 2)) &&
             (f.z_dtype != GSPC_BF16 || whole_pieces(f.z, a.cols * 2, f.ldz * 2));
    const auto run = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(g.threads), 0, s, a, f, g.team, each, div_magic(a.gate_rows));
        return hipGetLastError();
    };
    if (f.x_dtype == GSPC_F32) return f.h_dtype == GSPC_F32 ? run(residual_norm_kernel<float, float>) : run(residual_norm_kernel<float, uint16_t>);
    return f.h_dtype == GSPC_F32 ? run(residual_norm_kernel<uint16_t, float>) : run(residual_norm_kernel<uint16_t, uint16_t>);
}

}  // namespace gspc
