// x' = scale x + gate drop(post(h)), z = act(pre(x')): a block's output normalised, gated and added to the residual stream, and the stream normalised
// for the next block, in one pass.
#include "residual_common.h"

namespace gspc {

// A team keeps its parameters and walks down consecutive tokens; the next token's values are on their way while this one's are worked on.  x and h in, x'
// and z out: bound by memory without an h (50176 x 512 in bf16, 103 MB: 18 us, 5.7 TB/s), by vector instructions nearly as much with two
// norms, dropout and SiLU (206 MB: 50.2 us, 4.1 TB/s; 357 instructions for a wave's 512 values, three quarters of the time).  H: there is an h.
template <typename TX, typename TH, bool H, Rows ROWS, bool WAVES>
__global__ __launch_bounds__(WAVES ? kMaxTeam : kTeamThreads) void residual_norm_kernel(Residual a, ResidualForward f, int team, unsigned each, unsigned m_gate) {
    __shared__ float2 s_place[2][kMaxTeam / kWave];
    TeamSums sums{s_place, 0};
    const int lane = threadIdx.x & (team - 1), seg = lane / kWave;
    Place at = place_of(lane * 8, a.cols);
    const unsigned first = token<WAVES>((blockIdx.x * (blockDim.x / team) + threadIdx.x / team) * each);    // (fewer than 2^32)
    const unsigned last = min(first + each, a.rows);
    const TX *x = static_cast<const TX *>(f.x);
    const TH *h = static_cast<const TH *>(f.h);
    const auto some_row = [&](unsigned row) { return (size_t)min(row, a.rows - 1); };       // (one that is there)
    Raw<TX, 8> rx = fetch_some<ROWS>(x + some_row(first) * f.ldx, at);
    Raw<TH, 8> rh{};
    if constexpr (H) rh = fetch_some<ROWS>(h + some_row(first) * f.ldh, at);
    float g1[8], b1[8], g2[8], b2[8], gate[8];                  // (gate: times what makes up for the dropped)
    if constexpr (H) {
        some_params<ROWS>(a.post_gamma, at, 1.f, g1);
        some_params<ROWS>(a.post_beta, at, 0.f, b1);
    }
    some_params<ROWS>(a.pre_gamma, at, 1.f, g2);
    some_params<ROWS>(a.pre_beta, at, 0.f, b2);
    unsigned gate_row = ~0u;
    const uint64_t call = a.drop.offset + (a.drop.step ? *a.drop.step : 0);
    const There<ROWS> some = columns_there<ROWS>(at);
    const auto bytes = [&](int n) { return n >= 4 ? ~0u : n > 0 ? (1u << 8 * n) - 1 : 0u; };
    const u32x2 codes = {bytes(at.n), bytes(at.n - 4)};         // of 8-bit float rows: zeros past the last column, whatever the token
    for (unsigned k = 0; k < each; ++k) {                       // as often in every team: there are barriers
        const unsigned row = first + k;
        const bool there = row < last;
        asm volatile("" : "+v"(at.at), "+v"(at.start));     // (no address of a lane's own is kept over tokens: two registers for each tensor)
        float v[8], u[8];
        float2 st1 = make_float2(0.f, 1.f), st2 = make_float2(0.f, 1.f);
        widen_some<ROWS>(rx, at, v);
        if constexpr (H) widen_some<ROWS>(rh, at, u);
        rx = fetch_some<ROWS>(x + some_row(row + 1) * f.ldx, at);
        if constexpr (H) rh = fetch_some<ROWS>(h + some_row(row + 1) * f.ldh, at);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        if constexpr (H) {
            if (a.post != kNormNone) {
                st1 = team_stats<ROWS, WAVES>(u, some, a.cols, a.post, a.eps, team, seg, sums);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = fmaf(fmaf(-st1.x, some[e], u[e]) * st1.y, g1[e], b1[e]);
            }
            const unsigned now = a.gate ? fast_div_any(min(row, a.rows - 1), a.gate_rows, m_gate) : 0;
            if (now != gate_row) {
                some_params<ROWS>(a.gate ? a.gate + (size_t)now * a.cols : nullptr, at, 1.f, gate);
#pragma unroll
                for (int e = 0; e < 8; ++e) gate[e] *= a.drop.up;
                gate_row = now;
            }
            if (a.drop.limit) drop_some(a.drop, call, row, lane, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(gate[e], u[e], v[e]);
        }
        if (there && f.xo) store_some<ROWS>(static_cast<TX *>(f.xo) + row * f.ldxo, at, v, f.past);
        if (a.pre != kNormNone) {
            st2 = team_stats<ROWS, WAVES>(v, some, a.cols, a.pre, a.eps, team, seg, sums);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(fmaf(-st2.x, some[e], v[e]) * st2.y, g2[e], b2[e]);
            activate_all(a.act, v);
            if (f.z_dtype == GSPC_F8) {
                const unsigned code = block_code(lanes_umax(top_of(v), 16));
                const int pitch = f8_pitch(a.cols), s_pitch = f8_scale_pitch(a.cols);
                if (there && at.at < (unsigned)pitch) {
                    *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(f.z) + (size_t)row * pitch + at.at) = f8_codes(v, block_up(code)) & codes;
                    uint8_t *s = f.z_scale + (size_t)row * s_pitch + lane / 16;
                    if (lane % 16 == 0) *s = (uint8_t)code;
                    else if (lane / 16 == pitch / kBlock8 - 1 && lane / 16 + lane % 16 < s_pitch) s[lane % 16] = 0;
                }
            } else if (there && f.z) {
                if (f.z_dtype == GSPC_F32) store_some<ROWS>(static_cast<float *>(f.z) + row * f.ldz, at, v);
                else store_some<ROWS>(static_cast<uint16_t *>(f.z) + row * f.ldz, at, v, f.past);
            }
        }
        if (there && f.stats && lane == 0) *reinterpret_cast<float4 *>(f.stats + (size_t)row * 4) = make_float4(st1.x, st1.y, st2.x, st2.y);
    }
}

hipError_t launch_residual_norm(const Residual &a, ResidualForward f, hipStream_t s) {
    const TeamGrid g = team_grid(a.cols, f.z_dtype == GSPC_F8 ? 16 : 8);
    // Tokens of a team: as few as keep every compute unit full.  With h, waves of a compute unit 12, 16, 20, 24, 28, 32: 50176 x 512 in bf16 takes 52.4,
    // 49.2, 55.5, 52.7, 50.0, 50.2 us (16 is what its registers let a compute unit hold; more go in turns, of unlike lengths); without, 28 are there at once
    const size_t teams = (size_t)(256 * (f.h ? 16 : 28) * kWave / g.threads) * g.teams;
    const unsigned each = (unsigned)((a.rows + teams - 1) / teams), of_block = each * g.teams;
    const unsigned blocks = (a.rows - 1) / of_block + 1;
    f.past = (size_t)a.rows * a.cols * 2 >= kPastCaches && (!f.xo || f.x_dtype == GSPC_F32 || whole_pieces(f.xo, a.cols * 2, f.ldxo * 2)) &&
             (f.z_dtype != GSPC_BF16 || whole_pieces(f.z, a.cols * 2, f.ldz * 2));
    const Rows kind = rows_of(a.cols);
    const auto run = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(g.threads), 0, s, a, f, g.team, each, div_magic(a.gate_rows));
        return hipGetLastError();
    };
    const auto of = [&](auto x, auto h, auto has) {
        typedef decltype(x) TX;
        typedef decltype(h) TH;
        constexpr bool H = decltype(has)::value;
        if (g.team >= kWave) return kind == kWhole ? run(residual_norm_kernel<TX, TH, H, kWhole, true>) : run(residual_norm_kernel<TX, TH, H, kRagged, true>);
        return kind == kWhole ? run(residual_norm_kernel<TX, TH, H, kWhole, false>)
             : kind == kRagged ? run(residual_norm_kernel<TX, TH, H, kRagged, false>) : run(residual_norm_kernel<TX, TH, H, kThin, false>);
    };
    const std::true_type yes;
    const std::false_type no;
    if (f.x_dtype == GSPC_F32)
        return !f.h ? of(0.f, 0.f, no) : f.h_dtype == GSPC_F32 ? of(0.f, 0.f, yes) : of(0.f, uint16_t(), yes);
    return !f.h ? of(uint16_t(), uint16_t(), no) : f.h_dtype == GSPC_F32 ? of(uint16_t(), 0.f, yes) : of(uint16_t(), uint16_t(), yes);
}

}  // namespace gspc
