// Gradient of a block's residual norms.  With hh and xh the normalised h and x', w what dropout multiplies by, u = g1 hh + b1, v = g2 xh + b2:
//   dv = dz act'(v), t = g2 dv, dX = dx' + r2 (t - mean t - xh mean(t xh)), dx = scale dX,
//   q = g1 gate w dX, dh = r1 (q - mean q - hh mean(q hh))                     (no mean t, mean q behind a root mean square)
// and over tokens, with A = sum w dX hh and B = sum w dX of the tokens that share a gate: dg1 = gate A, db1 = gate B, dgate = g1 A + b1 B (two sums
// serve the three), dg2 = sum dv xh, db2 = sum dv.
#include "residual_common.h"

namespace gspc {

constexpr int kSums = 5;        // dg1, db1, dg2, db2, dgate

struct GradPlan {
    unsigned chunks;            // blocks that share a gate's tokens, or 0: a team takes whole gates
    unsigned rows;              // tokens of such a block, or of a team
    unsigned each;              // tokens of a team
    unsigned blocks;
};

// A team walks down its tokens and keeps the sums of its columns; a block's teams add theirs up and leave one part.  dz, dx', x' and h in, dx and dh out:
// bound by memory and, nearly as much, by vector instructions (50176 x 512 in bf16, two norms, dropout and SiLU, 309 MB: 66.5 us, 4.6 TB/s; 480
// instructions for a wave's 512 values).  GATES: a team's tokens have several gates, whose gradients it writes itself.  LARGE: teams of
// more than 512 lanes, which leave 128 registers each: parameters are in LDS, and no token is ahead (4096 x 8192, 403 MB, with
// the join: 113 us; with parameters read again for each token a quarter more; 8192 x 4096, as many bytes, 93).
template <typename TX, typename TH, bool GATES, bool LARGE, Rows ROWS, bool WAVES>
__global__ __launch_bounds__(LARGE ? kMaxTeam : kMaxTeam / 2) void residual_grad_kernel(Residual a, ResidualBackward f, GradPlan g, int of_team, unsigned m_chunks,
                                                                 float *__restrict__ parts) {
    __shared__ float2 s_place[2][kMaxTeam / kWave];
    __shared__ float s_sum[kTeamThreads * 8];              // (of several teams)
    __shared__ f32x4 s_mine[LARGE ? 6 : 1][LARGE ? kMaxTeam : 1];       // a lane's own parameters
    TeamSums sums{s_place, 0};
    const int team = LARGE ? kMaxTeam : of_team, lane = threadIdx.x & (team - 1);
    Place at = place_of(lane * 8, a.cols);
    const unsigned teams = LARGE ? 1 : blockDim.x / team, mine = LARGE ? 0 : threadIdx.x / team;
    unsigned first, last, gate_row = 0;
    if constexpr (GATES) {
        first = token<WAVES>((blockIdx.x * teams + mine) * g.each);
        last = min(first + g.each, a.rows);
        gate_row = first / a.gate_rows;
    } else {
        const unsigned group = fast_div_any(blockIdx.x, g.chunks, m_chunks), chunk = blockIdx.x - group * g.chunks;
        const unsigned end = min(chunk * g.rows + g.rows, a.gate_rows);
        first = token<WAVES>(group * a.gate_rows + min(chunk * g.rows + mine * g.each, end));
        last = min(first + g.each, group * a.gate_rows + end);
        gate_row = group;
    }
    const TX *const xo = static_cast<const TX *>(f.xo), *const dxo = static_cast<const TX *>(f.dxo);
    const TH *const h = static_cast<const TH *>(f.h);
    // A token's values, raw: the next one's are on their way while this one's are worked on.
    Raw32 r_dz{};
    Raw<TX, 8> r_xo{}, r_dxo{};
    Raw<TH, 8> r_h{};
    float4 r_st = make_float4(0.f, 1.f, 0.f, 1.f);
    // (of a token that is there; tensors that are not are read somewhere else, and not used)
    const auto load_norm = [&](unsigned row) {
        const size_t r = min(row, a.rows - 1);
        r_st = *reinterpret_cast<const float4 *>(f.stats + r * 4);
        r_dz = fetch_any<ROWS>(f.dz, f.dz_dtype, r * f.lddz, at);
        r_xo = fetch_some<ROWS>(xo + r * f.ldxo, at);
    };
    const auto load_stream = [&](unsigned row) { r_dxo = fetch_some<ROWS>(dxo + (size_t)min(row, a.rows - 1) * f.lddxo, at); };
    const auto load_h = [&](unsigned row) { r_h = fetch_some<ROWS>(h + (size_t)min(row, a.rows - 1) * f.ldh, at); };
    if constexpr (!LARGE) {
        load_norm(first);
        load_stream(first);
        load_h(first);
    }
    const float inv = 1.f / (float)a.cols;
    const There<ROWS> some = columns_there<ROWS>(at);
    const bool centre1 = a.post == kNormLayer, centre2 = a.pre == kNormLayer;
    const uint64_t call = a.drop.offset + (a.drop.step ? *a.drop.step : 0);
    float g2[8], b2[8], gg[8];                                  // gg: g1 gate, times what makes up for the dropped
    const auto pre_params = [&] {
        some_params<ROWS>(a.pre_gamma, at, 1.f, g2);
        some_params<ROWS>(a.pre_beta, at, 0.f, b2);
    };
    const auto keep = [&](int place, const float (&v)[8]) {     // (LARGE: in LDS instead of registers; nobody else reads them)
        if constexpr (LARGE) {
            s_mine[place][threadIdx.x] = (f32x4){v[0], v[1], v[2], v[3]};
            s_mine[place + 1][threadIdx.x] = (f32x4){v[4], v[5], v[6], v[7]};
        }
    };
    const auto get = [&](int place, float (&v)[8]) {
        if constexpr (LARGE) {
            const f32x4 a = s_mine[place][threadIdx.x], b = s_mine[place + 1][threadIdx.x];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
        }
    };
    pre_params();
    keep(0, g2);
    keep(2, b2);
    const auto new_gate = [&] {
        float gate[8];
        some_params<ROWS>(a.post_gamma, at, 1.f, gg);
        some_params<ROWS>(a.gate ? a.gate + (size_t)gate_row * a.cols : nullptr, at, 1.f, gate);
#pragma unroll
        for (int e = 0; e < 8; ++e) gg[e] *= gate[e] * a.drop.up * some[e];
        keep(4, gg);
    };
    if (!GATES || first < last) new_gate();
    float sa[8] = {}, sb[8] = {}, sg2[8] = {}, sb2[8] = {}, sg1[GATES ? 8 : 1] = {}, sb1[GATES ? 8 : 1] = {};
    // A gate's tokens are through: its gradient, and what its sums are to the parameters'.
    const auto end_gate = [&](float (&dgate)[8], float (&dg1)[8], float (&db1)[8]) {
        float gate[8], g1[8], b1[8];
        some_params<ROWS>(a.gate ? a.gate + (size_t)gate_row * a.cols : nullptr, at, 1.f, gate);
        some_params<ROWS>(a.post_gamma, at, 1.f, g1);
        some_params<ROWS>(a.post_beta, at, 0.f, b1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float da = sa[e] * a.drop.up, db = sb[e] * a.drop.up;
            dgate[e] = fmaf(g1[e], da, b1[e] * db);
            dg1[e] = gate[e] * da;
            db1[e] = gate[e] * db;
        }
    };
    const auto phase = [] {                                     // (nothing is loaded ahead of it where registers are few)
        if constexpr (LARGE) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    unsigned left = a.gate_rows;                                // tokens of this gate to come (GATES)
    for (unsigned k = 0; k < g.each; ++k) {                     // as often in every team: there are barriers
        const unsigned row = first + k;
        const bool there = row < last;
        asm volatile("" : "+v"(at.at), "+v"(at.start));     // (no address of a lane's own is kept over tokens: two registers for each tensor)
        if constexpr (LARGE) {
            load_norm(row);
            if constexpr (!GATES) {
                load_stream(row);
                load_h(row);
            }
        }
        const float4 st = there ? r_st : make_float4(0.f, 1.f, 0.f, 1.f);
        float dv[8] = {}, d[8] = {}, xh[8], hh[8];
        widen_any<ROWS>(r_dz, f.dz_dtype, at, dv, there && f.has_dz);
        widen_some<ROWS>(r_xo, at, xh, there);
        if constexpr (!LARGE) {
            widen_some<ROWS>(r_dxo, at, d, there && f.has_dxo);
            widen_some<ROWS>(r_h, at, hh, there);
            load_norm(row + 1);
            load_stream(row + 1);
            load_h(row + 1);
        }
        if (f.has_dz) {
            get(0, g2);
            get(2, b2);
            phase();
            float2 s = make_float2(0.f, 0.f);
            float t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) xh[e] = fmaf(-st.z, some[e], xh[e]) * st.w;
            if (a.act != kActNone) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = fmaf(xh[e], g2[e], b2[e]);
                    dv[e] *= a.act == kActRelu ? slope<kActRelu>(v) : slope<kActSilu>(v);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sg2[e] = fmaf(dv[e], xh[e], sg2[e]);
                sb2[e] += dv[e];
                t[e] = g2[e] * dv[e];
                s.x += t[e];
                s.y = fmaf(t[e], xh[e], s.y);
            }
            s = team_sum<WAVES>(s, team, sums);
            const float m = centre2 ? s.x * inv : 0.f, c = s.y * inv;
            phase();
            if constexpr (LARGE) {
                if constexpr (GATES) load_stream(row);
                widen_some<ROWS>(r_dxo, at, d, there && f.has_dxo);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = fmaf(st.w, t[e] - m - xh[e] * c, d[e]);
        } else if constexpr (LARGE) {
            if constexpr (GATES) load_stream(row);
            widen_some<ROWS>(r_dxo, at, d, there && f.has_dxo);
        }
        phase();
        if (there) {
            float out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = a.scale * d[e];
            store_some<ROWS>(static_cast<TX *>(f.dx) + row * f.lddx, at, out, f.past);
        }
        if (f.has_h) {
            Philox which{};
            if (a.drop.limit) {
                which = drop_numbers(a.drop, call, row, lane);
                drop_by(which, a.drop.limit, d);
            }
            phase();
            if constexpr (LARGE) {
                if constexpr (GATES) load_h(row);
                widen_some<ROWS>(r_h, at, hh, there);
                get(4, gg);
            }
            phase();
            float2 s = make_float2(0.f, 0.f);
            float q[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) hh[e] = fmaf(-st.x, some[e], hh[e]) * st.y;
            // What was dropped has no say in the sums, whatever it was: 0 times it need not be 0.  Behind a norm that is all of a token or nothing of it, as
            // 1 / deviation tells (never 0 of numbers but where squares pass fp32); the selection for each token cost 4 us of 91 on 8192 x 4096.
            if (a.drop.limit && (a.post == kNormNone || !(st.y > 0.f && st.y < __builtin_inff()))) {
                float kept[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) kept[e] = hh[e];
                drop_by(which, a.drop.limit, kept);
#pragma unroll
                for (int e = 0; e < 8; ++e) sa[e] = fmaf(d[e], kept[e], sa[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) sa[e] = fmaf(d[e], hh[e], sa[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sb[e] += d[e];
                q[e] = gg[e] * d[e];
                s.x += q[e];
                s.y = fmaf(q[e], hh[e], s.y);
            }
            if (a.post != kNormNone) {
                s = team_sum<WAVES>(s, team, sums);
                const float m = centre1 ? s.x * inv : 0.f, c = s.y * inv;
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = st.y * (q[e] - m - hh[e] * c);
            }
            if (there) store_some<ROWS>(static_cast<TH *>(f.dh) + row * f.lddh, at, q, f.past);
        }
        if constexpr (GATES) {
            if (--left == 0) {
                if (there) {
                    float dgate[8], dg1[8], db1[8];
                    end_gate(dgate, dg1, db1);
                    if (f.dgate) store_some<ROWS>(f.dgate + (size_t)gate_row * a.cols, at, dgate);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sg1[e] += dg1[e], sb1[e] += db1[e], sa[e] = sb[e] = 0.f;
                    ++gate_row;
                    if (row + 1 < last) new_gate();
                }
                left = a.gate_rows;
            }
        }
    }
    float dgate[8], dg1[8], db1[8];
    if constexpr (GATES) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dg1[e] = sg1[e], db1[e] = sb1[e];
    } else
        end_gate(dgate, dg1, db1);
    // The teams' sums as one part of the block, a kind at a time: those of a wave's teams by lanes, then waves through LDS.
    const auto leave = [&](float (&v)[8], float *to) {
        if constexpr (!WAVES)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = sum_across(v[e], team);
        const int width = WAVES ? team * 8 : kWave * 8, places = WAVES ? (int)teams : kTeamThreads / kWave;
        if (places == 1) {
            store_some<ROWS>(to, at, v);
            return;
        }
        __syncthreads();
        if (WAVES || threadIdx.x % kWave < (unsigned)team) store(s_sum + (WAVES ? mine : threadIdx.x / kWave) * width + lane * 8, v);
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            float sum = s_sum[c] + s_sum[width + c];
            if (places == 4) sum += s_sum[2 * width + c] + s_sum[3 * width + c];
            to[c] = sum;
        }
    };
    float *part = parts + (size_t)blockIdx.x * kSums * a.cols;
    if (f.dpost_gamma) leave(dg1, part);
    if (f.dpost_beta) leave(db1, part + a.cols);
    if (f.dpre_gamma) leave(sg2, part + 2 * a.cols);
    if (f.dpre_beta) leave(sb2, part + 3 * a.cols);
    if (!GATES && f.dgate) leave(dgate, g.chunks == 1 ? f.dgate + (size_t)gate_row * a.cols : part + 4 * a.cols);
}

// Adds up the blocks' parts, in 64 bits: 32 columns (a cache line of a part) a block, 32 stretches of the parts side by side, two of them in a wave.
// Block (kind, columns): the four parameters' over all parts, then each gate's over those of its own blocks.  Latency: eight loads on their way at
// once (761 parts of 512 columns, of five kinds, 7.8 MB: 4.9 us; 64 columns and 16 stretches, 6.4).
constexpr int kJoinCols = 32, kJoinSlices = 32;
__global__ __launch_bounds__(kJoinCols * kJoinSlices) void residual_join_kernel(const float *__restrict__ parts, unsigned blocks, unsigned chunks, int cols,
                                                                                unsigned slabs, float *dg1, float *db1, float *dg2, float *db2, float *dgate) {
    __shared__ double s_sum[kJoinSlices / 2][kJoinCols];
    const unsigned kind = blockIdx.x / slabs, slab = blockIdx.x - kind * slabs, gate = kind - 4;
    const int lane = threadIdx.x % kJoinCols, slice = threadIdx.x / kJoinCols, c = slab * kJoinCols + lane;
    float *to = kind == 0 ? dg1 : kind == 1 ? db1 : kind == 2 ? dg2 : kind == 3 ? db2 : dgate + (size_t)gate * cols;
    if (kind < 4 && !to) return;
    const unsigned first = kind < 4 ? 0 : gate * chunks, count = kind < 4 ? blocks : chunks;
    const float *p = parts + ((size_t)first * kSums + min(kind, 4u)) * cols + min(c, cols - 1);
    double sum = 0;
    for (unsigned k = slice; k < count; k += 8 * kJoinSlices) {     // (those past the end: the last one, not added)
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[(size_t)min(k + kJoinSlices * i, count - 1) * kSums * cols];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += k + kJoinSlices * i < count ? v[i] : 0.f;
    }
    sum += __shfl_xor(sum, kJoinCols);
    if (slice % 2 == 0) s_sum[slice / 2][lane] = sum;
    __syncthreads();
    if (slice != 0 || c >= cols) return;
#pragma unroll
    for (int k = 1; k < kJoinSlices / 2; ++k) sum += s_sum[k][lane];
    to[c] = (float)sum;
}

__global__ __launch_bounds__(256) void residual_clear_kernel(float *p, size_t count) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (size_t)gridDim.x * 256) p[i] = 0.f;
}

static_assert(kTeamThreads == 4 * kWave, "a block's teams are in one, two or four waves");

// As many blocks as are at work at once: of 1024 lanes one a compute unit, of fewer eight waves.  (Twelve, which the registers would hold, have half
// as many parts again to add up, and leave 1.5 blocks of 512 lanes for each compute unit: 12544 x 512 in bf16, layer norms, SiLU and dropout, with 4, 8, 12
// and 16: 28.9, 25.0, 26.2, 32.5 us; 2000 x 4096: 46.4, 31.5, 43.8, 39.6.  Of 1024 lanes, 4096 x 8192, 8, 16 and 32: 234, 134, 144.)  Twelve all
// the same where teams of one or two waves have 8 tokens each or more (faster at 52 of 70 sizes of 320 to 1024 channels, by 2.3 % in the mean of all), with 8
// waves and 12, behind the forward call: 24576 x 320 in bf16 56.7 and 54.4, 43008 x
// 320 90.8 and 84.5, 12288 x 640 62.5 and 59.4, 49152 x 640 207 and 190; where channels fill the team, 24576 x 512 63.6 and 62.2, 36864 x 512 88.6 and 90.7, 49152
// x 512 116 and 112, 15360 x 1024 83.5 and 81.8, 24576 x 1024 119 and 111, 24576 x 512 in fp32 115.5 and 114.8; with fewer tokens, 12288 x 512 38.2 and 39.3, 6144 x
// 1024 without dropout 33.0 and 34.3.  Teams of 32 or 256 lanes, 100352 x 256 and 20000 x 2048: 71.8 and 75.2, 110 and 115.
static GradPlan plan_grad(const Residual &a, const TeamGrid &t) {
    const bool many = (t.team == kWave || t.team == 2 * kWave) && a.rows / (256 * 12 * kWave / t.threads * t.teams) >= 8;
    const unsigned rows = a.rows, gates = a.gates, gate_rows = a.gate_rows;
    const unsigned wanted = 256 * (t.team > kMaxTeam / 2 ? 16 : many ? 12 : 8) * kWave / t.threads;
    GradPlan p;
    if (gates > 1 && gates >= wanted * t.teams && gate_rows <= 1024) {      // whole gates for each team
        const unsigned of_team = (gates - 1) / (wanted * t.teams) + 1, most = 1024 / gate_rows;
        p.chunks = 0;
        p.each = p.rows = (of_team < most ? of_team : most) * gate_rows;
        p.blocks = (unsigned)(((size_t)rows - 1) / ((size_t)p.each * t.teams) + 1);
        return p;
    }
    // blocks of a gate: until there are enough of them, of 1024 tokens a team at most
    const unsigned most = (gate_rows - 1) / t.teams + 1, least = (gate_rows - 1) / (1024 * t.teams) + 1;
    unsigned want = wanted / gates;
    if (want > most) want = most;
    if (want < least) want = least;
    p.rows = (gate_rows - 1) / want + 1;
    p.chunks = (gate_rows - 1) / p.rows + 1;
    p.each = (p.rows - 1) / t.teams + 1;
    p.blocks = gates * p.chunks;
    return p;
}

size_t residual_grad_bytes(const Residual &a) {
    return a.rows ? (size_t)plan_grad(a, team_grid(a.cols, 8)).blocks * kSums * a.cols * sizeof(float) : 0;
}

hipError_t launch_residual_grad(const Residual &a, ResidualBackward f, void *ws, hipStream_t s) {
    if (a.rows == 0) {          // no tokens: the parameters' gradients are zero
        const auto clear = [&](float *p, size_t count) {
            const size_t blocks = (count + 255) / 256;
            if (p) hipLaunchKernelGGL(residual_clear_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, p, count);
        };
        for (float *p : {f.dpost_gamma, f.dpost_beta, f.dpre_gamma, f.dpre_beta}) clear(p, a.cols);
        clear(f.dgate, (size_t)a.gates * a.cols);
        return hipGetLastError();
    }
    // (what is not there: the row's place of something that is, again and again)
    f.has_dz = f.dz != nullptr, f.has_dxo = f.dxo != nullptr, f.has_h = f.h != nullptr;
    const void *const some = f.dxo ? f.dxo : f.xo;
    if (!f.xo) f.xo = some, f.ldxo = 0;
    if (!f.dxo) f.dxo = some, f.lddxo = 0;
    if (!f.dz) f.dz = some, f.lddz = 0, f.dz_dtype = f.x_dtype;
    if (!f.h) f.h = some, f.ldh = 0, f.h_dtype = f.x_dtype;
    const TeamGrid g = team_grid(a.cols, 8);
    const GradPlan p = plan_grad(a, g);
    float *parts = static_cast<float *>(ws);
    f.past = (size_t)a.rows * a.cols * 2 >= kPastCaches && (f.x_dtype == GSPC_F32 || whole_pieces(f.dx, a.cols * 2, f.lddx * 2)) &&
             (!f.has_h || f.h_dtype == GSPC_F32 || whole_pieces(f.dh, a.cols * 2, f.lddh * 2));
    const auto run = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(p.blocks), dim3(g.threads), 0, s, a, f, p, g.team, div_magic(p.chunks ? p.chunks : 1), parts);
    };
    const auto of = [&](auto x, auto h, auto gates) {
        typedef decltype(x) TX;
        typedef decltype(h) TH;
        constexpr bool GATES = decltype(gates)::value;
        const Rows kind = rows_of(a.cols);
        if (g.team > kMaxTeam / 2) run(residual_grad_kernel<TX, TH, GATES, true, kRagged, true>);
        else if (g.team >= kWave) kind == kWhole ? run(residual_grad_kernel<TX, TH, GATES, false, kWhole, true>) : run(residual_grad_kernel<TX, TH, GATES, false, kRagged, true>);
        else if (kind == kWhole) run(residual_grad_kernel<TX, TH, GATES, false, kWhole, false>);
        else if (kind == kRagged) run(residual_grad_kernel<TX, TH, GATES, false, kRagged, false>);
        else run(residual_grad_kernel<TX, TH, GATES, false, kThin, false>);
    };
    const auto by_types = [&](auto gates) {
        if (f.x_dtype == GSPC_F32) f.h_dtype == GSPC_F32 ? of(0.f, 0.f, gates) : of(0.f, uint16_t(), gates);
        else f.h_dtype == GSPC_F32 ? of(uint16_t(), 0.f, gates) : of(uint16_t(), uint16_t(), gates);
    };
    p.chunks ? by_types(std::false_type()) : by_types(std::true_type());
    const unsigned slabs = (a.cols + kJoinCols - 1) / kJoinCols, kinds = 4 + (f.dgate && p.chunks > 1 ? a.gates : 0);
    if (kinds > 4 || f.dpost_gamma || f.dpost_beta || f.dpre_gamma || f.dpre_beta)
        hipLaunchKernelGGL(residual_join_kernel, dim3(kinds * slabs), dim3(kJoinCols * kJoinSlices), 0, s, parts, p.blocks, p.chunks, a.cols, slabs, f.dpost_gamma,
                           f.dpost_beta, f.dpre_gamma, f.dpre_beta, f.dgate);
    return hipGetLastError();
}

}  // namespace gspc
