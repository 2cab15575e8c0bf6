// What the forward and backward kernels of a block's residual norms share: a team of lanes holds one token, eight channels a lane.
#pragma once

#include "dropout.h"
#include "float8.h"
#include "tokens_internal.h"

namespace gspc {

// A team is a power of two of lanes, of a wave's or of several waves; a block has one or more, each with tokens of its own.
constexpr int kTeamThreads = 256;       // of a block, unless a team is larger
constexpr int kMaxTeam = 1024;

struct TeamGrid {
    int team, threads;
    unsigned teams;         // of a block
};
inline TeamGrid team_grid(int cols, int least) {
    TeamGrid g;
    g.team = least;
    while (g.team * 8 < cols) g.team *= 2;
    g.threads = g.team > kTeamThreads ? g.team : kTeamThreads;
    g.teams = g.threads / g.team;
    return g;
}

// Sums over a team of two numbers at once; every lane gets them.  Waves of a team meet in LDS, in two places by turns: when a place is written
// again, a barrier has passed since it was read.
struct TeamSums {
    float2 (*place)[kMaxTeam / kWave];
    int turn;
};
__device__ __forceinline__ float2 team_sum(float2 v, int team, TeamSums &t) {
    const int width = min(team, kWave);
    v.x = lanes_sum(v.x, width);
    v.y = lanes_sum(v.y, width);
    if (team > kWave) {
        const int waves = team / kWave, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
        if (lane == 0) t.place[t.turn][wave] = v;
        __syncthreads();
        v = t.place[t.turn][(wave & -waves) + (lane & (waves - 1))];
        v.x = lanes_sum(v.x, waves);
        v.y = lanes_sum(v.y, waves);
        t.turn ^= 1;
    }
    return v;
}

// Mean and 1 / deviation of a token, of the values of v that are there (n of a lane's; the others are 0): a wave's own mean and the squares around it,
// joined over the waves (so that an offset does not cancel in them).  seg: the wave's number in its team.
template <Rows ROWS>
__device__ __forceinline__ float2 team_stats(const float (&v)[8], int n, int cols, int kind, float eps, int team, int seg, TeamSums &t) {
    const float count = (float)cols;
    float sum = 0.f;
    if (kind == kNormRms) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
        return make_float2(0.f, 1.f / sqrtf(team_sum(make_float2(sum, 0.f), team, t).x / count + eps));
    }
    const int width = min(team, kWave);
    const auto of = [&](int wave) { return (float)max(0, min(cols - wave * 8 * kWave, 8 * kWave)); };
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[e];
    const float mine = of(seg);
    float mean = mine > 0.f ? lanes_sum(sum, width) / mine : 0.f, squares = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = ROWS == kWhole || e < n ? v[e] - mean : 0.f;
        squares = fmaf(d, d, squares);
    }
    squares = lanes_sum(ROWS == kWhole && n == 0 ? 0.f : squares, width);
    if (team > kWave) {
        const int waves = team / kWave, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, other = lane & (waves - 1);
        if (lane == 0) t.place[t.turn][wave] = make_float2(mean, squares);
        __syncthreads();
        const float2 o = t.place[t.turn][(wave & -waves) + other];
        mean = lanes_sum(of(other) * o.x, waves) / count;
        squares = lanes_sum(o.y + of(other) * (o.x - mean) * (o.x - mean), waves);
        t.turn ^= 1;
    }
    return make_float2(mean, 1.f / sqrtf(squares / count + eps));
}

// Eight values of a parameter, or `none` for each.
template <Rows ROWS> __device__ __forceinline__ void some_params(const float *__restrict__ p, const Place &at, float none, float (&v)[8]) {
    if (p) widen_some<ROWS>(fetch_some<ROWS>(p, at), at, v);
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = none;
    }
}

// Eight values of a type that the launch names, raw until they are used.
struct RawAny {
    Raw32 r;
};
template <Rows ROWS> __device__ __forceinline__ RawAny fetch_any(const void *t, int dtype, size_t off, const Place &at, bool there) {
    if (dtype == GSPC_F32) return {fetch_some<ROWS>(static_cast<const float *>(t) + off, at, there)};
    RawAny a{};
    a.r.a = __builtin_bit_cast(f32x4, fetch_some<ROWS>(static_cast<const uint16_t *>(t) + off, at, there).a);
    return a;
}
template <Rows ROWS> __device__ __forceinline__ void widen_any(const RawAny &a, int dtype, const Place &at, float (&v)[8]) {
    if (dtype == GSPC_F32) widen_some<ROWS>(a.r, at, v);
    else widen_some<ROWS>(Raw16{__builtin_bit_cast(u32x4, a.r.a)}, at, v);
}

}  // namespace gspc
