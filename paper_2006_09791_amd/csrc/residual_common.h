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

// Mean and 1 / deviation of a token, of v's first n values a lane: a wave's own mean and the squares around it, joined over the waves (so that
// an offset does not cancel in them).  seg: the wave's number in its team.
__device__ __forceinline__ float2 team_stats(const float (&v)[8], int n, int cols, int kind, float eps, int team, int seg, TeamSums &t) {
    const float count = (float)cols;
    if (kind == kNormRms) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = e < n ? fmaf(v[e], v[e], s) : s;
        return make_float2(0.f, 1.f / sqrtf(team_sum(make_float2(s, 0.f), team, t).x / count + eps));
    }
    const int width = min(team, kWave);
    const auto of = [&](int wave) { return (float)max(0, min(cols - wave * 8 * kWave, 8 * kWave)); };
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += e < n ? v[e] : 0.f;
    const float mine = of(seg);
    float mean = mine > 0.f ? lanes_sum(sum, width) / mine : 0.f, squares = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) squares = e < n ? fmaf(v[e] - mean, v[e] - mean, squares) : squares;
    squares = lanes_sum(squares, width);
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

// Eight values of a parameter of which the first n are there, or `none` for each.
__device__ __forceinline__ void some_params(const float *__restrict__ p, int at, int n, float none, float (&v)[8]) {
    if (p) widen(fetch_some(p + at, n), v);
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = none;
    }
}

}  // namespace gspc
