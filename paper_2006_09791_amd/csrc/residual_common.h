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
// again, a barrier has passed since it was read.  WAVES: the team is one wave or several (its width in a wave is a constant, and a sum is without
// branches); else it is 8, 16 or 32 lanes.
struct TeamSums {
    float2 (*place)[kMaxTeam / kWave];
    int turn;
};
template <bool WAVES> __device__ __forceinline__ float2 wave_sum(float2 v, int team) {
    const auto sums = [&](auto width) {
        constexpr int WIDTH = decltype(width)::value;
        return make_float2(lanes_sum(v.x, WIDTH), lanes_sum(v.y, WIDTH));
    };
    if constexpr (WAVES) return sums(std::integral_constant<int, 64>());
    else return team == 32 ? sums(std::integral_constant<int, 32>()) : team == 16 ? sums(std::integral_constant<int, 16>()) : sums(std::integral_constant<int, 8>());
}
// A sum over the teams of a wave, of 8, 16 or 32 lanes: of the lanes that have the same columns.
__device__ __forceinline__ float sum_across(float v, int team) {
    if (team == 8) v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x128, 0xf, 0xf, true));     // row_ror: lane ^ 8
    if (team <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// What the other waves of the team have: lane l of the first sixteen that of wave l, 0 where there is none.
__device__ __forceinline__ float2 team_exchange(float2 v, int team, TeamSums &t) {
    const int waves = team / kWave, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (lane == 0) t.place[t.turn][wave] = v;
    __syncthreads();
    v = t.place[t.turn][(wave & -waves) + (lane & (waves - 1))];
    t.turn ^= 1;
    return lane % 16 < waves ? v : make_float2(0.f, 0.f);
}
template <bool WAVES> __device__ __forceinline__ float2 team_sum(float2 v, int team, TeamSums &t) {
    v = wave_sum<WAVES>(v, team);
    if (WAVES && team > kWave) {
        const float2 o = team_exchange(v, team, t);
        v = make_float2(lanes_sum(o.x, 16), lanes_sum(o.y, 16));
    }
    return v;
}

template <bool WAVES> __device__ __forceinline__ float team_sum(float v, int team, TeamSums &t) {
    v = wave_sum<WAVES>(make_float2(v, 0.f), team).x;       // (the zero's sum is not made)
    return WAVES && team > kWave ? lanes_sum(team_exchange(make_float2(v, 0.f), team, t).x, 16) : v;
}

// a / n by the reciprocal, corrected once: exact where the quotient is a number (a constant token's mean is its value).  A sum past fp32's range stays
// infinite (its correction is no number, which the maximum drops), so that 1 / deviation becomes 0.
__device__ __forceinline__ float ratio(float a, float n) {
    const float r = __builtin_amdgcn_rcpf(n), q = a * r;
    return fmaf(fmaxf(fmaf(-q, n, a), -__FLT_MAX__), r, q);
}

// 1 for a lane's columns that are there, else 0.  A mean is subtracted times it, fmaf(-mean, there, v), so that what is not there stays 0 in every
// sum, at no cost (conditions would be kept in pairs of scalar registers, of which there are not enough).
template <Rows ROWS> struct There {
    float one[ROWS == kWhole ? 1 : 8];          // (all of a lane's eight, or none)
    __device__ __forceinline__ float operator[](int e) const { return one[ROWS == kWhole ? 0 : e]; }
};
template <Rows ROWS> __device__ __forceinline__ There<ROWS> columns_there(const Place &at) {
    There<ROWS> t;
#pragma unroll
    for (int e = 0; e < (ROWS == kWhole ? 1 : 8); ++e) t.one[e] = e < at.n ? 1.f : 0.f;
    return t;
}

// Mean and 1 / deviation of a token, of values of which those that are not there are 0: a wave's own mean and the squares around it, joined over the
// waves (so that an offset does not cancel in them).  seg: the wave's number in its team.
template <Rows ROWS, bool WAVES>
__device__ __forceinline__ float2 team_stats(const float (&v)[8], const There<ROWS> &there, int cols, int kind, float eps, int team, int seg, TeamSums &t) {
    const float count = (float)cols;
    float sum = 0.f;
    if (kind == kNormRms) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
        return make_float2(0.f, rsqrtf(ratio(team_sum<WAVES>(sum, team, t), count) + eps));
    }
    const auto of = [&](int wave) { return (float)max(0, min(cols - wave * 8 * kWave, 8 * kWave)); };
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[e];
    const float mine = of(seg);
    float mean = mine > 0.f ? ratio(wave_sum<WAVES>(make_float2(sum, 0.f), team).x, mine) : 0.f, squares = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = fmaf(-mean, there[e], v[e]);
        squares = fmaf(d, d, squares);
    }
    squares = wave_sum<WAVES>(make_float2(squares, 0.f), team).x;
    if (WAVES && team > kWave) {
        const float2 o = team_exchange(make_float2(mean, squares), team, t);
        const int other = threadIdx.x % 16;             // (a wave that is not there has no columns)
        mean = ratio(lanes_sum(of(other) * o.x, 16), count);
        squares = lanes_sum(o.y + of(other) * (o.x - mean) * (o.x - mean), 16);
    }
    return make_float2(mean, rsqrtf(ratio(squares, count) + eps));
}

// Eight values of a parameter, or `none` for each.
template <Rows ROWS> __device__ __forceinline__ void some_params(const float *__restrict__ p, const Place &at, float none, float (&v)[8]) {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = none;
    if (p) widen_some<ROWS>(fetch_some<ROWS>(p, at), at, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = w[e];        // (in one order, whichever: stores of two would be put together, and v into memory)
}

// Eight values of a type that the launch names, raw until they are used.
template <Rows ROWS> __device__ __forceinline__ Raw32 fetch_any(const void *t, int dtype, size_t off, const Place &at) {
    if (dtype == GSPC_F32) return fetch_some<ROWS>(static_cast<const float *>(t) + off, at);
    Raw32 r{};
    r.a = __builtin_bit_cast(f32x4, fetch_some<ROWS>(static_cast<const uint16_t *>(t) + off, at).a);
    return r;
}
template <Rows ROWS> __device__ __forceinline__ void widen_any(const Raw32 &r, int dtype, const Place &at, float (&v)[8], bool there) {
    if (dtype == GSPC_F32) widen_some<ROWS>(r, at, v, there);
    else widen_some<ROWS>(Raw16{__builtin_bit_cast(u32x4, r.a)}, at, v, there);
}

// The number of a team's token, the same for a wave where a team is one or more.
template <bool WAVES> __device__ __forceinline__ unsigned token(unsigned n) { return WAVES ? __builtin_amdgcn_readfirstlane(n) : n; }

}  // namespace gspc
