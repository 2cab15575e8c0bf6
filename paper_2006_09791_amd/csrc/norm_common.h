// What the forward and backward kernels of group norm share: how a tensor of tokens is cut into blocks.
#pragma once

#include "tokens.h"
#include "tokens_internal.h"

namespace gspc {

constexpr int kNormThreads = 512;
constexpr int kSlab = 2048;             // channels of a block at most: 256 vectors

// Blocks that keep their channels and walk down the rows of one image: thread (tx, ty) holds vector tx of the slab's channels
// and the rows r0 + ty, r0 + ty + TY, ...
struct NormGrid {
    int V;                  // channels of a vector
    int slabs, nvs, TY, threads;
    int chunks, rows;       // blocks down an image and rows of each (the last has the rest)
    unsigned m_nvs, m_chunks, m_slabs;
};

struct NormBlock {
    int n, chunk, c0, c1, r0, r1, tx, ty, nv;
    bool active;
    int at;                 // first channel of this thread's vector: the row's last vector ends with the row
};

__device__ __forceinline__ NormBlock norm_block(const NormShape &h, const NormGrid &g, unsigned block) {
    NormBlock b;
    const unsigned q = fast_div_any(block, g.chunks, g.m_chunks), n = fast_div_any(q, g.slabs, g.m_slabs);
    b.n = n;
    b.chunk = block - q * g.chunks;
    b.c0 = (q - n * g.slabs) * kSlab;
    b.c1 = min(b.c0 + kSlab, h.C);
    b.r0 = b.chunk * g.rows;
    b.r1 = b.r0 + min(g.rows, h.P - b.r0);
    b.ty = fast_div(threadIdx.x, g.m_nvs);
    b.tx = threadIdx.x - b.ty * g.nvs;
    b.nv = g.V == 1 ? b.c1 - b.c0 : (b.c1 - b.c0 + 7) / 8;
    b.active = b.ty < g.TY && b.tx < b.nv;
    b.at = g.V == 1 ? b.c0 + b.tx : min(b.c0 + b.tx * 8, h.C - 8);
    return b;
}

inline NormGrid norm_grid(const NormShape &h, int blocks_wanted, int most_chunks) {
    NormGrid g;
    g.V = h.C >= 8 ? 8 : 1;
    g.slabs = (h.C + kSlab - 1) / kSlab;
    const int first = h.C < kSlab ? h.C : kSlab;
    g.nvs = (first + g.V - 1) / g.V;
    g.TY = kNormThreads / g.nvs;
    if (g.TY > h.P) g.TY = h.P;
    g.threads = round_up(g.TY * g.nvs, kWave);
    // enough blocks to fill the chip, of at least four rows per thread, or one where four leave compute units without a block
    long want = blocks_wanted / ((long)h.N * g.slabs), most = (h.P + 4L * g.TY - 1) / (4L * g.TY);
    if (most * h.N * g.slabs < 256) most = (h.P - 1) / g.TY + 1, want = 256 / ((long)h.N * g.slabs);
    if (want > most) want = most;
    if (want > most_chunks) want = most_chunks;
    if (want < 1) want = 1;
    // a thread adds up 1024 rows at most: in 131072 values behind one another (2^31 - 1 rows of 8 channels in 256 blocks) what is small is lost against
    // the sum so far, 5e-5 of the deviation
    const long least = (h.P - 1) / (1024L * g.TY) + 1;
    if (want < least && least * g.slabs <= 1 << 16) want = least;
    g.rows = (int)((h.P + want - 1) / want);
    g.chunks = (h.P - 1) / g.rows + 1;
    g.m_nvs = div_magic(g.nvs);
    g.m_chunks = div_magic(g.chunks);
    g.m_slabs = div_magic(g.slabs);
    return g;
}

// Images of one launch at most of a grid's kernels, and of those with a block of 256 threads an image.
inline long norm_images(const NormGrid &g) {
    return most_blocks(g.threads > 256 ? g.threads : 256) / ((unsigned)g.chunks * (unsigned)g.slabs);
}

// Lanes that share a sum of `count` values, where `sums` of them are taken by `threads` threads: a power of two up to a wave.
inline int group_lanes(int count, long sums, long threads) {
    int w = 1;
    while (w < count && w < kWave && 2 * w * sums <= threads) w *= 2;
    return w;
}

__device__ __forceinline__ int group_of(const NormShape &h, int channel) { return fast_div_any(channel, h.D, h.m_D); }

// Blocks that hold an image's `seg` channels (whole groups) of all P tokens in registers: `width` lanes (a power of two) hold a
// token's vectors, `slots` tokens at a time, `held` times.
struct HeldGrid {
    int seg, segs, log_width, slots, threads;
    int unit, units;        // what group sums are made of: vectors that lie in one group, or single channels; and those of a group
    unsigned m_segs, m_units;
    unsigned xcds_more, per_xcd;    // blocks of an XCD: see held_block
    int log_lanes;          // gradient: lanes that share a channel's sum over the slots
};

// Workgroups go to the eight XCDs in turn.  Each XCD gets consecutive (image, segment) pairs, so that the pieces of a cache line
// that several segments share are read through, and joined in, one L2.
__device__ __forceinline__ unsigned held_block(const HeldGrid &g, unsigned b) {
    const unsigned xcd = b & 7;
    return xcd * g.per_xcd + min(xcd, g.xcds_more) + (b >> 3);
}

// Sums over the tokens of an image and the channels of a group.  `part` holds [slots][row] values, row = seg / unit; one wave
// takes a group, and one of its lanes calls f(group, sum).
template <typename F>
__device__ __forceinline__ void held_group_sums(const HeldGrid &g, const float *part, int row, int groups, F f) {
    const int lane = threadIdx.x % kWave, waves = (g.threads + kWave - 1) / kWave;
    for (int k = threadIdx.x / kWave; k < groups; k += waves) {
        float sum = 0.f;
        for (int j = lane; j < g.slots * g.units; j += kWave) {
            const int slot = fast_div(j, g.m_units);
            sum += part[slot * row + k * g.units + j - slot * g.units];
        }
        sum = lanes_sum(sum, kWave);
        if (lane == 0) f(k, sum);
    }
}

// Such blocks for segments of `groups` groups and up to `threads` threads that hold up to `held` vectors each, or false.
inline bool held_grid(const NormShape &h, int groups, int threads, int held, HeldGrid *g) {
    g->seg = groups * h.D;
    g->segs = h.groups / groups;
    const int nv = h.C >= 8 ? (g->seg + 7) / 8 : g->seg;
    if ((h.C >= 8 && g->seg < 8) || nv > kWave) return false;
    g->log_width = 0;
    while ((1 << g->log_width) < nv) ++g->log_width;
    const long wanted = (long)h.P << g->log_width;          // no more threads than there are vectors
    g->threads = wanted < threads ? round_up((int)wanted, kWave) : threads;
    g->slots = g->threads >> g->log_width;
    if ((h.P - 1) / g->slots >= held) return false;
    g->unit = h.D % 8 == 0 ? 8 : 1;
    g->units = h.D / g->unit;
    g->m_segs = div_magic(g->segs);
    g->m_units = div_magic(g->units);
    const size_t blocks = (size_t)h.N * g->segs;
    g->per_xcd = (unsigned)(blocks / 8);
    g->xcds_more = (unsigned)(blocks % 8);
    return blocks < 0x7fffffffu / 1024;
}

// The grid that is taken, or false: segments of 64 bytes of a token at least (of `size` bytes a value; half a cache line: in pieces of
// 32 group norm of 64 images of 56x56, 256 channels in bf16 took 71 us, and 114 past the caches), of 128 where that leaves four blocks for
// each compute unit; as few threads as hold them in `held` vectors each (`most` at most), more where the launch does not fill the
// chip with them (one image of 7x7, 512 channels in fp32: 3.8 us with 64 threads, 3.5 with 128).
inline bool plan_held(const NormShape &h, int size, int held, int most, HeldGrid *best) {
    bool found = false;
    for (int s = 1; s <= h.groups && s * (long)h.D <= 8 * kWave; ++s) {
        if (h.groups % s) continue;
        const int bytes = s * h.D * size;
        if (s < h.groups && bytes < 64) continue;
        if (found && (long)h.N * (h.groups / s) < 1024) break;
        for (int t = 64; t <= most; t *= 2) {
            HeldGrid g;
            if (!held_grid(h, s, t, held, &g)) continue;
            const bool fills = (long)h.N * g.segs * g.threads >= 65536;
            if (!fills && t < most && (h.P - 1) / g.slots >= 2) continue;
            *best = g;
            found = true;
            break;
        }
        if (bytes >= 128) break;
    }
    return found;
}

// V channels' parameters, or `none` for each where there are none.
template <int V> __device__ __forceinline__ void load_params(const float *__restrict__ p, int at, float none, float (&v)[V]) {
    if (p) widen(fetch<V>(p + at), v);
    else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = none;
    }
}

}  // namespace gspc
