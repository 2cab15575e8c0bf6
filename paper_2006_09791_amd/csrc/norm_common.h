// What the forward and backward kernels of group norm share: how a tensor of tokens is cut into blocks.
#pragma once

#include "tokens.h"
#include "tokens_internal.h"

namespace gspc {

constexpr int kNormThreads = 512;
constexpr int kSlab = 2048;             // channels of a block at most: 256 vectors
constexpr int kMaxChunks = 128;

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
    b.r1 = min(b.r0 + g.rows, h.P);
    b.ty = fast_div(threadIdx.x, g.m_nvs);
    b.tx = threadIdx.x - b.ty * g.nvs;
    b.nv = g.V == 1 ? b.c1 - b.c0 : (b.c1 - b.c0 + 7) / 8;
    b.active = b.ty < g.TY && b.tx < b.nv;
    b.at = g.V == 1 ? b.c0 + b.tx : min(b.c0 + b.tx * 8, h.C - 8);
    return b;
}

inline NormGrid norm_grid(const NormShape &h, int blocks_wanted) {
    NormGrid g;
    g.V = h.C >= 8 ? 8 : 1;
    g.slabs = (h.C + kSlab - 1) / kSlab;
    const int first = h.C < kSlab ? h.C : kSlab;
    g.nvs = (first + g.V - 1) / g.V;
    g.TY = kNormThreads / g.nvs;
    if (g.TY > h.P) g.TY = h.P;
    g.threads = round_up(g.TY * g.nvs, kWave);
    // enough blocks to fill the chip, of at least four rows per thread
    long want = blocks_wanted / ((long)h.N * g.slabs);
    const long most = (h.P + 4L * g.TY - 1) / (4L * g.TY);
    if (want > most) want = most;
    if (want > kMaxChunks) want = kMaxChunks;
    if (want < 1) want = 1;
    g.rows = (int)((h.P + want - 1) / want);
    g.chunks = (h.P + g.rows - 1) / g.rows;
    g.m_nvs = div_magic(g.nvs);
    g.m_chunks = div_magic(g.chunks);
    g.m_slabs = div_magic(g.slabs);
    return g;
}

// Lanes that share the sum of a group of `count` values: a power of two up to a wave.
inline int group_lanes(int count) {
    int w = 1;
    while (w < count && w < kWave) w *= 2;
    return w;
}

template <int V> __device__ __forceinline__ void activate_all(int act, float (&z)[V]) {
    if (act == kActRelu) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = activate<kActRelu>(z[e]);
    } else if (act == kActSilu) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = activate<kActSilu>(z[e]);
    }
}

}  // namespace gspc
