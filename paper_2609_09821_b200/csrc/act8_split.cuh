// How the weight gradient from 8 bits cuts its work: tile shape, workers (CTAs or pairs) to a tile, and the k-blocks (64 rows) of each.
#pragma once
#include <stddef.h>

namespace im {

constexpr int kTileK = 128;                // columns of H per CTA: the M of the instruction, or half of it
constexpr int kBlockRows = 64;             // rows of a k-block

// Narrow A: one CTA per tile, 64 or 128 columns; else pairs with 256, unless H is too narrow for both CTAs.  Each tile's rows are
// shared out to `slices` workers.  Workers left over may help: then every tile's workers take slice_kb k-blocks each, and the k-blocks
// behind those, tile after tile, are cut evenly among the helpers.
struct Split {
    int block_n;
    bool pair;
    int tiles_k, tiles, kb;                // tiles along H's columns, all tiles, k-blocks of a tile
    int workers;                           // CTAs or pairs
    int slices, slice_kb;                  // workers per tile and their k-blocks (no helpers: kb cut evenly)
    int helpers;
    size_t slot_bytes() const { return (size_t)block_n * (pair ? 2 : 1) * kTileK * sizeof(float); }
    bool whole() const { return slices == 1 && helpers == 0; }
};
// k-blocks of a part, at least (4096 x 256 x 256 12.4 us; with 2 13.2, with 8 13.7; 1024 x 69 x 512 9.2 us; 8.6 and 10.6)
constexpr int kLeastBlocks = 4;
// What helpers cost, in k-blocks, of a pair and of a lone CTA: another part of the same worker (its chain's end and its way to memory);
// partial tiles and their sum where whole tiles could go to C; and what has to be gained for sure.  Rows x 1280 x 1280 (25 tiles for 74
// pairs) with and without helpers: 4096 33 and 30 us, 8192 44 and 46, 16000 64 and 74, 131072 367 and 476; x 1024 x 1024 (16 tiles):
// 8192 33 and 30, 32768 73 and 76, 131072 237 and 253; x 2048 x 1280 (40): 4096 45 and 41, 8192 62 and 71; x 64 x 9600 (75 for 148
// CTAs): 2048 20.5 and 20.1, 4096 28 and 34.  Even shares, without the parts' cost, leave the helpers behind: 20000 x 512 x 1024 59 us and 30.
struct HelpCost { int part, sum, least; };
constexpr HelpCost kHelpPair = {12, 24, 6}, kHelpLone = {3, 9, 3};
inline Split split_for(int R, int Mo, int No, int ctas)
{
    Split s;
    s.pair = Mo > 128 && No > kTileK;
    s.block_n = s.pair ? 256 : Mo <= 64 ? 64 : 128;
    s.workers = s.pair ? ctas / 2 : ctas;
    const int cols = s.pair ? 2 * kTileK : kTileK;
    s.tiles_k = (No + cols - 1) / cols;
    s.tiles = s.tiles_k * ((Mo + s.block_n - 1) / s.block_n);
    s.kb = (R + kBlockRows - 1) / kBlockRows;
    const int most = s.kb / kLeastBlocks;
    s.slices = s.workers / s.tiles;
    s.slices = s.slices < most ? s.slices : most;
    s.slices = s.slices < 1 ? 1 : s.slices;
    s.slice_kb = s.kb;
    s.helpers = 0;
    const int left = s.workers - s.tiles * s.slices;
    if (left > 0 && s.workers / s.tiles == s.slices) {
        // a helper's range crosses at most `more` borders between tiles: its parts and the tiles' workers are done at the same time
        const HelpCost c = s.pair ? kHelpPair : kHelpLone;
        const long long more = (s.tiles + left - 1) / left;
        const long long share = ((long long)s.kb * s.tiles + more * c.part * left + s.workers - 1) / s.workers;
        if (share + c.least + (s.slices == 1 ? c.sum : 0) <= (s.kb + s.slices - 1) / s.slices) {
            s.helpers = left;
            s.slice_kb = (int)share;
        }
    }
    return s;
}

// The k-blocks [k0, k0 + n) of a tile, one after another for a worker; slot: where their sum goes.
struct Part {
    int tile, k0, n, slot;
};
// i-th part of worker w; false behind its last one.  S: a Split, or what has its fields.
template <typename S>
__host__ __device__ __forceinline__ bool part_at(const S &P, int w, int i, Part &p)
{
    const int mains = P.tiles * P.slices;
    if (w < mains || !P.helpers) {
        const int m = w + i * P.workers;
        if (m >= mains || (P.helpers && i > 0)) return false;
        const int slice = m / P.tiles;
        p.tile = m - slice * P.tiles;
        if (P.helpers) { p.k0 = slice * P.slice_kb; p.n = P.slice_kb; }
        else {
            p.k0 = (int)((long long)slice * P.kb / P.slices);
            p.n = (int)((long long)(slice + 1) * P.kb / P.slices) - p.k0;
        }
        p.slot = p.tile * P.slices + slice;
        return true;
    }
    const int h = w - mains, base = P.slices * P.slice_kb, rest = P.kb - base;
    const long long units = (long long)P.tiles * rest, u1 = (long long)(h + 1) * units / P.helpers;
    long long u = (long long)h * units / P.helpers;
    u = i == 0 ? u : (u / rest + i) * rest;                          // (a tile after the first begins at its first block)
    if (u >= u1) return false;
    p.tile = (int)(u / rest);
    const int in = (int)(u - (long long)p.tile * rest);
    p.k0 = base + in;
    p.n = (int)(rest - in < u1 - u ? rest - in : u1 - u);
    p.slot = mains + h + p.tile;
    return true;
}

}  // namespace im
