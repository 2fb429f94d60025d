// How the paged decode deals its work out: arithmetic shared by the kernel and its host-side replay.
//
// The work is a line of tiles of kDecodeTile tokens: request after request, within a request K/V head after K/V head
// (and block of 16 query heads after block), within those tile after tile.  CTA c of n takes tiles [total c / n, total (c + 1) / n): shares
// equal to a tile whatever the lengths are.  A request's tiles of one head that lie within one share make a complete
// result; those that a share's border cuts are joined afterwards from the parts of the CTAs involved.
// A CTA has at most two cut pieces: one that goes on from the CTA before (workspace entry 2 c), and one that starts in its share
// and goes on in the next (entry 2 c + 1); of these at most one starts in any CTA, so the CTA's number names the join.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SAW_DECODE_HD __host__ __device__ __forceinline__
#else
#define SAW_DECODE_HD inline
#endif

namespace sawtooth {

constexpr int kDecodeTile = 64;       // tokens of a tile
constexpr int kDecodeRows = 16;       // query heads of a block
constexpr int kDecodeMinTiles = 2;    // a share is at least this long, so that joining stays cheaper than reading

SAW_DECODE_HD int decode_tiles(int len) { return (int)(((unsigned)len + kDecodeTile - 1) / kDecodeTile); }

// CTAs that get work, of a grid of `grid`.
SAW_DECODE_HD int decode_ctas(uint64_t total, int grid) {
    const uint64_t most = (total + kDecodeMinTiles - 1) / kDecodeMinTiles;
    return most < (uint64_t)grid ? (int)most : grid;
}
SAW_DECODE_HD uint64_t decode_share_begin(uint64_t total, int ctas, int cta) { return total * (uint64_t)cta / (uint64_t)ctas; }
// The CTA whose share holds tile x: the largest c with total c / ctas <= x.
SAW_DECODE_HD int decode_cta_of(uint64_t total, int ctas, uint64_t x) { return (int)(((x + 1) * (uint64_t)ctas - 1) / total); }

}  // namespace sawtooth
