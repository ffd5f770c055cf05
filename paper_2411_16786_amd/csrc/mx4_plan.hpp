// Which kernel and tile the 4-bit expert FFN takes (mx4_ffn.hip), from sizes that the host knows: plain C++.
#pragma once
#include "ffn_plan.hpp"

namespace dicemoe {

constexpr int kLdsBytes = 160 * 1024;

// most row tiles of BM rows that a table of n segments with max_rows rows can have (one at least: a block reports the row count)
inline long long tile_bound(int max_rows, int n_seg, int BM)
{
    const long long most = static_cast<long long>(max_rows) / BM + n_seg;       // every segment may end in a part of a tile
    const long long tiles = most < max_rows ? most : max_rows;              // ... and a tile has a row at least
    return tiles > 1 ? tiles : 1;
}

// The tiles of mx4_tile_kernel: rows, columns, shares of the reduction; the first four are weighed against each other, the others take the place of
// one of them where few tiles leave compute units empty
struct TileSize { int rows, columns, shares; };
constexpr int kTiles = 6, kFewTile = 3;
constexpr TileSize kTile[kTiles] = {{128, 256, 1}, {128, 128, 1}, {64, 128, 1}, {32, 128, 2}, {32, 64, 4}, {64, 128, 2}};

// Scales by chunks where all of them at once would leave less than three workgroups per compute unit: 4608 -> 1152 with 256 x 128
// tiles 103 us instead of 113 and with 128 x 128 92 instead of 103, but with 128 x 64, where they leave three, 104 instead of 93
constexpr int tile_lds(int tile, int K, bool chunks)
{
    const TileSize t = kTile[tile];
    const int unit = 32 * t.columns * t.shares;                  // a workgroup's 16-byte loads
    return t.shares * (2 * t.rows * 128 + 2 * t.columns * 64 + (chunks ? 2 * t.columns * 16 : 0)) + (chunks ? 0 : (t.columns / 32 * K + unit - 1) / unit * unit);
}
inline bool tile_chunks(int tile, int K) { return K % 512 == 0 && 3 * tile_lds(tile, K, false) > kLdsBytes; }

// Tiles of BM rows x BN columns, a segment's last row tile half full on average
inline long long tile_count(int max_rows, int n_seg, int BM, int BN, int columns)
{
    const long long row_tiles = (max_rows + n_seg * BM / 2) / BM;
    return (row_tiles > n_seg ? row_tiles : n_seg) * ((columns + BN - 1) / BN);
}
// ... and by area what the compute unit with the most of them has to do
inline float tile_cost(long long tiles, int BM, int BN) { return static_cast<float>((tiles + kComputeUnits - 1) / kComputeUnits) * (BM * BN); }

// Columns per wavefront set of mx4_rows_kernel: 16 while that gives each compute unit no more than six workgroups (4608 -> 1152, one token
// 6.0 us against 9.6 with 32, eight tokens 9.1 and 10.0), else 32 (1152 -> 4608, eight tokens 9.2 against 11.6)
inline bool rows_narrow(int max_rows, int n_seg, int N) { return tile_bound(max_rows, n_seg, 16) * (N / 16) <= 6 * kComputeUnits; }

// Float rows, which have no tiles: 64 columns and four shares instead of eight where that leaves each compute unit more than four
// workgroups (1000 rows over 16 experts, 384 -> 1536 24 us against 31; 2000 over 8, 4608 -> 1152 224 against 252; with 468 workgroups,
// 300 rows over 8, 4608 -> 1152 57 against 55)
inline bool rows_wide(int max_rows, int n_seg, int N) { return tile_bound(max_rows, n_seg, 16) * ((N + 63) / 64) > 4 * kComputeUnits; }

// Tile of a product of many rows, -1: rows in sixteens (mx4_rows_kernel), which up to four rows a segment is faster while it has at
// most 12 workgroups per compute unit (eight tokens at the DiT-MoE-XL widths 9.2 and 9.1 us against 11.5 and 13.0; 26 rows over 16
// experts, 2048 -> 8192, 27.8 against 22.6).  Among the tiles that with their scales fit the LDS the cheapest by area, at the
// rates of 8192 -> 4096 of 8192 rows (444, 481 and 563 us; the tiles of 32 rows are for few rows); a compute unit with a single workgroup
// of four wavefronts waits more.  Of the two of 32 rows, in shares, the narrower one in more shares while each tile has a compute unit
// to itself (200 rows over 8 experts: 4608 -> 1152 13.4 us against 21.8, 1152 -> 4608, 288 tiles, 16.6 against 12.6).
// The factors 1.3 (that single workgroup) and 2.5 (tiles of 32 rows) over both products of 100 to 8192 rows, 1152 -> 4608 over 8 experts,
// 384 -> 1536 and 2048 -> 8192 over 16: the tile taken is 2.2 % above the fastest on average.  1 in place of 1.3: 3.1 % (2000 rows, 4608 -> 1152 44
// us against 35; 8192 rows, 1536 -> 384 18.6 against 16.3; the other way 1000 rows, 8192 -> 2048 76 against 85).  1.8 in place of 2.5: 2.6 % (400
// rows, 2048 -> 8192 53 against 44), 3: 3.0 % (200 rows, 1152 -> 4608 14.0 against 12.0); 2.1, which is their rate, takes the same tiles.
// Tiles of 64 rows in two shares while there are no more than 5/4 per compute unit (4608 -> 1152 over 8 experts, 1000 rows 29 us against
// 35.5, 2000 rows, 315 tiles, 39 both; 300 rows over 16 experts, 8192 -> 2048, 53 against 62.5).
inline int pick_tile(int max_rows, int n_seg, int N, int K)
{
    if (max_rows <= 4 * n_seg && tile_bound(max_rows, n_seg, 16) * (N / 32) <= 12 * kComputeUnits) return -1;
    constexpr float slow[kFewTile + 1] = {1.0f, 1.08f, 1.27f, 2.5f};
    int best = -1;
    float least = 0.f;
    for (int i = 0; i <= kFewTile; ++i) {
        if (tile_lds(i, K, tile_chunks(i, K)) > kLdsBytes) continue;
        const long long tiles = tile_count(max_rows, n_seg, kTile[i].rows, kTile[i].columns, N);
        float cost = slow[i] * tile_cost(tiles, kTile[i].rows, kTile[i].columns);
        if (tiles <= kComputeUnits && kTile[i].columns * kTile[i].shares == 128) cost *= 1.3f;
        if (best < 0 || cost < least) { best = i; least = cost; }
    }
    if (best == 2 && 4 * tile_count(max_rows, n_seg, kTile[best].rows, kTile[best].columns, N) <= 5 * kComputeUnits && tile_lds(5, K, tile_chunks(5, K)) <= kLdsBytes) return 5;
    if (best == kFewTile && tile_count(max_rows, n_seg, kTile[best].rows, kTile[best].columns, N) <= kComputeUnits &&
        tile_lds(kFewTile + 1, K, tile_chunks(kFewTile + 1, K)) <= kLdsBytes)
        ++best;
    return best;
}

// The same for mx4_tile_transposed_kernel (32 RT rows x 64 WN columns of K; its LDS does not depend on the reduction).  4608 -> 1152, 8192
// rows 64 x 256 tiles 100 us, 32 x 128 in two shares 129; 2000 rows 57 and 43, in four shares 48; 400 rows 56, 30 and 23, 1000 rows (315
// tiles, 320 being 5/4 per compute unit) two shares 33, four 27.  1152 -> 4608, 2000 rows 38 and 54, 400 rows 24, 20 and in four shares 31.  Rows in sixteens, two rows a segment: 11.6 us against 14.9 in four shares.
// 1.3 as above, and 1.6 by which a 32-row tile takes longer by area: over the same products the tile taken is 2.0 % above the fastest; 1 in
// place of 1.3 4.0 % (2000 rows, 4608 -> 1152 57 us against 43), 1.3 in place of 1.6 3.8 % (4000 rows, 8192 -> 2048 243 against 180), 2 3.8 %
// (1000 rows, 8192 -> 2048 131 against 93).
constexpr int kTilesT = 3;
constexpr TileSize kTileT[kTilesT] = {{64, 256, 1}, {32, 128, 2}, {32, 128, 4}};
inline int pick_tile_t(int max_rows, int n_seg, int K)
{
    constexpr TileSize large_tile = kTileT[0], small_tile = kTileT[1];
    if (max_rows <= 4 * n_seg && tile_bound(max_rows, n_seg, 16) * (K / 128) <= 12 * kComputeUnits) return -1;
    const long long large = tile_count(max_rows, n_seg, large_tile.rows, large_tile.columns, K), small = tile_count(max_rows, n_seg, small_tile.rows, small_tile.columns, K);
    if (tile_cost(large, large_tile.rows, large_tile.columns) * (large <= kComputeUnits ? 1.3f : 1.0f) <= 1.6f * tile_cost(small, small_tile.rows, small_tile.columns)) return 0;
    return 4 * small <= 5 * kComputeUnits ? 2 : 1;
}

}  // namespace dicemoe
