// How the experts' factors of a call are cut, on the host: rows of a range, width of the tiles, and the scratch for the most ranges that the
// offsets, which only the device knows, can make.
#pragma once

#include <algorithm>
#include <cmath>

#include "factor_cut.h"

namespace kfac {

constexpr int EXPERT_MAX = 1024;
constexpr long long EXPERT_LD_MAX = 1 << 18;   // elements: a range's bytes fit 32 bits

struct ExpertCut {
    int rows_per, tw, tiles_dim, ntiles, tile_floats;
    long long ranges, parts, splits;   // the most ranges, partial sums, and experts of several ranges there can be
    bool pad;                          // rows are copied
    int ld;                            // of what the tiles read
    size_t pad_bytes, tile_bytes, sum_bytes;
};

static bool expert_factor_ok(const kfac_expert_factor_desc* d) {
    return d && d->rows >= 0 && d->experts >= 1 && d->experts <= EXPERT_MAX && d->dim >= 1 && d->dim <= 32766 &&
           (d->dtype == KFAC_F32 || d->dtype == KFAC_BF16 || d->dtype == KFAC_F16) && (d->has_bias == 0 || d->has_bias == 1) &&
           (d->packed == 0 || d->packed == 1) && (d->ld == 0 || (d->ld >= d->dim && d->ld <= (1ll << 28)));
}

// Width of the tiles and rows of a range, from the call's rows and experts of equal size.  Rows: as many as let all ranges run in as few rounds of the
// workgroups that fit the chip (768, of 256-wide tiles 256, fp32 512 and one round more) as uncut experts would, counting half a range for every expert's
// end, and not so few that a second range costs a tile more in partial sums than it saves; ranges near an average expert's rows are made longer, so that
// most experts are one (three times as long where there are workgroups enough to even out the long ones: bf16, us, three and one and a half times, 32 experts of
// 1,024 rows, 1,024 columns and softmax(z) 79 and 94, 128 of 512 and 512 columns 59 and 69; 32 of 2,048, 512 columns, uncut and cut 45 and 57; fp32, ranges of 1.25
// times an average expert's rows and of 512: 71 experts of 572 rows, 624 columns 158 and 229, of softmax(0.8 z) 178 and 182; 40 of 700, 768 columns 152 and 205, of
// softmax(0.3 z) 166 and 182, of softmax(0.8 z) 172 and 170; 64 of 781, 512 columns 130 and 159, 149 and 160, 162 and 150); calls of few rows need no second launch
// (fp32, us, with one and with two: 18 experts' 1,187 rows of 59 columns 11.3 and 14.9, 9 experts' 1,045 of 114 13.3 and 15.4, 5 experts' 1,240 of 32 13.2 and 11.7).
// Width: 64 where wider tiles would leave CUs without one or cover much more than the matrix, 256 where there are many tiles of many rows, so that a
// workgroup outlasts its epilogue, with little padding.  Both sides, us:
//     128- and 256-wide, bf16, equal experts, then softmax(0.5 z) of the rows: 512 columns, 32 experts of 4,096 rows 84 and 84, 85 and 88; 64 of 2,048 75 and 60,
//     85 and 78; 1,024 columns, 8 of 4,096 74 and 60, 75 and 74; 32 of 1,024 62 and 70, 88 and 82; 64 of 512 72 and 86, 75 and 82; 2,048 columns, 8 of 1,024
//     63 and 75, 69 and 75; 8 of 2,048 100 and 109, 106 and 109; 32 of 1,024 197 and 196, 267 and 218; 64 of 512 278 and 263, 370 and 301; 32 of 2,048 411 and 319
//     64- and 128-wide: bf16, 512 columns, 8 experts of 64 rows 6.5 and 8.1; of 256 7.8 and 9.2; 32 of 64 12.8 and 11.8; fp32, 256 columns, 8 of 256 12 and 24; 8 of
//     2,048 28 and 27; 30 of 1,000 rows, 192 columns 30 and 39, 256 42 and 42, 320 53 and 59; 80 of 132 rows, 329 columns 43 and 37
// Rows of a range: 1,024 columns, 256 wide, 32 of 4,096 1,024 303, 2,048 256, 6,400 184; 8 of 4,096 81, 70, 85; 512 columns, 128 wide, 8 of 4,096
// 1,024 31, 1,536 26; fp32, 1,024 columns, 8 of 1,024 256 105, 512 109, 1,024 124; 512 columns, 64 of 1,024 512 198, 1,024 195, 1,600 164.
// Results in rows of whole halves of cache lines go past the caches where two of them do not stay in the 256 MB memory-side one (smaller parts of lines
// written past them cost as much again: 8,192 rows of 64 experts, 1,000 columns 96 and 119, 1,025 109 and 154; 88 experts' 1,233 206 and 318).  bf16, us, kept and
// past them: 8,192 rows, 64 experts of 1,024 columns (256 MB) 64 and 56, of 1,008 90 and 63, as running averages 118 and 91; 32 of 1,008 (124 MB) 57 and 39,
// 67 and 57; 56 of 736 (116 MB) 26.7 and 29.7, 34.6 and 42.5; 16 of 2,000 columns, 16,384 rows 168 and 118, 179 and 148; fp32, 64 of 816 78 and 56, 82 and 76.
constexpr size_t EXPERT_STREAM = (size_t)120 << 20;
constexpr double FEW_WGS = 160, WIDE_TILE_ROWS = 150000, WIDE_WORK = 6e8;      // (rows of all tiles; times an expert's rows)

static ExpertCut expert_cut(const kfac_expert_factor_desc& d) {
    ExpertCut c;
    const bool f32 = d.dtype == KFAC_F32;
    const int V = f32 ? 4 : 8;
    const long long ld = d.ld ? d.ld : d.dim;
    c.pad = ld % V != 0 || ld > EXPERT_LD_MAX;
    c.ld = c.pad ? (d.dim + V - 1) / V * V : (int)ld;
    c.pad_bytes = c.pad ? align_up((size_t)d.rows * c.ld * (f32 ? 4 : 2), 256) : 0;
    const double rows = d.rows, each = rows / d.experts;
    auto tiles = [&](int tw) { const double n = ceil_div(d.dim, tw); return 0.5 * n * (n + 1); };
    auto rows_of_width = [&](int tw) {
        const double slots = tw == 256 ? 256 : f32 ? 512 : 768, whole = tiles(tw) * d.experts, rounds = std::max(std::ceil(whole / slots), 1.0) + f32;
        double r = std::max(rows * tiles(tw) / (0.95 * rounds * slots - 0.5 * whole), !f32 ? 1024.0 : whole < slots ? 256.0 : 512.0);
        const bool many = whole >= (tw == 256 ? 1.5 : 0.75) * slots;
        if (r >= (whole >= 0.25 * slots ? 0.5 : 0.6) * each && (!f32 || many)) r = std::max(r, (f32 ? 1.25 : many ? 3 : 1.5) * each);
        if (rows <= (f32 ? ROWS_PER_WG_MAX_F32 : 2048) && (tw == 64 || !f32)) r = std::max(r, rows);
        return (int)(std::min(r, (double)(f32 ? ROWS_PER_WG_MAX_F32 : ROWS_PER_WG_MAX)) + 63) / 64 * 64;
    };
    c.tw = 128;
    const double fit = 0.25 * tiles(64) / tiles(128);
    if (d.dim <= 64 || fit <= (f32 ? 0.7 : 0.55) || tiles(128) * d.experts * std::max(1.0, std::ceil(each / rows_of_width(128))) < FEW_WGS) c.tw = 64;
    else if (!f32 && d.dim > 128 && 4 * tiles(256) <= WIDE_PADDING * tiles(128) && tiles(256) * rows >= WIDE_TILE_ROWS &&
             tiles(256) * rows * each >= WIDE_WORK) c.tw = 256;
    c.rows_per = rows_of_width(c.tw);
    c.tiles_dim = ceil_div(d.dim, c.tw);
    c.ntiles = c.tiles_dim * (c.tiles_dim + 1) / 2;
    c.tile_floats = tile_floats(c.tw, c.ntiles);
    // n ranges need more than (n - 1) rows_per rows
    c.ranges = (long long)d.rows / c.rows_per + d.experts;
    c.splits = std::min((long long)d.experts, (long long)d.rows / (c.rows_per + 1));
    c.parts = c.splits ? std::min(2ll * d.rows / c.rows_per, (long long)d.rows / c.rows_per + c.splits) : 0;
    c.tile_bytes = align_up((size_t)c.parts * c.ntiles * c.tile_floats * sizeof(float), 256);
    c.sum_bytes = d.has_bias ? align_up((size_t)c.parts * c.tiles_dim * c.tw * sizeof(float), 256) : 0;
    return c;
}

}  // namespace kfac
