// The experts' factors: how a call is cut, rows brought to 16-byte addresses, and the second pass over experts of several ranges.
#include <algorithm>
#include <cmath>

#include "factor_cut.h"
#include "factor_expert.h"
#include "factor_reduce.h"
#include "rows16.h"

namespace kfac {

// Rows that do not begin at 16-byte addresses, copied with zeros behind them; only those that belong to an expert.
template <int ES>
__global__ __launch_bounds__(256) void expert_pad_kernel(const char* x, const int* offsets, int experts, int rows, int dim, long long ld,
                                                         unsigned per_row, unsigned vectors, char* out) {
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= vectors) return;
    const unsigned row = i / per_row, c = i - row * per_row;
    if (row >= (unsigned)min(max(offsets[experts], 0), rows)) return;
    *(KFAC_AS1 u4*)((gchar*)out + (size_t)i * 16) = load_row16<ES>((const gchar*)x + row * ld + c * 16ll, dim - (int)c * (16 / ES));
}

// The parts (as factor_tile_reduce_kernel's workgroups take them) of the experts of several ranges, dealt to the launch's workgroups in runs: how
// many there are is known here only.  (A workgroup for every part that there could be: 131,072 rows of 1,024 columns for 128 experts 185 us.)
template <int GROUPS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4, 8))) void expert_reduce_kernel(ExpertArgs a, int per) {
    __shared__ __attribute__((aligned(16))) float lds[GROUPS == 1 ? 32 * 33 : RD_MANY_FLOATS];
    ExpertRange r;
    unsigned unit = 0, last = 0;
    int j = 0;
    bool there = expert_range<true>(a, [&](int all, auto&&, auto&&) {
        const unsigned units = (unsigned)all * (unsigned)per, each = units / gridDim.x, more = units - each * gridDim.x;
        unit = blockIdx.x * each + min(blockIdx.x, more);
        last = unit + each + (blockIdx.x < more);
        j = (int)(unit / (unsigned)per);
        return unit < last ? j : -1;
    }, r);
    for (unsigned in = unit - (unsigned)j * (unsigned)per; unit < last; ++unit, ++in) {
        if (in == (unsigned)per) {
            in = 0;
            ++j;
            there = expert_range<true>(a, [&](int, auto&&, auto&&) { return j; }, r);
        }
        if (there) {
            FactorPlan pl;
            pl.tw = a.tw;
            pl.tiles_dim = a.tiles_dim;
            pl.ntiles = a.ntiles;
            pl.nsplit = r.ranges;
            pl.rows_per_split = a.rows_per;
            pl.tile_floats = a.tile_floats;
            pl.ws_bytes = 0;
            Partial part;
            part.tiles = as_global(a.tiles) + (size_t)r.part * a.ntiles * a.tile_floats;
            part.sums = as_global(a.sums) + (size_t)r.part * (a.tiles_dim * a.tw);
            reduce_partials<GROUPS>(expert_view(a, r.rows, r.rows), pl, part, expert_out(a, r.expert), expert_scale(a, r.rows), (int)in, lds);
        }
        __syncthreads();                                               // (the next part's sums go where these were)
    }
}

constexpr int EXPERT_MAX = 1024, REDUCE_WGS = 2048;
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

using namespace kfac;

extern "C" size_t kfac_expert_factor_workspace_bytes(const kfac_expert_factor_desc* desc) {
    if (!expert_factor_ok(desc)) return 0;
    const ExpertCut c = expert_cut(*desc);
    return c.pad_bytes + c.tile_bytes + c.sum_bytes;
}

extern "C" int kfac_expert_factor(const kfac_expert_factor_desc* desc, const void* x, const int32_t* offsets, float scale, float* out,
                                  float* running, float decay, void* ws, size_t ws_bytes, void* stream) {
    if (!expert_factor_ok(desc)) return KFAC_ERR_INVALID_ARG;
    const kfac_expert_factor_desc& d = *desc;
    const bool f32 = d.dtype == KFAC_F32;
    const int es = f32 ? 4 : 2;
    if (!offsets || (uintptr_t)offsets % 4 || (!out == !running)) return KFAC_ERR_INVALID_ARG;
    if (running && (d.packed || !(decay >= 0.f && decay <= 1.f))) return KFAC_ERR_INVALID_ARG;
    float* dst = out ? out : running;
    if ((uintptr_t)dst % 4) return KFAC_ERR_INVALID_ARG;
    const ExpertCut c = expert_cut(d);
    if (d.rows > 0 && (!x || (uintptr_t)x % (c.pad ? es : 16))) return KFAC_ERR_INVALID_ARG;
    const size_t need = kfac_expert_factor_workspace_bytes(desc);
    if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)) return KFAC_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    ExpertArgs a;
    a.x = c.pad ? ws : x;
    a.offsets = offsets;
    a.dst = dst;
    a.tiles = (float*)((char*)ws + c.pad_bytes);
    a.sums = (float*)((char*)ws + c.pad_bytes + c.tile_bytes);
    a.dout = d.dim + d.has_bias;
    a.result = d.packed ? (size_t)a.dout * (a.dout + 1) / 2 : (size_t)a.dout * a.dout;
    a.rows = d.rows;
    a.experts = d.experts;
    a.dim = d.dim;
    a.ld = c.ld;
    a.dtype = d.dtype;
    a.mode = running ? OUT_EMA : d.packed ? OUT_PACKED : OUT_PLAIN;
    a.scale = scale;
    a.decay = decay;
    a.rows_per = c.rows_per;
    a.tw = c.tw;
    a.tiles_dim = c.tiles_dim;
    a.ntiles = c.ntiles;
    a.tile_floats = c.tile_floats;
    a.ranges = (int)c.ranges;
    a.parts = (int)c.parts;
    a.streams = a.mode != OUT_PACKED && a.dout % 16 == 0 && (uintptr_t)dst % 64 == 0 && a.result * sizeof(float) * d.experts > EXPERT_STREAM;
    // Where the tiles may fill half the chip, an XCD gets an eighth of their work and not of their number (bf16, us, by number and by work: 16,384 rows, 32
    // experts of 768 columns, equal and of softmax(1.5 z) of the rows, 34 and 35, 54 and 47; 32 of 512 22 and 22, 28 and 26; 20,000 rows, 40 of 256 11.9 and 12.3).
    const long long most = c.ranges * c.ntiles;
    const float beside = c.tw == 256 ? 500.f : f32 ? 100.f : 300.f;
    const bool by_work = most > (c.tw == 256 ? 256 : f32 ? 512 : 768) / 2 && d.rows >= 0.5f * beside * c.ranges;   // (of few rows units are alike)
    a.beside = by_work ? beside : 0.f;
    const long long wgs = (most + 7) / 8 * 8;
    // (Four workgroups to a part, which share out its rows and its sums, where there are many ranges to an expert and few parts: 64 columns, 4 experts
    // of 16 ranges 15.0 -> 13.4 us, 192 columns, 2 of 10 16.5 -> 14.9; 256 columns, 8 of 8, 384 parts, 23.8 and 26.8.)
    const int groups = d.rows / d.experts >= 4 * c.rows_per && (long long)d.experts * c.ntiles * (c.tw / 32) * (c.tw / 32) <= 256 ? 4 : 1;
    const long long wgs_per = (long long)c.ntiles * (c.tw / 32) * (c.tw / 32) * groups + (d.has_bias ? ceil_div(d.dim, 256) : 0);
    const long long reduce_wgs = std::min(c.splits * wgs_per, (long long)REDUCE_WGS);
    const int V = f32 ? 4 : 8;
    const long long vectors = c.pad ? (long long)d.rows * (c.ld / V) : 0;
    // (a launch has fewer than 2^32 threads)
    if (wgs * (c.tw == 256 ? 512 : 256) >= 1ll << 32 || c.splits * wgs_per >= 1ll << 32 || vectors > 0x7fffffffll) return KFAC_ERR_TOO_LARGE;
    if (vectors) {
        const dim3 grid((unsigned)((vectors + 255) / 256));
        const long long ld = (d.ld ? d.ld : d.dim) * es;
        if (f32) KFAC_LAUNCH(expert_pad_kernel<4>, grid, dim3(256), st, (const char*)x, offsets, d.experts, d.rows, d.dim, ld, (unsigned)(c.ld / V),
                             (unsigned)vectors, (char*)ws);
        else KFAC_LAUNCH(expert_pad_kernel<2>, grid, dim3(256), st, (const char*)x, offsets, d.experts, d.rows, d.dim, ld, (unsigned)(c.ld / V),
                         (unsigned)vectors, (char*)ws);
    }
    const int rc = d.dtype == KFAC_BF16 ? launch_expert_tiles<0>(a, (unsigned)wgs, st)
                 : d.dtype == KFAC_F16 ? launch_expert_tiles<1>(a, (unsigned)wgs, st)
                                       : launch_expert_tiles<2>(a, (unsigned)wgs, st);
    if (rc != KFAC_OK) return rc;
    if (reduce_wgs) {
        if (groups == 4) KFAC_LAUNCH(expert_reduce_kernel<4>, dim3((unsigned)reduce_wgs), dim3(256), st, a, (int)wgs_per);
        else KFAC_LAUNCH(expert_reduce_kernel<1>, dim3((unsigned)reduce_wgs), dim3(256), st, a, (int)wgs_per);
    }
    return KFAC_OK;
}
