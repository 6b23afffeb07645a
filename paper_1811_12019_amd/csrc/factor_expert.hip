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

// One workgroup to a part of an expert of several ranges, as factor_tile_reduce_kernel's to a build's.
template <int GROUPS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4, 8))) void expert_reduce_kernel(ExpertArgs a, int wgs_per) {
    __shared__ __attribute__((aligned(16))) float lds[GROUPS == 1 ? 32 * 33 : RD_MANY_FLOATS];
    const int j = blockIdx.x / wgs_per, local = blockIdx.x - j * wgs_per;
    ExpertRange r;
    if (!expert_range<true>(a, (int*)lds, [&](int) { return j; }, r)) return;
    __syncthreads();                                                   // (the sums go where the range was found)
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
    reduce_partials<GROUPS>(expert_view(a, r.rows, r.rows), pl, part, expert_out(a, r.expert), expert_scale(a, r.rows), local, lds);
}

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

static ExpertCut expert_cut(const kfac_expert_factor_desc& d) {
    ExpertCut c;
    const bool f32 = d.dtype == KFAC_F32;
    const int V = f32 ? 4 : 8;
    const long long ld = d.ld ? d.ld : d.dim;
    c.pad = ld % V != 0 || ld > EXPERT_LD_MAX;
    c.ld = c.pad ? (d.dim + V - 1) / V * V : (int)ld;
    c.pad_bytes = c.pad ? align_up((size_t)d.rows * c.ld * (f32 ? 4 : 2), 256) : 0;
    // The work as a call of the other builders counts it, with equal experts (factor_cut.h).
    TileWork w;
    const double n = ceil_div(d.dim, 128), m = ceil_div(d.dim, 256), rows = d.rows;
    w.narrow = 0.5 * n * (n + 1) * rows;
    w.wide = d.dim <= 128 ? w.narrow : 2.0 * m * (m + 1) * rows;
    c.rows_per = (rows_of(w, f32) + 63) / 64 * 64;
    if (d.dim > 128) {
        w.over = w.narrow;
        w.area = 256.0 * m * 256.0 * m * rows;
        w.filled = (double)d.dim * d.dim * rows;
        const double tiles = 0.5 * m * (m + 1), each = rows / d.experts;
        w.wide_rows = tiles * rows;
        w.wide_wgs = (int)std::min(1e9, tiles * d.experts * std::max(1.0, std::ceil(each / c.rows_per)));
    }
    c.tw = d.dim <= 64 ? 64 : d.dim <= 128 || f32 || !takes_wide(w, c.rows_per) ? 128 : 256;
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
    const long long wgs = (c.ranges * c.ntiles + 7) / 8 * 8;
    const int groups = ceil_div(d.rows, c.rows_per) >= MANY_SPLITS ? 4 : 1;
    const int wgs_per = c.ntiles * (c.tw / 32) * (c.tw / 32) * groups + (d.has_bias ? ceil_div(d.dim, 256) : 0);
    const long long reduce_wgs = c.splits * wgs_per;
    const int V = f32 ? 4 : 8;
    const long long vectors = c.pad ? (long long)d.rows * (c.ld / V) : 0;
    // (a launch has fewer than 2^32 threads)
    if (wgs * (c.tw == 256 ? 512 : 256) >= 1ll << 32 || reduce_wgs * 256 >= 1ll << 32 || vectors > 0x7fffffffll) return KFAC_ERR_TOO_LARGE;
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
        if (groups == 4) KFAC_LAUNCH(expert_reduce_kernel<4>, dim3((unsigned)reduce_wgs), dim3(256), st, a, wgs_per);
        else KFAC_LAUNCH(expert_reduce_kernel<1>, dim3((unsigned)reduce_wgs), dim3(256), st, a, wgs_per);
    }
    return KFAC_OK;
}
