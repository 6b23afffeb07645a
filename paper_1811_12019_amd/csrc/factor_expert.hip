// The experts' factors: the calls, rows brought to 16-byte addresses, and the second pass over experts of several ranges.
#include <algorithm>

#include "expert_cut.h"
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

constexpr int REDUCE_WGS = 2048;

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
