// The experts' factors: tiles of X_e^T X_e, X_e the rows of expert e, whose bounds lie on the device.  Tile products and epilogues are the matrix-core
// builder's (factor_tile.h).
//
// Cut.  Rows of an expert are cut into ranges of rows_per, which the host chooses from the rows of all experts; how many ranges there are is
// known on the device only.  A launch has workgroups for the most there can be: rows / rows_per whole ones and a part for every expert, times
// the tiles.  Every wavefront reads the offsets, adds up the ranges before each expert's (one scan in registers) and finds its own; those behind
// the last range end.  Ranges of all experts, tiles inside a range, are one work list, of which every XCD gets a contiguous part, so that the tiles of a
// range, which read the same rows, share an L2 (tiles of 2, 4 and 8 ranges in turns: 387 -> 502, 634 and 534 us): an eighth of the units, or, where they are
// not few, of the work (equal numbers of experts of unequal rows left XCDs waiting: 65,536 rows of 2,048 columns, 32 experts of softmax(0.5 z) and
// softmax(2 z) of them, 375 -> 341 and 574 -> 409 us; of equal experts 330 and 337), the longest ranges first, so that none begins when the others end (343 -> 324
// and 413 -> 389, of equal experts 342 and 339; 64 of 1,024 columns and softmax(z) of the rows 138 -> 122).  Workgroups are as many as there can be units
// in all, an eighth of them on every XCD; those that find none of their XCD's take what another has more (twice as many workgroups, of which most found
// nothing, took 8 to 12 us of 340).
// An expert of one range goes straight to its destination; the others' partial sums are added up by a second launch, which there is if
// an expert can have more than rows_per rows at all.
// Addresses.  A workgroup takes its range's first row for the tensor's beginning and its last one for the end: offsets inside it fit 32 bits
// however long x is, and no row of another expert can be read.
#pragma once

#include "common.h"
#include "factor_batch.h"

namespace kfac {

struct ExpertArgs {
    const void* x;           // rows at 16-byte addresses
    const int* offsets;
    float* dst;              // the experts' results one after another
    float* tiles;            // partial sums: [part][ntiles][tile_floats]
    float* sums;             // column sums: [part][tiles_dim * tw]
    size_t result;           // floats of an expert's result
    int rows, experts, dim, dout, ld, dtype, mode;
    float scale, decay;
    int rows_per, tw, tiles_dim, ntiles, tile_floats;
    int ranges, parts;       // the most there can be
    int streams;             // results go past the caches
    float beside;            // what a tile costs beside its rows, in rows (0: units are dealt by number, not by work)
};

// What a workgroup works on.
struct ExpertRange {
    int expert, sub, ranges; // range `sub` of `ranges` of the expert
    int part;                // the expert's first partial sum, if it has several ranges
    int row, rows;           // the expert's rows
};

// Rows of expert e: offsets that lie outside or descend are cut off.
__device__ __forceinline__ void expert_rows(const ExpertArgs& a, int from, int to, int& row, int& rows) {
    const int r0 = min(max(from, 0), a.rows), r1 = min(max(to, r0), a.rows);
    row = r0;
    rows = r1 - r0;
}

// Sums of the lanes up to and with this one (unsigned or float): within rows of 16 lanes, then across them.
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
#define KFAC_SCAN_STEP(ctrl, rows) v += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, rows, 0xf, false))
    KFAC_SCAN_STEP(0x111, 0xf);        // row_shr 1, 2, 4, 8
    KFAC_SCAN_STEP(0x112, 0xf);
    KFAC_SCAN_STEP(0x114, 0xf);
    KFAC_SCAN_STEP(0x118, 0xf);
    KFAC_SCAN_STEP(0x142, 0xa);        // row_bcast 15: rows 0 and 2 to 1 and 3
    KFAC_SCAN_STEP(0x143, 0xc);        // row_bcast 31: rows 0 and 1 to 2 and 3
#undef KFAC_SCAN_STEP
    return v;
}

// Of the ranges of all experts (SPLIT: of the experts of several ranges) the one that `pick` names (-1: none).  False: none.
// Every wavefront works it out by itself, some experts to a lane: without LDS and barriers.  pick(all, units_before): the number of ranges, and a function that
// tells how many of their tiles lie before a fraction of all the work (experts' rows and `beside` for each range; a lane's experts count as alike), and
// one that gives number `at` of the tiles lo .. hi - 1 in the order of their ranges' rows, the longest first (by a lane's longest).
template <bool SPLIT, class Pick>
__device__ __forceinline__ bool expert_range(const ExpertArgs& a, Pick&& pick, ExpertRange& out) {
    const int lane = threadIdx.x & 63, per = (a.experts + 63) >> 6, e0 = lane * per, e1 = min(e0 + per, a.experts);
    const gint* o = as_global((int*)a.offsets);
    auto ranges_of = [&](int rows) -> unsigned {
        const unsigned n = ((unsigned)rows + a.rows_per - 1) / (unsigned)a.rows_per;
        return n == 0 && a.mode != OUT_EMA ? 1 : n;                    // (an average without rows stays as it is)
    };
    unsigned key = 0, part = 0;                                        // of this lane's experts
    int row = 0, rows = 0;                                             // of the last of them
    unsigned n = 0;
    int there_rows = 0, largest = 0;                                   // of this lane's ranges
    auto take = [&](int from, int to) {
        expert_rows(a, from, to, row, rows);
        n = ranges_of(rows);
    };
    int at = o[min(e0, a.experts)];
#pragma unroll 8
    for (int e = e0; e < e1; ++e) {
        const int next = o[e + 1];
        take(at, next);
        at = next;
        key += SPLIT ? (n > 1) : n;
        part += n > 1 ? n : 0;
        there_rows += rows;
        largest = max(largest, min(rows, a.rows_per));
    }
    unsigned k = wave_scan(key), p = wave_scan(part);
    unsigned all = (unsigned)__builtin_amdgcn_readlane((int)k, 63);
    if (all > (unsigned)a.ranges) all = (unsigned)a.ranges;            // (offsets that do not ascend could name more)
    auto units_before = [&](float fraction) -> unsigned {
        const float some = wave_scan((float)there_rows), total = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, some), 63));
        const float work = (float)there_rows + a.beside * (float)key;
        const float upto = some + a.beside * (float)k, goal = (total + a.beside * (float)all) * fraction;
        const unsigned long long beyond = __ballot(upto > goal);
        if (!beyond || fraction >= 1.f) return all * a.ntiles;
        const float inside = work > 0.f ? max(goal - (upto - work), 0.f) / work : 0.f;
        const unsigned tiles = key * a.ntiles, mine = (k - key) * a.ntiles + min((unsigned)(inside * (float)tiles), tiles);
        return min((unsigned)__builtin_amdgcn_readlane((int)mine, __builtin_amdgcn_readfirstlane(__ffsll(beyond) - 1)), all * a.ntiles);
    };
    auto by_size = [&](unsigned lo, unsigned hi, unsigned at) -> int {
        const unsigned begin = max((k - key) * a.ntiles, lo), end = min(k * a.ntiles, hi), here = end > begin ? end - begin : 0;   // this lane's of them
        unsigned before = 0;
        for (unsigned long long m = __ballot(here > 0); m; m &= m - 1) {
            const int other = __builtin_amdgcn_readfirstlane(__ffsll(m) - 1), size = __builtin_amdgcn_readlane(largest, other);
            const unsigned units = (unsigned)__builtin_amdgcn_readlane((int)here, other);
            before += (size > largest) | ((size == largest) & (other < lane)) ? units : 0;
        }
        const unsigned long long mine = __ballot((at >= before) & (at - before < here));
        return mine ? __builtin_amdgcn_readlane((int)(begin + at - before), __builtin_amdgcn_readfirstlane(__ffsll(mine) - 1)) : -1;
    };
    const int want = pick((int)all, units_before, by_size);            // (the same in all lanes)
    if (want < 0 || (unsigned)want >= all) return false;
    auto owner_of = [&]() { return __builtin_amdgcn_readfirstlane(__ffsll(__ballot((unsigned)want >= k - key && (unsigned)want < k)) - 1); };
    int owner = owner_of(), first = 0;
    if (per > 1) {                                                     // the owner's experts, one to a lane
        first = owner * per;
        const unsigned kb = (unsigned)__builtin_amdgcn_readlane((int)(k - key), owner), pb = (unsigned)__builtin_amdgcn_readlane((int)(p - part), owner);
        const int e = min(first + min(lane, per - 1), a.experts - 1);
        take(o[e], o[e + 1]);
        const bool own = lane < per && first + lane < a.experts;
        key = own ? (SPLIT ? (n > 1) : n) : 0;
        part = own && n > 1 ? n : 0;
        k = kb + wave_scan(key);
        p = pb + wave_scan(part);
        owner = owner_of();
    }
    out.expert = first + owner;
    out.sub = want - __builtin_amdgcn_readlane((int)(k - key), owner);
    out.ranges = __builtin_amdgcn_readlane((int)n, owner);
    out.part = __builtin_amdgcn_readlane((int)(p - part), owner);
    out.row = __builtin_amdgcn_readlane(row, owner);
    out.rows = __builtin_amdgcn_readlane(rows, owner);
    return out.ranges == 1 || (long long)out.part + out.ranges <= a.parts;
}

// `rows` rows, all of them an expert's or a range of its R rows, as the matrix-core builder sees them.
__host__ __device__ __forceinline__ View expert_view(const ExpertArgs& a, int rows, int R) {
    View v;
    Unfold& u = v.u;
    u.N = rows;
    u.C = v.run = a.ld;
    u.H = u.W = u.Ho = u.Wo = u.kh = u.kw = u.stride = 1;
    u.pad = 0;
    u.has_bias = a.dout > a.dim;
    u.layout = KFAC_NHWC;
    u.dtype = a.dtype;
    u.order = KFAC_ORDER_KH_KW_C;
    u.R = R;
    u.d = v.cout = a.dim;
    v.dout = a.dout;
    v.kw = 1;
    v.chunked = v.mapped = v.repack = v.rows = v.shared = v.planes = 0;
    return v;
}
__device__ __forceinline__ float expert_scale(const ExpertArgs& a, int rows) {
    return a.scale != 0.f ? a.scale : rows > 0 ? 1.f / (float)rows : 0.f;
}
__device__ __forceinline__ OutSpec expert_out(const ExpertArgs& a, int expert) {
    OutSpec o;
    o.dst = as_global(a.dst) + (size_t)expert * a.result;
    o.decay = a.decay;
    o.one_minus = 1.f - a.decay;
    o.mode = a.mode;
    return o;
}

// Zeros to a workgroup's share of an expert's result that has no rows: its floats share / shares .. (share + 1) / shares, in whole 16-byte vectors
// where they lie on the grid.  (By way of tiles of zeros, 88 experts of 1,233 columns with 5 rows 206 us.)
__device__ __forceinline__ void expert_zeros(gfloat* out, size_t count, int share, int shares) {
    const size_t lead = ((16 - ((uintptr_t)out & 15)) & 15) / 4, vectors = count > lead ? (count - lead) / 4 : 0;
    const size_t v0 = vectors * share / shares, v1 = vectors * (share + 1) / shares;
    const v4f zero = {0.f, 0.f, 0.f, 0.f};
    for (size_t v = v0 + threadIdx.x; v < v1; v += blockDim.x) *(KFAC_AS1 v4f*)(out + lead + 4 * v) = zero;
    if (share == 0) {                                                  // (up to three floats before and behind the vectors)
        if (threadIdx.x < min(lead, count)) out[threadIdx.x] = 0.f;
        const size_t end = lead + 4 * vectors;
        if (end + threadIdx.x < count) out[end + threadIdx.x] = 0.f;
    }
}

// (the tile kernel's launch bounds: factor_launch.h)
template <int TW, int KIND, bool STREAM>
__global__ __launch_bounds__((tile_threads<TW, KIND == 2 ? 4 : 2>())) __attribute__((amdgpu_waves_per_eu(TW == 256 || KIND == 2 ? 2 : 3, 8)))
void expert_tile_kernel(ExpertArgs a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    constexpr int ES = KIND == 2 ? 4 : 2;
    ExpertRange r;
    int tile = 0;
    const bool there = expert_range<false>(a, [&](int all, auto&& units_before, auto&& by_size) {
        int unit;
        if (a.beside > 0.f) {                                          // workgroups k, k + 8, ..: the eighth of the work that XCD k gets
            const int xcd = blockIdx.x & 7;
            const unsigned wgs = gridDim.x >> 3;                       // of an XCD
            unsigned lo = units_before(0.125f * xcd), hi = units_before(0.125f * (xcd + 1)), at = blockIdx.x >> 3;
            if (at >= hi - lo) {                                       // those without any take, in order, what is more than another XCD's workgroups
                unsigned more = at - (hi - lo);
                unsigned from = 0;
                for (int y = 0; y < xcd; ++y) {
                    const unsigned to = units_before(0.125f * (y + 1));
                    more += to - from < wgs ? wgs - (to - from) : 0;
                    from = to;
                }
                bool found = false;
                for (int y = 0; y < 8 && !found; ++y) {
                    lo = y ? hi : 0;
                    hi = units_before(0.125f * (y + 1));
                    const unsigned over = hi - lo > wgs ? hi - lo - wgs : 0;
                    found = more < over;
                    if (!found) more -= over;
                }
                if (!found) return -1;
                at = wgs + more;
            }
            unit = by_size(lo, hi, at);
            if (unit < 0) return -1;
        } else {
            unit = unit_of(all * a.ntiles, blockIdx.x, 0);
            if (unit < 0) return -1;
        }
        const int range = unit / a.ntiles;
        tile = unit - range * a.ntiles;
        return range;
    }, r);
    if (!there) return;                                                // (uniform)
    if (r.rows == 0) {                                                 // (uniform)
        expert_zeros(as_global(a.dst) + (size_t)r.expert * a.result, a.result, tile, a.ntiles);
        return;
    }
    // The expert's ranges are alike, of whole slabs (65,536 rows, 2,048 columns, us, of rows_per and what is left, and alike: 4 experts 316 and 290, 8 370 and
    // 348; 131,072 rows of 1,024, 16 equal experts 178 and 208, of softmax(z) 260 and 249).
    const int each = (((unsigned)r.rows + r.ranges - 1) / (unsigned)r.ranges + 63) & ~63, first = r.sub * each, count = min(each, r.rows - first);
    const View v = expert_view(a, count, r.rows);
    TileJob job;
    tri_decode_blocked<4>(a.tiles_dim, tile, job.I, job.J);
    job.r_begin = 0;
    job.r_end = count;
    job.scale = expert_scale(a, r.rows);
    job.split = r.ranges > 1;
    job.lower = a.ntiles == 1;
    const size_t part = (size_t)r.part + r.sub;
    job.tile_dst = as_global(a.tiles) + (part * a.ntiles + tile) * a.tile_floats;
    job.sums_dst = as_global(a.sums) + part * (a.tiles_dim * a.tw);
    job.first_pixel = job.partner = 0;
    const KFAC_AS1 unsigned char* x = (const KFAC_AS1 unsigned char*)a.x + (size_t)(r.row + first) * a.ld * ES;
    const OutSpec os = expert_out(a, r.expert);
    if (job.I == job.J) {
        if (TW == 128 && a.tw == 64) factor_tile_run<TW == 128 ? 64 : TW, KIND, FEED_PIXELS, true, STREAM>(v, x, job, os, smem);
        else factor_tile_run<TW, KIND, FEED_PIXELS, true, STREAM>(v, x, job, os, smem);
    } else {
        if (TW == 128 && a.tw == 64) factor_tile_run<TW == 128 ? 64 : TW, KIND, FEED_PIXELS, false, STREAM>(v, x, job, os, smem);
        else factor_tile_run<TW, KIND, FEED_PIXELS, false, STREAM>(v, x, job, os, smem);
    }
}

template <int TW, int KIND, bool STREAM>
static int launch_expert_tile_kernel(const char* name, const ExpertArgs& a, unsigned wgs, hipStream_t stream) {
    constexpr int ES = KIND == 2 ? 4 : 2, LDS = tile_lds_bytes<TW, ES>();
    if constexpr (LDS > 64 * 1024) {                                   // (see launch_tile_kernel)
        if (hipFuncSetAttribute((const void*)expert_tile_kernel<TW, KIND, STREAM>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess)
            return KFAC_ERR_HIP;
    }
    void* tok = nullptr;
    if (timing_enabled()) timing_begin(name, stream, &tok);
    hipLaunchKernelGGL((expert_tile_kernel<TW, KIND, STREAM>), dim3(wgs), dim3(tile_threads<TW, ES>()), LDS, stream, a);
    if (tok) timing_end(stream, tok);
    if (hipGetLastError() != hipSuccess) return KFAC_ERR_HIP;
    return KFAC_OK;
}

// KIND 0: bf16, 1: fp16, 2: fp32 (one to a source file).
template <int KIND>
int launch_expert_tiles(const ExpertArgs& a, unsigned wgs, hipStream_t stream)
#ifdef KFAC_EXPERT_KIND
{
    if constexpr (KIND != 2) {
        if (a.tw == 256 && a.streams) return launch_expert_tile_kernel<256, KIND, true>("expert_tile_kernel<256, 16-bit, stream>", a, wgs, stream);
        if (a.tw == 256) return launch_expert_tile_kernel<256, KIND, false>("expert_tile_kernel<256, 16-bit>", a, wgs, stream);
    }
    const bool narrow = a.tw == 64;                                    // (the kernel for 128-wide tiles has both; timed apart)
    if (a.streams) {
        const char* name = KIND == 2 ? narrow ? "expert_tile_kernel<64, f32, stream>" : "expert_tile_kernel<128, f32, stream>"
                                     : narrow ? "expert_tile_kernel<64, 16-bit, stream>" : "expert_tile_kernel<128, 16-bit, stream>";
        return launch_expert_tile_kernel<128, KIND, true>(name, a, wgs, stream);
    }
    const char* name = KIND == 2 ? narrow ? "expert_tile_kernel<64, f32>" : "expert_tile_kernel<128, f32>"
                                 : narrow ? "expert_tile_kernel<64, 16-bit>" : "expert_tile_kernel<128, 16-bit>";
    return launch_expert_tile_kernel<128, KIND, false>(name, a, wgs, stream);
}
template int launch_expert_tiles<KFAC_EXPERT_KIND>(const ExpertArgs&, unsigned, hipStream_t);
#else
    ;
#endif

}  // namespace kfac
