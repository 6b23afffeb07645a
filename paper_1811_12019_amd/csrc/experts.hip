// Tokens on their way to the experts and back: a stable counting sort of the assignments, rows copied to the experts' order, weighted sums
// back, and their gradients.
//
// Sort.  place(i) = offsets[e_i] + #{j < i : e_j = e_i}.  The T K assignments are cut into as many runs as there are workgroups, a run into
// one for each wavefront, a wavefront's into steps of 64.  expert_count_kernel counts a run's experts; expert_place_kernel adds up the
// counts of the runs before its own (all workgroups read all counts: no scan between; a cost that grows with the square of the runs from 4 million
// assignments on, of which a run then has 15,360: 2^24, 2^26, 2^28 and 2^29 assignments to 64 experts 0.17, 0.74, 4.1 and 10.9 ms, to 1,000 0.29, 1.6, 12.3
// and 53), then its wavefronts' counts in LDS, and ranks the
// 64 assignments of a step among themselves: the lanes of the same expert are found bit by bit with ballots, and their number below a
// lane is its rank.  No atomics that return a value: the order is the assignments'.  Runs of one workgroup need one launch.
// Rows.  HBM bound.  A thread takes 16 bytes of a token's row, so that x and y are touched once, whatever the number of choices, and dy once for every
// four of them.
#include <algorithm>

#include "rows16.h"

namespace kfac {

template <bool B> struct BoolConstant { static constexpr bool value = B; };
template <int N> struct IntConstant { static constexpr int value = N; };

constexpr int EX_MAX_EXPERTS = 1024, EX_MAX_CHOICES = 64, EX_MAX_DIM = 1 << 20;

struct SortCut {
    int blocks, waves, per_wave;          // assignments of a wavefront, a multiple of 64
    int bits;                             // of an expert's number
    int group;                            // runs that a workgroup of the first kernel counts
    int width;                            // threads of the second kernel that read a run's counts, 8 each: a power of two
    int lds;                              // bytes of the second kernel
};
constexpr int SORT_STEPS = 2, SORT_STEPS_MANY = 8, SORT_BLOCKS = 256, SORT_ALONE = 6144;
// Runs that one workgroup counts: of many experts several, since every workgroup of the second kernel reads all counts (524,288 assignments to
// 64, 256, 512 and 1,000 experts with 1 11.8, 14.1, 17.9 and 29.6 us, with 4 12.4, 13.6, 15.4 and 17.4).
constexpr int SORT_GROUP = 4, SORT_GROUP_EXPERTS = 256;
constexpr long long SORT_RUN_MAX = 15360;  // (counts of SORT_GROUP runs have 16 bits; whole steps of 8 and of 16 wavefronts)

static SortCut sort_cut(int n, int experts) {
    SortCut c;
    const int most = experts <= 512 ? 16 : 8;                 // (counts of every wavefront in LDS)
    long long blocks = 1;
    c.waves = most;
    if (n <= SORT_ALONE) {                                    // one workgroup, of as few wavefronts as have something to do
        const int want = std::max((n + 64 * SORT_STEPS - 1) / (64 * SORT_STEPS), (experts + 255) / 256);
        c.waves = std::min(std::max(want, 1), most);
    } else {
        const long long run = (long long)most * 64;
        blocks = std::max(std::min((n + run - 1) / run, (long long)SORT_BLOCKS), (n + SORT_RUN_MAX - 1) / SORT_RUN_MAX);
    }
    const long long per = (n + blocks * c.waves - 1) / (blocks * c.waves);
    c.per_wave = std::max((int)((per + 63) / 64 * 64), 64);
    const long long run = (long long)c.per_wave * c.waves;
    c.blocks = (int)std::max((n + run - 1) / run, 1ll);
    c.group = experts >= SORT_GROUP_EXPERTS ? SORT_GROUP : 1;
    c.bits = 0;
    while ((1 << c.bits) < experts) ++c.bits;
    c.width = 1;
    while (c.width * 8 < experts) c.width *= 2;
    c.lds = (c.waves * experts + 2 * c.width * 8 + 1) * 4;
    return c;
}

static unsigned count_wgs(const SortCut& c) { return (unsigned)((c.blocks + c.group - 1) / c.group); }

// The experts of `group` runs, counted: of all of them, counts[blockIdx][e], and of those before each, ahead[run][e], 8 * width of either.
__global__ __launch_bounds__(1024) void expert_count_kernel(const int* expert, int n, int experts, int per_block, int blocks, int group, int width, uint16_t* counts,
                                                            uint16_t* ahead) {
    __shared__ int cnt[SORT_GROUP][EX_MAX_EXPERTS];
    const int t = threadIdx.x, nt = blockDim.x;
    for (int k = 0; k < group; ++k)
        for (int e = t; e < 8 * width; e += nt) cnt[k][e] = 0;
    __syncthreads();
    const int run0 = blockIdx.x * group, steps = per_block / nt;      // (a run is whole steps of the workgroup)
    const long long i0 = (long long)run0 * per_block + t;
    auto count = [&](int k, int e) {
        if ((unsigned)e < (unsigned)experts) atomicAdd(&cnt[k][e], 1);
    };
    if (group == 1) {
        const long long i1 = min((long long)(run0 + 1) * per_block, (long long)n);
#pragma unroll 4
        for (long long i = i0; i < i1; i += nt) count(0, expert[i]);
    } else {
        for (int j0 = 0; j0 < group * steps; j0 += 8) {
            int e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const long long i = i0 + (long long)(j0 + j) * nt;
                e[j] = j0 + j < group * steps && i < n ? expert[i] : -1;
            }
            int k = j0 / steps, left = (k + 1) * steps - j0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                count(k, e[j]);
                if (--left == 0) {
                    ++k;
                    left = steps;
                }
            }
        }
    }
    __syncthreads();
    for (int e = t; e < 8 * width; e += nt) {
        int sum = 0;
        for (int k = 0; k < group; ++k) {
            if (run0 + k < blocks) ahead[(size_t)(run0 + k) * (8 * width) + e] = (uint16_t)sum;
            sum += cnt[k][e];
        }
        counts[(size_t)blockIdx.x * (8 * width) + e] = (uint16_t)sum;
    }
}

// STEPS: a wavefront's assignments and their ranks stay in registers (0: are looked up again).
template <int STEPS>
__global__ __launch_bounds__(1024) void expert_place_kernel(const int* expert, int n, int experts, int per_wave, int bits, int group, int width,
                                                            const uint16_t* counts, const uint16_t* ahead, int* offsets, int* order, int* place) {
    extern __shared__ int lds[];
    const int t = threadIdx.x, nt = blockDim.x, lane = t & 63, wave = t >> 6, waves = nt >> 6;
    int* cnt = lds;                                     // [waves][experts]: a wavefront's counts, then where its rows go
    int* total = cnt + waves * experts;                 // [8 width], at(e): of all runs, then the expert's first row
    int* before = total + 8 * width;                    // the same of the runs before this one
    int* all_rows = before + 8 * width;
    auto at = [&](int e) { return (e & 7) * width + (e >> 3); };   // (neighbouring threads' eights in neighbouring banks)
    const int blk = blockIdx.x, nblk = gridDim.x;
    const long long i0 = ((long long)blk * waves + wave) * per_wave, i1 = i0 + per_wave < n ? i0 + per_wave : n;
    constexpr int HELD = STEPS ? STEPS : 1;
    int held[HELD], rank[HELD];
    if constexpr (STEPS > 0) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) held[k] = i0 + 64 * k + lane < i1 ? expert[i0 + 64 * k + lane] : -1;
    }
    for (int e = t; e < waves * experts + 16 * width; e += nt) cnt[e] = 0;
    // The counts of all runs and of those before this one: groups of `width` threads share out what there is of them, a thread takes 8 experts.
    int all[8] = {}, some[8] = {};
    const int col = t & (width - 1), lists = (nblk + group - 1) / group;
    // (four rows of counts to a thread: the fewer threads, the fewer sums to add up; 65,536 assignments to 8 experts 10.1 -> 8.6 us)
    const int adders = nblk > 1 ? min(nt, max(64, ((lists + 3) / 4 * width + 63) / 64 * 64)) : 0, groups = adders / width;
    if (t < adders) {                                   // (whole wavefronts)
        const int mine = blk / group;
        auto eight = [&](const uint16_t* from, int row, bool to_all, bool to_some) {
            const u4 c = *(const KFAC_AS1 u4*)((const gchar*)from + ((size_t)row * width + col) * 16);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int v = (int)(c[k / 2] >> (k & 1) * 16 & 0xffff);
                all[k] += to_all ? v : 0;
                some[k] += to_some ? v : 0;
            }
        };
        if (group > 1 && t < width) eight(ahead, blk, false, true);
#pragma unroll 8
        for (int b = t / width; b < lists; b += groups) eight(counts, b, true, b < mine);
        for (int off = width; off < 64; off <<= 1) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                all[k] += __shfl_xor(all[k], off, 64);
                some[k] += __shfl_xor(some[k], off, 64);
            }
        }
    }
    __syncthreads();
    if (t < adders && lane < width) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (all[k]) atomicAdd(&total[k * width + col], all[k]);
            if (some[k]) atomicAdd(&before[k * width + col], some[k]);
        }
    }
    // Lanes of the same expert among the 64, and where the wavefront's earlier ones end: the lane's rank.  Counts them.
    int* mine = cnt + wave * experts;
    const unsigned long long below = (1ull << lane) - 1;
    auto rank_of = [&](int e) -> int {
        const bool there = (unsigned)e < (unsigned)experts;
        unsigned long long same = __ballot(there);
        for (int k = 0; k < bits; ++k) {
            const bool bit = (e >> k) & 1;
            const unsigned long long set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        int r = -1;
        if (there) r = mine[e] + __popcll(same & below);
        __builtin_amdgcn_wave_barrier();                // (all have read before one of an expert's lanes writes)
        if (there && (same & below) == 0) mine[e] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
        return r;
    };
    if constexpr (STEPS > 0) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) rank[k] = i0 + 64 * k < i1 ? rank_of(held[k]) : -1;
    } else {
#pragma unroll 8
        for (long long i = i0 + lane; i < i1; i += 64) {
            const int e = expert[i];
            if ((unsigned)e < (unsigned)experts) atomicAdd(&mine[e], 1);
        }
    }
    __syncthreads();
    // The experts' first rows: an exclusive scan by one wavefront, some experts to a lane.  Beside it (of one run: before it) the others go
    // from counts to what lies before a wavefront's rows.
    auto scan = [&]() {
        const int per = (experts + 63) >> 6, e0 = lane * per;
        int own = 0;
        for (int k = 0; k < per; ++k) own += e0 + k < experts ? total[at(e0 + k)] : 0;
        int s = own;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(s, off, 64);
            if (lane >= off) s += up;
        }
        int first = s - own;
        for (int k = 0; k < per && e0 + k < experts; ++k) {
            const int c = total[at(e0 + k)];
            total[at(e0 + k)] = first;
            first += c;
        }
        if (lane == 63) *all_rows = s;
    };
    const int helpers = nblk > 1 ? 64 : 0;              // (threads that scan meanwhile; several runs have at least 8 wavefronts)
    if (t < helpers) {
        scan();
    } else {
        for (int e = t - helpers; e < experts; e += nt - helpers) {
            int sum = 0;
#pragma unroll 8
            for (int w = 0; w < waves; ++w) {
                const int c = cnt[w * experts + e];
                cnt[w * experts + e] = sum;
                sum += c;
            }
            if (nblk == 1) total[at(e)] = sum;
        }
    }
    __syncthreads();
    if (nblk == 1) {
        if (wave == 0) scan();
        __syncthreads();
    }
    const int rows = *all_rows;
    if (blk == 0) {
        for (int e = t; e < experts; e += nt) offsets[e] = total[at(e)];
        if (t == 0) offsets[experts] = rows;
    }
    if constexpr (STEPS > 0) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const long long i = i0 + 64 * k + lane;
            const int e = max(held[k], 0);
            const bool there = rank[k] >= 0;
            const int row = there ? total[at(e)] + before[at(e)] + mine[e] + rank[k] : -1;
            if (i < i1) place[i] = row;
            if (there && order) order[row] = (int)i;
        }
    } else {
        for (int e = lane; e < experts; e += 64) mine[e] += total[at(e)] + before[at(e)];
        __builtin_amdgcn_wave_barrier();
        int next = i0 + lane < i1 ? expert[i0 + lane] : -1;
        for (long long i = i0; i < i1; i += 64) {
            const bool in = i + lane < i1;
            const int e = next;
            next = i + 64 + lane < i1 ? expert[i + 64 + lane] : -1;
            const int row = rank_of(e);
            if (in) place[i + lane] = row;
            if (row >= 0 && order) order[row] = (int)(i + lane);
        }
    }
    if (order)
        for (long long p = rows + (long long)blk * nt + t; p < n; p += (long long)nblk * nt) order[p] = -1;
}

// Thread i: vector i % per_row of token i / per_row.
struct RowArgs {
    unsigned vectors, per_row;
    int choices, rows, dim;
    long long ld_token, ld_row, ld_grad;  // bytes
};

// Vector c of a row.  The last one ends with the row and shares its first elements with the one before, so that all of them are whole (element by
// element, rows of 2,052 bf16 values took 170 us in the gradient of the weighted sum, and take 125); what both store is the same.  Rows shorter than a vector
// are one of `count` elements: f(false).
template <int ES, class F>
__device__ __forceinline__ void by_vector(int dim, unsigned c, F&& f) {
    constexpr int V = 16 / ES;
    if (dim >= V) {                                                    // (uniform)
        const int col = (int)c * V, first = min(col, dim - V);
        f(BoolConstant<true>{}, (long long)first * ES, V, col - first);
    } else {
        f(BoolConstant<false>{}, 0ll, dim, 0);
    }
}

constexpr int GROUP = 4;                  // choices whose rows are fetched together
// Vectors of a row from which on a whole workgroup takes a token's gradients, and tokens up to which it does so for rows of more than 64: the
// rows of a token are then on their way at once.  bf16, us, a wavefront and a workgroup to a token: 16,384 tokens x 4 of 2,048 values (256 vectors) 113 and 103,
// 8,192 x 2 of 1,024 (128) 15.1 and 19.4, 8,192 x 4 of 1,700 78 and 84; 16 x 8 of 4,096 13.3 and 7.5.  Short rows take part of a wavefront.
constexpr unsigned BACK_WORKGROUP = 256;
constexpr int BACK_FEW = 512;
constexpr int DISPATCH_LONG = 4000;       // bytes

template <int ES, bool STREAM>
__global__ __launch_bounds__(256) void expert_dispatch_kernel(RowArgs a, const char* x, const int* place, char* xs) {
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= a.vectors) return;
    const unsigned token = i / a.per_row, c = i - token * a.per_row;
    const gint* p = as_global((int*)place) + (size_t)token * a.choices;
    by_vector<ES>(a.dim, c, [&](auto whole, long long at, int some, int) {
        const int count = decltype(whole)::value ? 16 / ES : some;
        const u4 r = load_row16<ES>((const gchar*)x + token * a.ld_token + at, count);
        for (int k = 0; k < a.choices; ++k) {
            const int row = p[k];
            if ((unsigned)row < (unsigned)a.rows) store_row16<ES, STREAM>((gchar*)xs + row * a.ld_row + at, r, count);
        }
    });
}

template <int KIND, bool STREAM>
__global__ __launch_bounds__(256) void expert_combine_kernel(RowArgs a, const char* ys, const float* weights, const int* place, char* y) {
    constexpr int ES = elem_bytes<KIND>, V = elems16<KIND>;
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= a.vectors) return;
    const unsigned token = i / a.per_row, c = i - token * a.per_row;
    const gint* p = as_global((int*)place) + (size_t)token * a.choices;
    const gfloat* pw = as_global(weights ? (float*)weights : (float*)place) + (size_t)token * a.choices;   // (read and not used without weights)
    by_vector<ES>(a.dim, c, [&](auto whole, long long at, int some, int) {
        const int count = decltype(whole)::value ? V : some;
        float sum[V] = {};
        for (int k0 = 0; k0 < a.choices; k0 += GROUP) {
            int row[GROUP];
            float w[GROUP];
            u4 r[GROUP];
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                const int i = min(k0 + k, a.choices - 1);
                row[k] = k0 + k < a.choices ? p[i] : -1;
                w[k] = pw[i];
            }
#pragma unroll
            for (int k = 0; k < GROUP; ++k)                         // (row 0 stands in for none)
                r[k] = load_row16<ES, STREAM>((const gchar*)ys + ((unsigned)row[k] < (unsigned)a.rows ? row[k] : 0) * a.ld_row + at, count);
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                float f[V];
                unpack16<KIND>(r[k], f);
                const bool there = (unsigned)row[k] < (unsigned)a.rows;
                const float wk = weights ? w[k] : 1.f;
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] = there ? fmaf(wk, f[j], sum[j]) : sum[j];
            }
        }
        store_row16<ES>((gchar*)y + token * a.ld_token + at, pack16<KIND>(sum), count);
    });
}

// LANES threads per token: part of a wavefront, one, or a workgroup; dy's row is fetched once for every GROUP choices.
template <int KIND, bool STREAM, int LANES>
__global__ __launch_bounds__(256) void expert_combine_backward_kernel(RowArgs a, int tokens, const char* dy, const char* ys, const float* weights,
                                                                      const int* place, char* dys, float* dweights) {
    constexpr int ES = elem_bytes<KIND>, V = elems16<KIND>, ACROSS = LANES < 64 ? LANES : 64;
    __shared__ float red[GROUP][4];
    const int lane = threadIdx.x & (LANES - 1);
    unsigned token = blockIdx.x * (256u / LANES) + threadIdx.x / LANES;
    if constexpr (LANES >= 64) token = __builtin_amdgcn_readfirstlane(token);
    const bool in = token < (unsigned)tokens;                          // (a workgroup for a token: always)
    const size_t at = (size_t)(in ? token : 0) * a.choices;
    for (int k0 = 0; k0 < a.choices; k0 += GROUP) {
        int row[GROUP];
        float w[GROUP], dot[GROUP];
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {
            const int i = min(k0 + k, a.choices - 1);
            const int r = place[at + i];
            row[k] = in && k0 + k < a.choices && (unsigned)r < (unsigned)a.rows ? r : -1;
            if constexpr (LANES >= 64) row[k] = __builtin_amdgcn_readfirstlane(row[k]);
            w[k] = weights ? weights[at + i] : 1.f;
            dot[k] = 0.f;
        }
        for (unsigned c = lane; in && c < a.per_row; c += LANES) {
            by_vector<ES>(a.dim, c, [&](auto whole, long long in_row, int some, int shared) {
                const int count = decltype(whole)::value ? V : some;
                const u4 d = load_row16<ES>((const gchar*)dy + token * a.ld_token + in_row, count);
                u4 r[GROUP];
                if (dweights) {                                        // (row 0 stands in for none)
#pragma unroll
                    for (int k = 0; k < GROUP; ++k) r[k] = load_row16<ES, STREAM>((const gchar*)ys + max(row[k], 0) * a.ld_row + in_row, count);
                }
                float g[V], f[V];
                unpack16<KIND>(d, g);
                if (dweights) {
#pragma unroll
                    for (int k = 0; k < GROUP; ++k) {
                        unpack16<KIND>(r[k], f);
#pragma unroll
                        for (int j = 0; j < V; ++j) dot[k] = j >= shared ? fmaf(g[j], f[j], dot[k]) : dot[k];
                    }
                }
#pragma unroll
                for (int k = 0; k < GROUP; ++k) {
                    if (row[k] < 0) continue;
#pragma unroll
                    for (int j = 0; j < V; ++j) f[j] = g[j] * w[k];
                    store_row16<ES, STREAM>((gchar*)dys + row[k] * a.ld_grad + in_row, pack16<KIND>(f), count);
                }
            });
        }
        if (dweights) {
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
#pragma unroll
                for (int off = ACROSS / 2; off > 0; off >>= 1) dot[k] += __shfl_down(dot[k], off, ACROSS);
                const float sum = row[k] >= 0 ? dot[k] : 0.f;
                if (LANES <= 64 && lane == 0 && in && k0 + k < a.choices) dweights[at + k0 + k] = sum;
                if (LANES == 256 && (lane & 63) == 0) red[k][lane >> 6] = sum;
            }
            if constexpr (LANES == 256) {
                __syncthreads();
                if (lane < GROUP && k0 + lane < a.choices) dweights[at + k0 + lane] = (red[lane][0] + red[lane][1]) + (red[lane][2] + red[lane][3]);
                __syncthreads();
            }
        }
    }
}

static bool route_ok(const kfac_expert_desc* d) {
    return d && d->tokens >= 0 && d->choices >= 1 && d->choices <= EX_MAX_CHOICES && d->experts >= 1 && d->experts <= EX_MAX_EXPERTS &&
           (long long)d->tokens * d->choices <= 0x7fffffffLL;
}

// The arguments of the kernels over rows.  KFAC_OK with vectors = 0: no tokens.
static int row_args(const kfac_expert_desc* d, RowArgs* a) {
    if (!route_ok(d) || d->dim < 1 || d->dim > EX_MAX_DIM) return KFAC_ERR_INVALID_ARG;
    if (d->dtype != KFAC_F32 && d->dtype != KFAC_BF16 && d->dtype != KFAC_F16) return KFAC_ERR_INVALID_ARG;
    const int es = d->dtype == KFAC_F32 ? 4 : 2;
    const long long lt = d->ld_token ? d->ld_token : d->dim, lr = d->ld_row ? d->ld_row : d->dim, lg = d->ld_grad ? d->ld_grad : d->dim;
    for (long long ld : {lt, lr, lg})
        if (ld < d->dim || ld > (1ll << 28)) return KFAC_ERR_INVALID_ARG;
    a->per_row = (unsigned)(((long long)d->dim * es + 15) / 16);
    const unsigned long long vectors = (unsigned long long)d->tokens * a->per_row;
    if (vectors > 0x7fffffffull) return KFAC_ERR_TOO_LARGE;
    a->vectors = (unsigned)vectors;
    a->choices = d->choices;
    a->rows = d->tokens * d->choices;
    a->dim = d->dim;
    a->ld_token = lt * es;
    a->ld_row = lr * es;
    a->ld_grad = lg * es;
    return KFAC_OK;
}

static bool on_grid(const void* p, size_t align) { return p && (uintptr_t)p % align == 0; }

// Whether two tensors of np and nq rows of `row` bytes, ldp and ldq bytes from one to the next, share any.  (Rows with gaps may lie in each other's; with
// gaps of two kinds that is not looked into.)
static bool rows_overlap(const void* p, long long np, long long ldp, const void* q, long long nq, long long ldq, long long row) {
    const long long apart = (long long)((uintptr_t)q - (uintptr_t)p);
    if (np == 1) ldp = row;
    if (nq == 1) ldq = row;
    const long long end_p = (np - 1) * ldp + row, end_q = (nq - 1) * ldq + row;
    if (apart >= end_p || -apart >= end_q) return false;
    if (ldp == row) {                                         // the first of q's rows that ends behind p's beginning
        const long long j = apart + row > 0 ? 0 : -(apart + row) / ldq + 1;
        return apart + j * ldq < end_p;
    }
    if (ldq == row) return rows_overlap(q, nq, ldq, p, np, ldp, row);
    if (ldp != ldq) return apart == 0;
    // Row j of q begins `in` bytes behind the place of p's row first + j.
    const long long in = (apart % ldp + ldp) % ldp, first = (apart - in) / ldp;
    auto meet = [&](long long i) { return i < np && i + nq > 0; };
    return (in < row && meet(first)) || (ldp - in < row && meet(first + 1));
}

}  // namespace kfac

using namespace kfac;

// f(kind, streams): the constants of a dtype, and of a pass over `bytes` bytes.
template <class F>
static int by_type(int dtype, size_t bytes, F&& f) {
    auto kind = [&](auto streams) -> int {
        if (dtype == KFAC_BF16) return f(IntConstant<0>{}, streams);
        if (dtype == KFAC_F16) return f(IntConstant<1>{}, streams);
        return f(IntConstant<2>{}, streams);
    };
    return bytes > STREAM_BYTES ? kind(BoolConstant<true>{}) : kind(BoolConstant<false>{});
}
// Bytes of `token_rows` tensors in tokens' order and `sorted_rows` in the experts'.
static size_t moved(const RowArgs& a, int token_rows, int sorted_rows) { return ((size_t)token_rows + (size_t)sorted_rows * a.choices) * a.vectors * 16; }

extern "C" size_t kfac_expert_sort_workspace_bytes(const kfac_expert_desc* desc) {
    if (!route_ok(desc)) return 0;
    const SortCut c = sort_cut(desc->tokens * desc->choices, desc->experts);
    return c.blocks > 1 ? align_up((size_t)(c.blocks + count_wgs(c)) * c.width * 16, 256) : 0;
}

extern "C" int kfac_expert_sort(const kfac_expert_desc* desc, const int32_t* expert, int32_t* offsets, int32_t* order, int32_t* place,
                                void* ws, size_t ws_bytes, void* stream) {
    if (!route_ok(desc) || !on_grid(offsets, 4)) return KFAC_ERR_INVALID_ARG;
    const int n = desc->tokens * desc->choices, E = desc->experts;
    if (n > 0) {
        if (!on_grid(expert, 4) || !on_grid(place, 4) || (uintptr_t)order % 4) return KFAC_ERR_INVALID_ARG;
        const long long bytes = 4ll * n;
        if (rows_overlap(expert, 1, bytes, place, 1, bytes, bytes) || (order && (rows_overlap(expert, 1, bytes, order, 1, bytes, bytes) ||
                                                                                 rows_overlap(place, 1, bytes, order, 1, bytes, bytes))))
            return KFAC_ERR_INVALID_ARG;
    }
    const size_t need = kfac_expert_sort_workspace_bytes(desc);
    if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)) return KFAC_ERR_WORKSPACE;
    const SortCut c = sort_cut(n, E);
    hipStream_t st = (hipStream_t)stream;
    const int threads = 64 * c.waves;
    uint16_t* counts = (uint16_t*)ws;
    uint16_t* ahead = c.blocks > 1 ? counts + (size_t)count_wgs(c) * c.width * 8 : nullptr;
    if (c.blocks > 1)
        KFAC_LAUNCH(expert_count_kernel, dim3(count_wgs(c)), dim3(threads), st, expert, n, E, c.waves * c.per_wave, c.blocks, c.group, c.width, counts, ahead);
    void* tok = nullptr;
    if (timing_enabled()) timing_begin("expert_place_kernel", st, &tok);
    auto kernel = c.per_wave <= 64 * SORT_STEPS        ? expert_place_kernel<SORT_STEPS>
                  : c.per_wave <= 64 * SORT_STEPS_MANY ? expert_place_kernel<SORT_STEPS_MANY>
                                                       : expert_place_kernel<0>;
    hipLaunchKernelGGL(kernel, dim3(c.blocks), dim3(threads), c.lds, st, expert, n, E, c.per_wave, c.bits, c.group, c.width, counts, ahead, offsets,
                       n > 0 ? order : nullptr, place);
    if (tok) timing_end(st, tok);
    KFAC_LAUNCH_CHECK();
    return KFAC_OK;
}

extern "C" int kfac_expert_dispatch(const kfac_expert_desc* desc, const void* x, const int32_t* place, void* xs, void* stream) {
    RowArgs a;
    const int rc = row_args(desc, &a);
    if (rc != KFAC_OK || a.vectors == 0) return rc;
    const int es = desc->dtype == KFAC_F32 ? 4 : 2;
    if (!on_grid(x, es) || !on_grid(xs, es) || !on_grid(place, 4)) return KFAC_ERR_INVALID_ARG;
    if (rows_overlap(x, desc->tokens, a.ld_token, xs, a.rows, a.ld_row, (long long)a.dim * es)) return KFAC_ERR_INVALID_ARG;
    // Short rows that begin and end inside a half cache line are kept: past the caches each end costs a line (bf16, us, kept and past them: 126,030 tokens x 4
    // of 260 columns 91 and 101; 16,384 x 4 of 2,001 76 and 77, of 2,008 74 and 73, of 2,048 66 and 51).
    const bool halves = ((uintptr_t)xs | (uintptr_t)a.ld_row | (uintptr_t)a.dim * es) % 64 == 0;
    return by_type(desc->dtype, halves || a.dim * es >= DISPATCH_LONG ? moved(a, 1, 1) : 0, [&](auto kind, auto streams) -> int {
        constexpr int ES = elem_bytes<decltype(kind)::value>;
        constexpr bool STREAM = decltype(streams)::value;
        KFAC_LAUNCH_AS(STREAM ? "expert_dispatch_kernel<stream>" : "expert_dispatch_kernel", (expert_dispatch_kernel<ES, STREAM>),
                       dim3((a.vectors + 255) / 256), dim3(256), (hipStream_t)stream, a, (const char*)x, place, (char*)xs);
        return KFAC_OK;
    });
}

extern "C" int kfac_expert_combine(const kfac_expert_desc* desc, const void* ys, const float* weights, const int32_t* place, void* y,
                                   void* stream) {
    RowArgs a;
    const int rc = row_args(desc, &a);
    if (rc != KFAC_OK || a.vectors == 0) return rc;
    const int es = desc->dtype == KFAC_F32 ? 4 : 2;
    if (!on_grid(ys, es) || !on_grid(y, es) || !on_grid(place, 4) || (uintptr_t)weights % 4) return KFAC_ERR_INVALID_ARG;
    if (rows_overlap(y, desc->tokens, a.ld_token, ys, a.rows, a.ld_row, (long long)a.dim * es)) return KFAC_ERR_INVALID_ARG;
    return by_type(desc->dtype, moved(a, 1, 1), [&](auto kind, auto streams) -> int {
        constexpr bool STREAM = decltype(streams)::value;
        KFAC_LAUNCH_AS(STREAM ? "expert_combine_kernel<stream>" : "expert_combine_kernel", (expert_combine_kernel<decltype(kind)::value, STREAM>),
                       dim3((a.vectors + 255) / 256), dim3(256), (hipStream_t)stream, a, (const char*)ys, weights, place, (char*)y);
        return KFAC_OK;
    });
}

extern "C" int kfac_expert_combine_backward(const kfac_expert_desc* desc, const void* dy, const void* ys, const float* weights,
                                            const int32_t* place, void* dys, float* dweights, void* stream) {
    RowArgs a;
    const int rc = row_args(desc, &a);
    if (rc != KFAC_OK || a.vectors == 0) return rc;
    const int es = desc->dtype == KFAC_F32 ? 4 : 2;
    if (!on_grid(dy, es) || !on_grid(dys, es) || !on_grid(place, 4) || (uintptr_t)weights % 4 || (uintptr_t)dweights % 4) return KFAC_ERR_INVALID_ARG;
    if (dweights && !on_grid(ys, es)) return KFAC_ERR_INVALID_ARG;
    const long long row = (long long)a.dim * es;
    if (rows_overlap(dy, desc->tokens, a.ld_token, dys, a.rows, a.ld_grad, row)) return KFAC_ERR_INVALID_ARG;
    if (dweights && rows_overlap(ys, a.rows, a.ld_row, dys, a.rows, a.ld_grad, row)) return KFAC_ERR_INVALID_ARG;
    return by_type(desc->dtype, moved(a, 1, dweights ? 2 : 1), [&](auto kind, auto streams) -> int {
        constexpr int KIND = decltype(kind)::value;
        constexpr bool STREAM = decltype(streams)::value;
        const char* name = STREAM ? "expert_combine_backward_kernel<stream>" : "expert_combine_backward_kernel";
        auto launch = [&](auto lanes) -> int {
            constexpr int LANES = decltype(lanes)::value;
            const long long wgs = (desc->tokens + 256ll / LANES - 1) / (256 / LANES);
            if (wgs * 256 > 0xffffffffll) return KFAC_ERR_TOO_LARGE;                            // (threads of a launch)
            KFAC_LAUNCH_AS(name, (expert_combine_backward_kernel<KIND, STREAM, LANES>), dim3((unsigned)wgs), dim3(256),
                           (hipStream_t)stream, a, desc->tokens, (const char*)dy, (const char*)ys, weights, place, (char*)dys, dweights);
            return KFAC_OK;
        };
        if (a.per_row >= BACK_WORKGROUP || (desc->tokens <= BACK_FEW && a.per_row > 64)) return launch(IntConstant<256>{});
        return a.per_row > 32 ? launch(IntConstant<64>{}) : a.per_row > 8 ? launch(IntConstant<32>{}) : launch(IntConstant<8>{});
    });
}
