// Tokens on their way to the experts and back: a stable counting sort of the assignments, rows copied to the experts' order, weighted sums
// back, and their gradients.
//
// Sort.  place(i) = offsets[e_i] + #{j < i : e_j = e_i}.  The T K assignments are cut into as many runs as there are workgroups, a run into
// one for each wavefront, a wavefront's into steps of 64.  expert_count_kernel counts a run's experts; expert_place_kernel adds up the
// counts of the runs before its own (all workgroups read all counts: no scan between), then its wavefronts' counts in LDS, and ranks the
// 64 assignments of a step among themselves: the lanes of the same expert are found bit by bit with ballots, and their number below a
// lane is its rank.  No atomics that return a value: the order is the assignments'.  Runs of one workgroup need one launch.
// Rows.  HBM bound.  A thread takes 16 bytes of a token's row, so that x, y and dy are touched once, whatever the number of choices.
#include "rows16.h"

namespace kfac {

constexpr int EX_MAX_EXPERTS = 1024, EX_MAX_CHOICES = 64, EX_MAX_DIM = 1 << 20;

struct SortCut {
    int blocks, waves, per_wave;          // assignments of a wavefront, a multiple of 64
    int bits;                             // of an expert's number
    int lds;                              // bytes of the second kernel
};
constexpr int SORT_STEPS = 4, SORT_BLOCKS = 256, SORT_ALONE = 8192;

static SortCut sort_cut(int n, int experts) {
    SortCut c;
    c.waves = experts <= 512 ? 16 : 8;    // (counts of every wavefront in LDS)
    const long long run = (long long)c.waves * 64 * SORT_STEPS;
    long long blocks = n <= SORT_ALONE ? 1 : (n + run - 1) / run;
    if (blocks > SORT_BLOCKS) blocks = SORT_BLOCKS;
    const long long per = (n + blocks * c.waves - 1) / (blocks * c.waves);
    c.per_wave = (int)((per + 63) / 64 * 64);
    if (c.per_wave < 64) c.per_wave = 64;
    c.blocks = (int)((n + (long long)c.per_wave * c.waves - 1) / ((long long)c.per_wave * c.waves));
    if (c.blocks < 1) c.blocks = 1;
    c.bits = 0;
    while ((1 << c.bits) < experts) ++c.bits;
    c.lds = (c.waves * experts + 2 * experts + 2 * c.waves * 64 + 32) * 4;
    return c;
}

// A run's experts, counted: counts[blockIdx][e].
__global__ __launch_bounds__(1024) void expert_count_kernel(const int* expert, int n, int experts, int per_block, int* counts) {
    __shared__ int cnt[EX_MAX_EXPERTS];
    const int t = threadIdx.x, nt = blockDim.x;
    for (int e = t; e < experts; e += nt) cnt[e] = 0;
    __syncthreads();
    const long long i0 = (long long)blockIdx.x * per_block, i1 = i0 + per_block < n ? i0 + per_block : n;
    for (long long i = i0 + t; i < i1; i += nt) {
        const int e = expert[i];
        if ((unsigned)e < (unsigned)experts) atomicAdd(&cnt[e], 1);
    }
    __syncthreads();
    for (int e = t; e < experts; e += nt) counts[(size_t)blockIdx.x * experts + e] = cnt[e];
}

__global__ __launch_bounds__(1024) void expert_place_kernel(const int* expert, int n, int experts, int per_wave, int bits, const int* counts,
                                                            int* offsets, int* order, int* place) {
    extern __shared__ int lds[];
    const int t = threadIdx.x, nt = blockDim.x, lane = t & 63, wave = t >> 6, waves = nt >> 6;
    int* cnt = lds;                                     // [waves][experts]: a wavefront's counts, then where its next rows go
    int* total = cnt + waves * experts;                 // [experts]: of all runs, then the expert's first row
    int* before = total + experts;                      // [experts]: of the runs before this one
    int* red = before + experts;                        // [2][nt]
    int* scan = red + 2 * nt;                           // [waves] and the number of rows
    const int blk = blockIdx.x, nblk = gridDim.x;
    for (int e = t; e < waves * experts; e += nt) cnt[e] = 0;
    __syncthreads();
    const long long i0 = ((long long)blk * waves + wave) * per_wave, i1 = i0 + per_wave < n ? i0 + per_wave : n;
    for (long long i = i0 + lane; i < i1; i += 64) {
        const int e = expert[i];
        if ((unsigned)e < (unsigned)experts) atomicAdd(&cnt[wave * experts + e], 1);
    }
    if (nblk > 1) {                                     // thread groups share out the runs
        const int width = (experts + 63) & ~63, groups = width <= nt ? nt / width : 1;
        for (int e0 = 0; e0 < experts; e0 += groups > 1 ? experts : nt) {
            const int g = groups > 1 ? t / width : 0, e = e0 + (groups > 1 ? t % width : t);
            int all = 0, mine = 0;
            if (g < groups && e < experts) {
#pragma unroll 8
                for (int b = g; b < nblk; b += groups) {
                    const int c = counts[(size_t)b * experts + e];
                    all += c;
                    mine += b < blk ? c : 0;
                }
            }
            red[t] = all;
            red[nt + t] = mine;
            __syncthreads();
            if (g == 0 && e < experts) {
                for (int k = 1; k < groups; ++k) {
                    all += red[k * width + t];
                    mine += red[nt + k * width + t];
                }
                total[e] = all;
                before[e] = mine;
            }
            __syncthreads();
        }
    } else {
        __syncthreads();
        for (int e = t; e < experts; e += nt) {
            int all = 0;
            for (int w = 0; w < waves; ++w) all += cnt[w * experts + e];
            total[e] = all;
            before[e] = 0;
        }
        __syncthreads();
    }
    // the experts' first rows: an exclusive scan, two experts to a thread
    {
        const int a = 2 * t < experts ? total[2 * t] : 0, b = 2 * t + 1 < experts ? total[2 * t + 1] : 0;
        int s = a + b;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(s, off, 64);
            if (lane >= off) s += up;
        }
        if (lane == 63) scan[wave] = s;
        __syncthreads();
        int base = 0, rows = 0;
        for (int w = 0; w < waves; ++w) {
            if (w < wave) base += scan[w];
            rows += scan[w];
        }
        const int first = base + s - a - b;
        if (2 * t < experts) total[2 * t] = first;
        if (2 * t + 1 < experts) total[2 * t + 1] = first + a;
        if (t == 0) scan[waves] = rows;
    }
    __syncthreads();
    const int rows = scan[waves];
    if (blk == 0) {
        for (int e = t; e < experts; e += nt) offsets[e] = total[e];
        if (t == 0) offsets[experts] = rows;
    }
    for (int e = t; e < experts; e += nt) {
        int at = total[e] + before[e];
        for (int w = 0; w < waves; ++w) {
            const int c = cnt[w * experts + e];
            cnt[w * experts + e] = at;
            at += c;
        }
    }
    __syncthreads();
    int* next = cnt + wave * experts;
    const unsigned long long below = (1ull << lane) - 1;
    for (long long i = i0; i < i1; i += 64) {
        const bool in = i + lane < i1;
        const int e = in ? expert[i + lane] : -1;
        const bool there = (unsigned)e < (unsigned)experts;
        unsigned long long same = __ballot(there);
        for (int k = 0; k < bits; ++k) {
            const bool bit = (e >> k) & 1;
            const unsigned long long set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        int row = -1;
        if (there) row = next[e] + __popcll(same & below);
        __builtin_amdgcn_wave_barrier();                // (all have read before one of an expert's lanes writes)
        if (there && (same & below) == 0) next[e] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (in) place[i + lane] = row;
        if (there && order) order[row] = (int)(i + lane);
    }
    if (order)
        for (long long p = rows + (long long)blk * nt + t; p < n; p += (long long)nblk * nt) order[p] = -1;
}

// Thread i: vector i % per_row of token i / per_row.
struct RowArgs {
    unsigned vectors, per_row;
    int choices, rows, dim;
    long long ld_token, ld_row;           // bytes
};

template <int ES>
__global__ __launch_bounds__(256) void expert_dispatch_kernel(RowArgs a, const char* x, const int* place, char* xs) {
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= a.vectors) return;
    const unsigned token = i / a.per_row, c = i - token * a.per_row;
    const int left = a.dim - (int)c * (16 / ES);
    const u4 r = load_row16<ES>((const gchar*)x + token * a.ld_token + c * 16ll, left);
    const gint* p = as_global((int*)place) + (size_t)token * a.choices;
    for (int k = 0; k < a.choices; ++k) {
        const int row = p[k];
        if ((unsigned)row < (unsigned)a.rows) store_row16<ES>((gchar*)xs + row * a.ld_row + c * 16ll, r, left);
    }
}

template <int KIND>
__global__ __launch_bounds__(256) void expert_combine_kernel(RowArgs a, const char* ys, const float* weights, const int* place, char* y) {
    constexpr int ES = elem_bytes<KIND>, V = elems16<KIND>;
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= a.vectors) return;
    const unsigned token = i / a.per_row, c = i - token * a.per_row;
    const int left = a.dim - (int)c * V;
    const size_t at = (size_t)token * a.choices;
    float sum[V] = {};
    for (int k = 0; k < a.choices; ++k) {
        const int row = place[at + k];
        if ((unsigned)row >= (unsigned)a.rows) continue;
        const float w = weights ? weights[at + k] : 1.f;
        float f[V];
        unpack16<KIND>(load_row16<ES>((const gchar*)ys + row * a.ld_row + c * 16ll, left), f);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = fmaf(w, f[j], sum[j]);
    }
    store_row16<ES>((gchar*)y + token * a.ld_token + c * 16ll, pack16<KIND>(sum), left);
}

// One wavefront per token.
template <int KIND>
__global__ __launch_bounds__(256) void expert_combine_backward_kernel(RowArgs a, int tokens, const char* dy, const char* ys, const float* weights,
                                                                      const int* place, char* dys, float* dweights) {
    constexpr int ES = elem_bytes<KIND>, V = elems16<KIND>;
    const int lane = threadIdx.x & 63;
    const unsigned token = blockIdx.x * 4u + (threadIdx.x >> 6);
    if (token >= (unsigned)tokens) return;
    const size_t at = (size_t)token * a.choices;
    for (int k = 0; k < a.choices; ++k) {
        const int row = place[at + k];
        const bool there = (unsigned)row < (unsigned)a.rows;
        float dot = 0.f;
        if (there) {
            const float w = weights ? weights[at + k] : 1.f;
            for (unsigned c = lane; c < a.per_row; c += 64) {
                const int left = a.dim - (int)c * V;
                float g[V], f[V];
                unpack16<KIND>(load_row16<ES>((const gchar*)dy + token * a.ld_token + c * 16ll, left), g);
                if (dweights) {
                    unpack16<KIND>(load_row16<ES>((const gchar*)ys + row * a.ld_row + c * 16ll, left), f);
#pragma unroll
                    for (int j = 0; j < V; ++j) dot = fmaf(g[j], f[j], dot);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) g[j] *= w;
                store_row16<ES>((gchar*)dys + row * a.ld_row + c * 16ll, pack16<KIND>(g), left);
            }
        }
        if (dweights) {
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) dot += __shfl_down(dot, off, 64);
            if (lane == 0) dweights[at + k] = there ? dot : 0.f;
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
    const long long lt = d->ld_token ? d->ld_token : d->dim, lr = d->ld_row ? d->ld_row : d->dim;
    if (lt < d->dim || lr < d->dim || lt > (1ll << 28) || lr > (1ll << 28)) return KFAC_ERR_INVALID_ARG;
    a->per_row = (unsigned)(((long long)d->dim * es + 15) / 16);
    const unsigned long long vectors = (unsigned long long)d->tokens * a->per_row;
    if (vectors > 0x7fffffffull) return KFAC_ERR_TOO_LARGE;
    a->vectors = (unsigned)vectors;
    a->choices = d->choices;
    a->rows = d->tokens * d->choices;
    a->dim = d->dim;
    a->ld_token = lt * es;
    a->ld_row = lr * es;
    return KFAC_OK;
}

static bool on_grid(const void* p, size_t align) { return p && (uintptr_t)p % align == 0; }

// Whether two tensors of rows may share elements (rows with gaps may lie in each other's).
static bool rows_overlap(const void* p, long long np, long long ldp, const void* q, long long nq, long long ldq, long long row) {
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    if (a == b) return true;
    if (ldp != row || ldq != row) return false;
    return a < b + (uintptr_t)(nq * row) && b < a + (uintptr_t)(np * row);
}

}  // namespace kfac

using namespace kfac;

#define KFAC_BY_DTYPE(dtype, kernel, grid, block, stream, ...)                                     \
    do {                                                                                          \
        if ((dtype) == KFAC_BF16) KFAC_LAUNCH(kernel<0>, grid, block, stream, __VA_ARGS__);       \
        else if ((dtype) == KFAC_F16) KFAC_LAUNCH(kernel<1>, grid, block, stream, __VA_ARGS__);   \
        else KFAC_LAUNCH(kernel<2>, grid, block, stream, __VA_ARGS__);                            \
    } while (0)

extern "C" size_t kfac_expert_sort_workspace_bytes(const kfac_expert_desc* desc) {
    if (!route_ok(desc)) return 0;
    const SortCut c = sort_cut(desc->tokens * desc->choices, desc->experts);
    return c.blocks > 1 ? align_up((size_t)c.blocks * desc->experts * sizeof(int), 256) : 0;
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
    if (c.blocks > 1) KFAC_LAUNCH(expert_count_kernel, dim3(c.blocks), dim3(threads), st, expert, n, E, c.waves * c.per_wave, (int*)ws);
    void* tok = nullptr;
    if (timing_enabled()) timing_begin("expert_place_kernel", st, &tok);
    hipLaunchKernelGGL(expert_place_kernel, dim3(c.blocks), dim3(threads), c.lds, st, expert, n, E, c.per_wave, c.bits, (const int*)ws, offsets,
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
    const dim3 grid((a.vectors + 255) / 256);
    if (es == 4) KFAC_LAUNCH(expert_dispatch_kernel<4>, grid, dim3(256), (hipStream_t)stream, a, (const char*)x, place, (char*)xs);
    else KFAC_LAUNCH(expert_dispatch_kernel<2>, grid, dim3(256), (hipStream_t)stream, a, (const char*)x, place, (char*)xs);
    return KFAC_OK;
}

extern "C" int kfac_expert_combine(const kfac_expert_desc* desc, const void* ys, const float* weights, const int32_t* place, void* y,
                                   void* stream) {
    RowArgs a;
    const int rc = row_args(desc, &a);
    if (rc != KFAC_OK || a.vectors == 0) return rc;
    const int es = desc->dtype == KFAC_F32 ? 4 : 2;
    if (!on_grid(ys, es) || !on_grid(y, es) || !on_grid(place, 4) || (uintptr_t)weights % 4) return KFAC_ERR_INVALID_ARG;
    if (rows_overlap(y, desc->tokens, a.ld_token, ys, a.rows, a.ld_row, (long long)a.dim * es)) return KFAC_ERR_INVALID_ARG;
    KFAC_BY_DTYPE(desc->dtype, expert_combine_kernel, dim3((a.vectors + 255) / 256), dim3(256), (hipStream_t)stream, a, (const char*)ys, weights,
                  place, (char*)y);
    return KFAC_OK;
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
    if (rows_overlap(dy, desc->tokens, a.ld_token, dys, a.rows, a.ld_row, row)) return KFAC_ERR_INVALID_ARG;
    if (dweights && rows_overlap(ys, a.rows, a.ld_row, dys, a.rows, a.ld_row, row)) return KFAC_ERR_INVALID_ARG;
    KFAC_BY_DTYPE(desc->dtype, expert_combine_backward_kernel, dim3((desc->tokens + 3) / 4), dim3(256), (hipStream_t)stream, a, desc->tokens,
                  (const char*)dy, (const char*)ys, weights, place, (char*)dys, dweights);
    return KFAC_OK;
}
