// The norm over the gradients of many tensors, and clipping by it:
//     norm = sqrt(sum g^2),   out = g min(1, max_norm / norm).
// HBM bound: a gradient's bytes once for the norm, twice more for the clipping.  Launches:
//   grad_partial_kernel   up to NORM_WGS workgroups, each some steps of one or several 4096-element chunks; a double each
//   grad_norm_kernel      (the norm alone) adds those up
//   grad_clip_kernel      every workgroup adds them up itself, in the same order, which saves the launch between
// Squares are added in double precision: fp32 squares of bf16 or fp32 gradients beyond 1.8e19 overflow, and those below 1e-23 vanish.
#include "rows16.h"

namespace kfac {

constexpr int GN_FEW = 64, GN_MAX = 512;  // tensors per launch (argument blocks of 1.9 and 15 KB)
constexpr unsigned GN_CHUNK = 4096;       // elements
constexpr int NORM_WGS = 1024;            // four workgroups to a CU

template <int MAX>
struct GradBatch {
    int count;
    unsigned step;                        // chunks that a workgroup takes at a time
    unsigned prefix[MAX + 1];             // first chunk of tensor i
    unsigned char dtype[MAX];
    unsigned long long n[MAX];
    const void* g[MAX];
    void* out[MAX];
};

// Chunks c0 .. c1 - 1, tensor by tensor from tensor m on, which is the first one's or an earlier one: f(tensor, first element, behind the last one).
template <int MAX, class F>
__device__ __forceinline__ void for_chunks(const GradBatch<MAX>& b, unsigned c0, unsigned c1, int& m, F&& f) {
    if (b.prefix[m + 1] <= c0) {          // the last tensor that begins at c0 or before (one by one, us: clipping 512 tensors of 3 million elements 31 and 16, of 12 million 44 and 33)
        for (int end = b.count - 1; m < end;) {
            const int mid = (m + end + 1) >> 1;
            if (b.prefix[mid] <= c0) m = mid;
            else end = mid - 1;
        }
    }
    for (int k = m; k < b.count && b.prefix[k] < c1; ++k) {
        const unsigned first = b.prefix[k];
        const unsigned long long from = c0 > first ? (unsigned long long)(c0 - first) * GN_CHUNK : 0;
        const unsigned long long n = b.n[k], to = (unsigned long long)(c1 - first) * GN_CHUNK;
        f(k, from, to < n ? to : n);
    }
}
// The tensor of chunk c.
template <int MAX>
__device__ __forceinline__ int tensor_of(const GradBatch<MAX>& b, unsigned c) {
    int m = 0;
#pragma unroll
    for (int k = 0; k < MAX; k += 256) {
        const int i = threadIdx.x + k;
        m += __syncthreads_count(i < b.count - 1 && b.prefix[min(i, MAX - 1) + 1] <= c);
    }
    return m;
}

template <int KIND, bool STREAM>
__device__ __forceinline__ double square_run(const gchar* g, unsigned long long count) {
    constexpr int V = elems16<KIND>, ES = elem_bytes<KIND>;
    const int t = threadIdx.x;
    double s = 0.0;
    auto add = [&](const u4& r) {
        float x[V];
        unpack16<KIND>(r, x);
#pragma unroll
        for (int i = 0; i < V; ++i) s = fma((double)x[i], (double)x[i], s);
    };
    const unsigned long long vecs = count / V;
    unsigned long long v = t;
    for (; v + 3 * 256 < vecs; v += 4 * 256) {
        u4 r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = load_row16<ES, STREAM>(g + (v + j * 256) * 16, V);
#pragma unroll
        for (int j = 0; j < 4; ++j) add(r[j]);
    }
    for (; v < vecs; v += 256) add(load_row16<ES>(g + v * 16, V));
    if (t == 0 && count % V) add(load_row16<ES>(g + vecs * 16, (int)(count % V)));
    return s;
}

template <bool STREAM>
__device__ __forceinline__ double square_part(int dtype, const gchar* g, unsigned long long from, unsigned long long to) {
    if (dtype == KFAC_F32) return square_run<2, STREAM>(g + from * 4, to - from);
    if (dtype == KFAC_BF16) return square_run<0, STREAM>(g + from * 2, to - from);
    return square_run<1, STREAM>(g + from * 2, to - from);
}

template <int MAX, bool STREAM>
__global__ __launch_bounds__(256) void grad_partial_kernel(GradBatch<MAX> b, double* partial) {
    __shared__ double red[4];
    const int t = threadIdx.x;
    const unsigned chunks = b.prefix[b.count];
    int m = tensor_of(b, min(blockIdx.x * b.step, chunks - 1));
    double s = 0.0;
    for (unsigned long long c = (unsigned long long)blockIdx.x * b.step; c < chunks; c += (unsigned long long)gridDim.x * b.step)
        for_chunks(b, (unsigned)c, min((unsigned)c + b.step, chunks), m, [&](int k, unsigned long long from, unsigned long long to) {
            const gchar* g = (const gchar*)b.g[k];
            s += square_part<STREAM>(b.dtype[k], g, from, to);
        });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_down(s, off, 64);
    if ((t & 63) == 0) red[t >> 6] = s;
    __syncthreads();
    if (t == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// All 256 threads get the sum of n doubles, added in an order that depends on n alone.
__device__ __forceinline__ double sum_of(const double* partial, int n, double* red) {
    const int t = threadIdx.x;
    double s = 0.0;
    for (int c = t; c < n; c += 256) s += partial[c];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_down(s, off, 64);
    if ((t & 63) == 0) red[t >> 6] = s;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const double* partial, int n, float* norm) {
    __shared__ double red[4];
    const double s = sum_of(partial, n, red);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <int KIND, bool STREAM>
__device__ __forceinline__ void clip_run(const gchar* g, gchar* out, unsigned long long count, float scale) {
    constexpr int V = elems16<KIND>, ES = elem_bytes<KIND>;
    const int t = threadIdx.x;
    auto scaled = [&](const u4& r) {
        float x[V];
        unpack16<KIND>(r, x);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] *= scale;
        return pack16<KIND>(x);
    };
    const unsigned long long vecs = count / V;
    unsigned long long v = t;
    for (; v + 3 * 256 < vecs; v += 4 * 256) {
        u4 r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = load_row16<ES, STREAM>(g + (v + j * 256) * 16, V);
#pragma unroll
        for (int j = 0; j < 4; ++j) store_row16<ES, STREAM>(out + (v + j * 256) * 16, scaled(r[j]), V);
    }
    for (; v < vecs; v += 256) store_row16<ES>(out + v * 16, scaled(load_row16<ES>(g + v * 16, V)), V);
    if (t == 0 && count % V) store_row16<ES>(out + vecs * 16, scaled(load_row16<ES>(g + vecs * 16, (int)(count % V))), (int)(count % V));
}

template <int MAX, bool STREAM>
__global__ __launch_bounds__(256) void grad_clip_kernel(GradBatch<MAX> b, const double* partial, int n, const float* given, float max_norm, float* norm) {
    __shared__ double red[4];
    double len;
    if (given) {
        len = (double)*given;
    } else {
        len = sqrt(sum_of(partial, n, red));
        if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)len;
    }
    // (finite: as the float that the caller sees)
    const float scale = len > (double)max_norm && (float)len < __builtin_inff() ? (float)((double)max_norm / len) : 1.f;
    const unsigned chunks = b.prefix[b.count];
    const unsigned c0 = (gridDim.x - 1 - blockIdx.x) * b.step;           // (what the first pass read last comes first)
    int m = tensor_of(b, c0);
    for_chunks(b, c0, min(c0 + b.step, chunks), m, [&](int k, unsigned long long from, unsigned long long to) {
        const gchar* g = (const gchar*)b.g[k];
        gchar* out = (gchar*)b.out[k];
        if (scale == 1.f && g == out) return;
        const int dt = b.dtype[k];
        if (dt == KFAC_F32) clip_run<2, STREAM>(g + from * 4, out + from * 4, to - from, scale);
        else if (dt == KFAC_BF16) clip_run<0, STREAM>(g + from * 2, out + from * 2, to - from, scale);
        else clip_run<1, STREAM>(g + from * 2, out + from * 2, to - from, scale);
    });
}

static size_t gn_elem_bytes(int dtype) { return dtype == KFAC_F32 ? 4 : 2; }
static unsigned long long gn_chunks(int64_t n) { return ((unsigned long long)n + GN_CHUNK - 1) / GN_CHUNK; }

constexpr unsigned long long GN_MOST_CHUNKS = 1ull << 31;   // 2^43 elements

// Chunks of all items; 0 if one of them is not valid or they are too many.
static bool gn_total(const kfac_grad_item* items, int count, unsigned long long* total) {
    *total = 0;
    for (int i = 0; i < count; ++i) {
        const kfac_grad_item& it = items[i];
        if (it.n < 0 || it.n >= (int64_t)(GN_MOST_CHUNKS * GN_CHUNK)) return false;
        *total += gn_chunks(it.n);
        if (*total >= GN_MOST_CHUNKS) return false;
    }
    return true;
}

// How the items that have elements are dealt to launches: f(first item, behind the last one, their number, their chunks).
template <class F>
static int gn_launches(const kfac_grad_item* items, int count, F&& f) {
    for (int i = 0; i < count;) {
        const int first = i;
        unsigned chunks = 0;
        int n = 0;
        for (; i < count && n < GN_MAX; ++i) {
            chunks += (unsigned)gn_chunks(items[i].n);
            n += items[i].n != 0;
        }
        if (chunks) {
            const int rc = f(first, i, n, chunks);
            if (rc != KFAC_OK) return rc;
        }
    }
    return KFAC_OK;
}

// Chunks to a step: one where that makes no more than 4096 workgroups, four (32 or 64 KB) of more, and as many as keep their number small.
static unsigned gn_step(unsigned chunks) { return chunks <= 4096 ? 1 : chunks <= 4u << 20 ? 4 : (chunks >> 20); }
static unsigned gn_steps(unsigned chunks) {
    const unsigned step = gn_step(chunks);
    return (unsigned)(((unsigned long long)chunks + step - 1) / step);
}

template <int MAX>
static void gn_fill(const kfac_grad_item* items, int first, int last, GradBatch<MAX>* b) {
    b->count = 0;
    b->prefix[0] = 0;
    for (int i = first; i < last; ++i) {
        const kfac_grad_item& it = items[i];
        if (it.n == 0) continue;
        const int k = b->count++;
        b->prefix[k + 1] = b->prefix[k] + (unsigned)gn_chunks(it.n);
        b->dtype[k] = (unsigned char)it.dtype;
        b->n[k] = (unsigned long long)it.n;
        b->g[k] = it.g;
        b->out[k] = it.out ? it.out : const_cast<void*>(it.g);
    }
    b->step = gn_step(b->prefix[b->count]);
}

static size_t gn_bytes(const kfac_grad_item* items, int count) {
    size_t bytes = 0;
    for (int i = 0; i < count; ++i) bytes += (size_t)items[i].n * gn_elem_bytes(items[i].dtype);
    return bytes;
}

// Workgroups, and sums, of the first pass's launch: all workgroups of the second one read them, at most 4096 of up to 64 launches (32,768 tensors), and
// 64 a launch of more.
static unsigned norm_wgs(unsigned chunks, int count) {
    const unsigned launches = (unsigned)((count + GN_MAX - 1) / GN_MAX), steps = gn_steps(chunks);
    const unsigned most = launches <= 4 ? NORM_WGS : launches >= 64 ? 64 : 4096 / launches;
    return steps < most ? steps : most;
}

static int gn_check(const kfac_grad_item* items, int32_t count, bool clip) {
    if (count < 0 || (count > 0 && !items)) return KFAC_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        const kfac_grad_item& it = items[i];
        if (it.dtype != KFAC_F32 && it.dtype != KFAC_BF16 && it.dtype != KFAC_F16) return KFAC_ERR_INVALID_ARG;
        if (it.n < 0) return KFAC_ERR_INVALID_ARG;
        if (it.n == 0) continue;
        const size_t es = gn_elem_bytes(it.dtype);
        if (!it.g || (uintptr_t)it.g % es) return KFAC_ERR_INVALID_ARG;
        if (clip && it.out && it.out != it.g) {
            const uintptr_t a = (uintptr_t)it.g, b = (uintptr_t)it.out, bytes = (uintptr_t)it.n * es;
            if (b % es || (a < b + bytes && b < a + bytes)) return KFAC_ERR_INVALID_ARG;
        }
    }
    unsigned long long total;
    return gn_total(items, count, &total) ? KFAC_OK : KFAC_ERR_TOO_LARGE;
}

static int gn_first_pass(const kfac_grad_item* items, int count, double* partial, int* n, hipStream_t stream) {
    *n = 0;
    const bool stream_pass = gn_bytes(items, count) > STREAM_BYTES;
    return gn_launches(items, count, [&](int first, int last, int held, unsigned chunks) -> int {
        const unsigned wgs = norm_wgs(chunks, count);
        auto launch = [&](auto& b) -> int {
            gn_fill(items, first, last, &b);
            constexpr int MAX = sizeof(b.dtype);
            if (stream_pass)
                KFAC_LAUNCH_AS("grad_partial_kernel<stream>", (grad_partial_kernel<MAX, true>), dim3(wgs), dim3(256), stream, b, partial + *n);
            else
                KFAC_LAUNCH_AS("grad_partial_kernel", (grad_partial_kernel<MAX, false>), dim3(wgs), dim3(256), stream, b, partial + *n);
            return KFAC_OK;
        };
        GradBatch<GN_FEW> few;
        GradBatch<GN_MAX> many;
        const int rc = held <= GN_FEW ? launch(few) : launch(many);
        *n += (int)wgs;
        return rc;
    });
}

}  // namespace kfac

using namespace kfac;

extern "C" size_t kfac_grad_norm_workspace_bytes(const kfac_grad_item* items_host, int32_t count) {
    unsigned long long total;
    if (!items_host || count <= 0 || !gn_total(items_host, count, &total)) return 0;
    size_t n = 0;
    gn_launches(items_host, count, [&](int, int, int, unsigned chunks) -> int {
        n += norm_wgs(chunks, count);
        return KFAC_OK;
    });
    return align_up(n * sizeof(double), 256);
}

extern "C" int kfac_grad_norm_batched(const kfac_grad_item* items_host, int32_t count, float* norm, void* ws, size_t ws_bytes, void* stream) {
    int rc = gn_check(items_host, count, false);
    if (rc != KFAC_OK) return rc;
    if (!norm || (uintptr_t)norm % 4) return KFAC_ERR_INVALID_ARG;
    unsigned long long total;
    gn_total(items_host, count, &total);
    if (total && (!ws || ((uintptr_t)ws & 255) || ws_bytes < kfac_grad_norm_workspace_bytes(items_host, count))) return KFAC_ERR_WORKSPACE;
    int n;
    rc = gn_first_pass(items_host, count, (double*)ws, &n, (hipStream_t)stream);
    if (rc != KFAC_OK) return rc;
    KFAC_LAUNCH(grad_norm_kernel, dim3(1), dim3(256), (hipStream_t)stream, (const double*)ws, n, norm);
    return KFAC_OK;
}

extern "C" int kfac_grad_clip_batched(const kfac_grad_item* items_host, int32_t count, float max_norm, const float* given_norm, float* norm,
                                      void* ws, size_t ws_bytes, void* stream) {
    int rc = gn_check(items_host, count, true);
    if (rc != KFAC_OK) return rc;
    if (!(max_norm >= 0.f) || (given_norm ? norm != nullptr : norm == nullptr)) return KFAC_ERR_INVALID_ARG;
    if ((uintptr_t)given_norm % 4 || (uintptr_t)norm % 4) return KFAC_ERR_INVALID_ARG;
    unsigned long long total;
    gn_total(items_host, count, &total);
    if (!given_norm && total && (!ws || ((uintptr_t)ws & 255) || ws_bytes < kfac_grad_norm_workspace_bytes(items_host, count))) return KFAC_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    int n = 0;
    if (!given_norm) {
        rc = gn_first_pass(items_host, count, (double*)ws, &n, st);
        if (rc != KFAC_OK) return rc;
        if (!total) {                                          // no elements: a norm of 0
            KFAC_LAUNCH(grad_norm_kernel, dim3(1), dim3(256), st, (const double*)ws, 0, norm);
            return KFAC_OK;
        }
    }
    const bool stream_pass = 2 * gn_bytes(items_host, count) > STREAM_BYTES;
    return gn_launches(items_host, count, [&](int first, int last, int held, unsigned chunks) -> int {
        auto launch = [&](auto& b) -> int {
            gn_fill(items_host, first, last, &b);
            constexpr int MAX = sizeof(b.dtype);
            if (stream_pass)
                KFAC_LAUNCH_AS("grad_clip_kernel<stream>", (grad_clip_kernel<MAX, true>), dim3(gn_steps(chunks)), dim3(256), st, b, (const double*)ws, n,
                               given_norm, max_norm, norm);
            else
                KFAC_LAUNCH_AS("grad_clip_kernel", (grad_clip_kernel<MAX, false>), dim3(gn_steps(chunks)), dim3(256), st, b, (const double*)ws, n,
                               given_norm, max_norm, norm);
            return KFAC_OK;
        };
        GradBatch<GN_FEW> few;
        GradBatch<GN_MAX> many;
        return held <= GN_FEW ? launch(few) : launch(many);
    });
}
