// Operators over a list of tensors: the norm of all gradients of a step, clipping by it, and Adam on every tensor.
//
//   norm = sqrt(sum over all tensors and elements of g^2)
//   c    = min(1, max_norm / (norm + 1e-6))
//   gsr_grad_clip: out = c g          gsr_adam_update_list: gsr_adam_update with c g in the place of the gradient
//
// Tensors are contiguous arrays anywhere in device memory.  Their addresses and sizes go to the kernels as arguments, so a call
// leaves nothing behind on the device and can be captured; lists longer than an argument block holds take several launches.
#include "gsr_internal.h"
#include "gsr_device.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace gsr {

constexpr int kArgBytes = 4096 - 256;           // tensor table of a launch (kernel arguments: 4 KB)
// Elements that a workgroup takes at a time.  Every kernel here is bound by memory, reads and writes past the caches, and was timed with 2,048 to
// 16,384: norm of 400M 16-bit values (up to 16,384 workgroups, several chunks each) 152 us at 16,384, 139 at 8,192, 130 at 4,096,
// 175 at 2,048; clipping 201M floats (one chunk per workgroup) 472, 426, 412, 402 us at 2,048; clipped Adam on 120M weights with 16-bit
// gradients 706, 662, 617, 593 us.  With cached accesses at 8,192: 161, 488 and 726 us.  A tensor found in one round trip (tensor_of):
// 126 (6.4 TB/s; a loop that does nothing else reads 7.1), 397 (two passes over the gradients: 6.1 TB/s) and 586 us (5.7, the norm before it included).
constexpr int kNormChunk = 4096, kUpdateChunk = 2048;
constexpr int kMaxPartials = 16384;             // workgroups, hence partial sums, of one launch of the norm
constexpr double kClipEps = 1e-6;
// Chunks of which one workgroup takes the norm in one launch. In a captured graph, 4 chunks 4.0 us against 5.0 with two launches, 8: 4.8 / 5.5,
// 16: 7.1 / 5.6 (with the tensor of a chunk found in one round trip 8: 4.2); a call from Python 9.5 / 12.5.
constexpr int kSmallNorm = 8;
// Partial sums that every workgroup of the clipping adds up by itself instead of waiting for a launch that does.  In a captured graph, tensors of 28,372
// floats into others, 14 / 252 / 497 / 798 / 1,015 partial sums 7.4 / 8.7 / 10.9 / 13.3 / 17.9 us against 8.7 / 9.9 / 11.4 / 14.2 / 18.2 with the launch;
// built for 2,048 of them 1,498 take as long either way (25.3), 2,037 33.8 against 32.9, and 498 11.3.
constexpr int kClipPartials = 1024;

// The tensors of one launch: P addresses each (gradient; gradient and output; w, dw, m, v).
template <int P>
struct TensorTable {
    static constexpr int kMax = (kArgBytes - 16) / (8 * P + 8 + 4);
    int32_t count, chunks;
    void* at[P][kMax];
    int64_t size[kMax];
    int32_t first[kMax];                        // chunks of the tensors before
};

// The tensor that chunk c (the same for a wave) belongs to: the last that begins at or before it, counted by the wave's lanes in one round trip to the
// table (a search takes eight, one after the other).
template <int P>
__device__ __forceinline__ int tensor_of(const TensorTable<P>& t, int c) {
    constexpr int ROUNDS = (TensorTable<P>::kMax + 63) / 64;
    int first[ROUNDS], before = 0;
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u) {
        const int i = lane_id() + 64 * u;
        first[u] = t.first[i < TensorTable<P>::kMax ? i : 0];
    }
#pragma unroll
    for (int u = 0; u < ROUNDS; ++u) before += __popcll(ballot(lane_id() + 64 * u < t.count && first[u] <= c));
    return __builtin_amdgcn_readfirstlane(before - 1);
}

// ---- V elements at a time, past the caches, aligned to their elements only -------------------------------------
__device__ __forceinline__ void load_v(const float* p, float (&v)[4]) {
    const u32x4a* q = reinterpret_cast<const u32x4a*>(p);
    const u32x4a t = __builtin_nontemporal_load(q);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(t[i]);
}
__device__ __forceinline__ void load_v(const bf16_t* p, float (&v)[4]) {
    const u32x2h* q = reinterpret_cast<const u32x2h*>(p);
    const u32x2h t = __builtin_nontemporal_load(q);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float((i & 1) ? (t[i >> 1] & 0xFFFF0000u) : (t[i >> 1] << 16));
}
__device__ __forceinline__ void load_v(const bf16_t* p, float (&v)[8]) {
    const u32x4h* q = reinterpret_cast<const u32x4h*>(p);
    const u32x4h t = __builtin_nontemporal_load(q);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((i & 1) ? (t[i >> 1] & 0xFFFF0000u) : (t[i >> 1] << 16));
}
__device__ __forceinline__ void store_v(float* p, const float (&v)[4]) {
    u32x4a t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __float_as_uint(v[i]);
    __builtin_nontemporal_store(t, reinterpret_cast<u32x4a*>(p));
}
template <int V>
__device__ __forceinline__ void store_v(bf16_t* p, const float (&v)[V]) {
    typedef uint32_t words __attribute__((ext_vector_type(V / 2), aligned(2)));
    words t;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) t[i] = bf16_bits(v[2 * i]) | (bf16_bits(v[2 * i + 1]) << 16);
    __builtin_nontemporal_store(t, reinterpret_cast<words*>(p));
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { p->bits = (uint16_t)bf16_bits(v); }

// ---- norm -------------------------------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// the sum over a workgroup of W waves, in the lanes of the first
template <int W>
__device__ __forceinline__ double wg_sum(double v) {
    __shared__ double s_sum[W];
    v = wave_sum(v);
    if (lane_id() == 0) s_sum[threadIdx.x >> 6] = v;
    __syncthreads();
    return threadIdx.x < 64 ? wave_sum(lane_id() < W ? s_sum[lane_id()] : 0.0) : 0.0;
}

// Squares and sums in 64 bits: no float's square overflows or vanishes there, and how elements are dealt out hardly matters. It costs one
// 64-bit multiply-add per element, of which the chip does some thirty for every float that memory delivers.
template <typename T>
__device__ __forceinline__ double chunk_squares(const TensorTable<1>& t, int c, int thread) {     // a share of chunk c for each of 256 threads
    double sum = 0.0;
    const int i = tensor_of(t, c);
    const int64_t a = (int64_t)(c - t.first[i]) * kNormChunk;
    const int left = (int)(t.size[i] - a < kNormChunk ? t.size[i] - a : kNormChunk);
    const T* g = static_cast<const T*>(t.at[0][i]) + a;
    if (left == kNormChunk) {
        constexpr int V = 16 / sizeof(T), U = kNormChunk / (256 * V);
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load_v(g + 256 * V * u + V * thread, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < V; ++j) sum = fma((double)v[u][j], (double)v[u][j], sum);
    } else {
        for (int e = thread; e < left; e += 256) {
            const double x = to_float(g[e]);
            sum = fma(x, x, sum);
        }
    }
    return sum;
}
template <typename T>
__global__ __launch_bounds__(256) void k_norm_partial(TensorTable<1> t, double* __restrict__ partial) {
    double sum = 0.0;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) sum += chunk_squares<T>(t, c, threadIdx.x);
    sum = wg_sum<4>(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}
// the whole norm of up to kSmallNorm chunks, four at a time
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_small(TensorTable<1> t, double* __restrict__ norm, float* __restrict__ norm_out) {
    double sum = 0.0;
    for (int c = threadIdx.x >> 8; c < t.chunks; c += 4) sum += chunk_squares<T>(t, c, threadIdx.x & 255);
    sum = wg_sum<16>(sum);
    if (threadIdx.x == 0) {
        const double r = sqrt(sum);
        *norm = r;
        if (norm_out) *norm_out = (float)r;
    }
}
__global__ __launch_bounds__(1024) void k_norm_final(const double* __restrict__ partial, int count, double* __restrict__ norm,
                                                     float* __restrict__ norm_out) {
    constexpr int U = 4;                        // (16: 3.4 us instead of 2.2 for 800 partial sums, no less for 30,000)
    double sum = 0.0;
    for (int i = threadIdx.x; i < count; i += U * 1024) {
        double p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) p[u] = partial[i + 1024 * u < count ? i + 1024 * u : i];
#pragma unroll
        for (int u = 0; u < U; ++u) sum += i + 1024 * u < count ? p[u] : 0.0;
    }
    sum = wg_sum<16>(sum);
    if (threadIdx.x == 0) {
        const double r = sqrt(sum);
        *norm = r;
        if (norm_out) *norm_out = (float)r;
    }
}

// NaN stays NaN (a comparison with it is false), an infinite norm gives 0
__device__ __forceinline__ double clip_coefficient(double norm, double max_norm) {
    const double c = max_norm / (norm + kClipEps);
    return c >= 1.0 ? 1.0 : c;
}

// ---- clipping ---------------------------------------------------------------------------------------------
// The product is taken in 64 bits, so a gradient is rounded once (16-bit output: twice).
struct ClipNorm {
    const double* norm;         // the norm, or, with partials, the sums of squares that every workgroup adds up by itself
    int partials;
    float* norm_out;            // written by the first workgroup if it added them up
    double max_norm;
};
template <typename T, typename O>
__global__ __launch_bounds__(256) void k_clip(TensorTable<2> t, ClipNorm n, bool in_place) {
    double norm;
    if (n.partials) {
        __shared__ double s_norm;
        double sum = 0.0;
#pragma unroll
        for (int u = 0; u < kClipPartials / 256; ++u) {
            const int i = threadIdx.x + 256 * u;
            const double p = n.norm[i < n.partials ? i : 0];
            sum += i < n.partials ? p : 0.0;
        }
        sum = wg_sum<4>(sum);
        if (threadIdx.x == 0) {
            s_norm = sqrt(sum);
            if (n.norm_out && blockIdx.x == 0) *n.norm_out = (float)s_norm;
        }
        __syncthreads();
        norm = s_norm;
    } else {
        norm = *n.norm;
    }
    const double k = clip_coefficient(norm, n.max_norm);
    if (in_place && k == 1.0) return;           // multiplied by one: already there
    const int c = t.chunks - 1 - blockIdx.x, i = tensor_of(t, c);       // backwards: what the norm read last may still be cached
    const int64_t a = (int64_t)(c - t.first[i]) * kUpdateChunk;
    const int left = (int)(t.size[i] - a < kUpdateChunk ? t.size[i] - a : kUpdateChunk);
    const T* g = static_cast<const T*>(t.at[0][i]) + a;
    O* out = static_cast<O*>(t.at[1][i]) + a;
    if (left == kUpdateChunk) {
        constexpr int V = sizeof(T) == 2 && sizeof(O) == 2 ? 8 : 4, U = kUpdateChunk / (256 * V);
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load_v(g + 256 * V * u + V * threadIdx.x, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[u][j] = (float)(k * (double)v[u][j]);
            store_v(out + 256 * V * u + V * threadIdx.x, v[u]);
        }
    } else {
        for (int e = threadIdx.x; e < left; e += 256) store1(out + e, (float)(k * (double)to_float(g[e])));
    }
}

// ---- Adam -------------------------------------------------------------------------------------------------
struct AdamParams {
    float lr, b1, b2, r1, r2, eps, wd, inv_c1, inv_c2;          // r = 1 - b, rounded once (1.0f - 0.999f is off by 1.3e-5 of itself)
};
// the arithmetic of k_adam but for r1 and r2, the gradient multiplied by the clipping coefficient first (by one, exactly, without clipping)
__device__ __forceinline__ void adam_one(const AdamParams& p, float k, float& w, float dw, float& m, float& v) {
    const float x = w;
    const float gk = k * dw;
    const float g = gk + p.wd * x;
    const float mi = p.b1 * m + p.r1 * g;
    const float vi = p.b2 * v + p.r2 * g * g;
    m = mi;
    v = vi;
    w = x - p.lr * (mi * p.inv_c1) / (sqrtf(vi * p.inv_c2) + p.eps);
}
template <typename T>
__global__ __launch_bounds__(256) void k_adam_list(TensorTable<4> t, const float* __restrict__ norm, double max_norm, AdamParams p) {
    const float k = norm ? (float)clip_coefficient((double)*norm, max_norm) : 1.0f;
    const int c = t.chunks - 1 - blockIdx.x, i = tensor_of(t, c);       // backwards, as k_clip
    const int64_t a = (int64_t)(c - t.first[i]) * kUpdateChunk;
    const int left = (int)(t.size[i] - a < kUpdateChunk ? t.size[i] - a : kUpdateChunk);
    float* w = static_cast<float*>(t.at[0][i]) + a;
    const T* dw = static_cast<const T*>(t.at[1][i]) + a;
    float* m = static_cast<float*>(t.at[2][i]) + a;
    float* v = static_cast<float*>(t.at[3][i]) + a;
    if (left == kUpdateChunk) {
#pragma unroll
        for (int u = 0; u < kUpdateChunk / 1024; ++u) {
            const int e = 1024 * u + 4 * threadIdx.x;
            float x[4], g[4], y[4], z[4];
            load_v(w + e, x);
            load_v(dw + e, g);
            load_v(m + e, y);
            load_v(v + e, z);
#pragma unroll
            for (int j = 0; j < 4; ++j) adam_one(p, k, x[j], g[j], y[j], z[j]);
            store_v(w + e, x);
            store_v(m + e, y);
            store_v(v + e, z);
        }
    } else {
        for (int e = threadIdx.x; e < left; e += 256) {
            float x = w[e], y = m[e], z = v[e];
            adam_one(p, k, x, to_float(dw[e]), y, z);
            w[e] = x;
            m[e] = y;
            v[e] = z;
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------
namespace {

constexpr int64_t kMaxLaunchChunks = (int64_t)1 << 23;         // (a grid holds fewer than 2^32 threads)

// Calls launch(table) for the tensors of the list, an argument block at a time; empty tensors are left out.  A tensor of more chunks
// than one launch takes goes on in the next.
template <int P, int kChunk, typename Launch>
void over_list(void* const* const (&lists)[P], const size_t (&width)[P], const int64_t* counts, int32_t tensors, Launch launch) {
    TensorTable<P> t;
    t.count = t.chunks = 0;
    for (int32_t i = 0; i < tensors; ++i) {
        for (int64_t at = 0; at < counts[i];) {
            const int64_t room = kMaxLaunchChunks - t.chunks, size = std::min(counts[i] - at, room * kChunk);
            for (int p = 0; p < P; ++p) t.at[p][t.count] = (char*)lists[p][i] + at * (int64_t)width[p];
            t.size[t.count] = size;
            t.first[t.count] = t.chunks;
            t.chunks += (int32_t)((size + kChunk - 1) / kChunk);
            at += size;
            if (++t.count == TensorTable<P>::kMax || t.chunks == kMaxLaunchChunks) {
                launch(t);
                t.count = t.chunks = 0;
            }
        }
    }
    if (t.count) launch(t);
}

// Launches that over_list makes at most: some end with a full table, some with a full grid (of tensors that are cut there, each of which
// takes a place in a second table), the last with neither.
int64_t list_launches(int64_t tensors, int64_t elements, int per_launch) {
    const int64_t full_grids = elements / ((kMaxLaunchChunks - per_launch) * (int64_t)kNormChunk);
    return (tensors + full_grids) / per_launch + full_grids + 1;
}

struct Range {
    uintptr_t from, to;
    bool written;
};

// Sizes and addresses of a list: P arrays of `tensors` pointers, bit p of `written` set where array p is written.  What a call
// writes may overlap nothing else of it (a tensor named twice would be updated twice, in no fixed order).
template <int P>
gsr_status_t check_list(void* const* const (&lists)[P], const size_t (&width)[P], unsigned written, const int64_t* counts, int32_t tensors,
                        int64_t* elements) {
    if (tensors < 0) return fail(GSR_ERR_INVALID_ARG, "negative number of tensors");
    *elements = 0;
    if (tensors == 0) return GSR_OK;
    if (!counts) return fail(GSR_ERR_INVALID_ARG, "null pointer");
    for (int p = 0; p < P; ++p)
        if (!lists[p]) return fail(GSR_ERR_INVALID_ARG, "null pointer");
    try {
        std::vector<Range> r;
        if (written) r.reserve((size_t)tensors * P);
        for (int32_t i = 0; i < tensors; ++i) {
            if (counts[i] < 0) return fail(GSR_ERR_INVALID_ARG, "tensor %d has a negative size", i);
            if (counts[i] > ((int64_t)1 << 40) - *elements) return fail(GSR_ERR_UNSUPPORTED, "more than 2^40 elements");
            *elements += counts[i];
            if (counts[i] == 0) continue;
            for (int p = 0; p < P; ++p) {
                const uintptr_t at = (uintptr_t)lists[p][i];
                if (!at) return fail(GSR_ERR_INVALID_ARG, "tensor %d is a null pointer", i);
                if (at & (width[p] - 1)) return fail(GSR_ERR_INVALID_ARG, "tensor %d is not aligned to its elements", i);
                if (written) r.push_back({at, at + (uintptr_t)counts[i] * width[p], ((written >> p) & 1) != 0});
            }
        }
        auto before = [](const Range& a, const Range& b) { return a.from < b.from; };
        if (!std::is_sorted(r.begin(), r.end(), before)) std::sort(r.begin(), r.end(), before);
        uintptr_t read_to = 0, written_to = 0;              // ends of what lies before
        for (const Range& x : r) {
            if (x.from < written_to || (x.written && x.from < read_to))
                return fail(GSR_ERR_INVALID_ARG, "tensors overlap, one of them is written");
            if (x.written) written_to = std::max(written_to, x.to);
            else read_to = std::max(read_to, x.to);
        }
    } catch (const std::bad_alloc&) {
        return fail(GSR_ERR_INVALID_ARG, "out of host memory for a list of %d tensors", tensors);
    }
    return GSR_OK;
}

// Whether `bytes` at p overlap a tensor of the arrays of pointers whose bits of `which` are set.  Addresses and sizes have passed check_list.
template <int P>
bool over_tensor(const void* p, size_t bytes, void* const* const (&lists)[P], const size_t (&width)[P], unsigned which, const int64_t* counts,
                 int32_t tensors) {
    const uintptr_t from = (uintptr_t)p, to = from + bytes;
    for (int k = 0; k < P; ++k)
        for (int32_t i = 0; ((which >> k) & 1) && i < tensors; ++i) {
            const uintptr_t at = (uintptr_t)lists[k][i];
            if (counts[i] && at < to && from < at + (uintptr_t)counts[i] * width[k]) return true;
        }
    return false;
}

gsr_status_t list_dtype(int32_t dtype) {
    if (dtype != GSR_F32 && dtype != GSR_BF16) return fail(GSR_ERR_UNSUPPORTED, "dtype %d", dtype);
    return GSR_OK;
}

// workspace of the norm: the norm in 64 bits, then the partial sums
size_t norm_workspace(int64_t tensors, int64_t elements) {
    const int64_t launches = list_launches(tensors, elements, TensorTable<1>::kMax);
    return 256 + sizeof(double) * (size_t)std::min(kMaxPartials * launches, elements / kNormChunk + tensors + launches);
}

// Leaves the norm at workspace and at norm_out, or, if clip is given and the partial sums are few, only the partial sums: ClipNorm says which.
ClipNorm launch_norm(void* const* grads, const int64_t* counts, int32_t tensors, int32_t dtype, float* norm_out, bool clip, void* workspace,
                     hipStream_t s) {
    double *norm = (double*)workspace, *partial = (double*)((char*)workspace + 256);
    int made = 0;
    bool done = false;
    int64_t chunks = 0;
    for (int32_t i = 0; i < tensors; ++i) chunks += (counts[i] + kNormChunk - 1) / kNormChunk;
    const bool small = chunks <= kSmallNorm;
    over_list<1, kNormChunk>({grads}, {dtype_size(dtype)}, counts, tensors, [&](const TensorTable<1>& t) {
        if (small) {            // (chunks are of one tensor each: no more tables than one)
            if (dtype == GSR_F32) hipLaunchKernelGGL((k_norm_small<float>), dim3(1), dim3(1024), 0, s, t, norm, norm_out);
            else hipLaunchKernelGGL((k_norm_small<bf16_t>), dim3(1), dim3(1024), 0, s, t, norm, norm_out);
            done = true;
            return;
        }
        const int wgs = std::min(t.chunks, kMaxPartials);
        if (dtype == GSR_F32) hipLaunchKernelGGL((k_norm_partial<float>), dim3(wgs), dim3(256), 0, s, t, partial + made);
        else hipLaunchKernelGGL((k_norm_partial<bf16_t>), dim3(wgs), dim3(256), 0, s, t, partial + made);
        made += wgs;
    });
    if (clip && made && made <= kClipPartials) return {partial, made, norm_out, 0.0};
    if (!done) hipLaunchKernelGGL(k_norm_final, dim3(1), dim3(1024), 0, s, partial, made, norm, norm_out);
    return {norm, 0, nullptr, 0.0};
}

gsr_status_t check_norm_workspace(int64_t tensors, int64_t elements, const void* workspace, size_t bytes) {
    const size_t need = norm_workspace(tensors, elements);
    if (bytes < need) return fail(GSR_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, %zu needed", bytes, need);
    if (!workspace) return fail(GSR_ERR_INVALID_ARG, "null workspace");
    if ((uintptr_t)workspace & 7) return fail(GSR_ERR_INVALID_ARG, "workspace not aligned to 8 bytes");
    return GSR_OK;
}

// norm_out and the workspace lie apart from the tensors and from each other: the first workgroup of k_clip writes norm_out while others still read
// gradients and partial sums.
template <int P>
gsr_status_t check_apart(const float* norm_out, const void* workspace, void* const* const (&lists)[P], const size_t (&width)[P],
                         const int64_t* counts, int32_t tensors, int64_t elements) {
    const size_t bytes = norm_workspace(tensors, elements);
    const unsigned all = (1u << P) - 1;
    if (norm_out && over_tensor<P>(norm_out, 4, lists, width, all, counts, tensors)) return fail(GSR_ERR_INVALID_ARG, "norm_out overlaps a tensor");
    if (over_tensor<P>(workspace, bytes, lists, width, all, counts, tensors)) return fail(GSR_ERR_INVALID_ARG, "the workspace overlaps a tensor");
    if (norm_out && (uintptr_t)norm_out + 4 > (uintptr_t)workspace && (uintptr_t)norm_out < (uintptr_t)workspace + bytes)
        return fail(GSR_ERR_INVALID_ARG, "norm_out lies in the workspace");
    return GSR_OK;
}

}  // namespace
}  // namespace gsr

using namespace gsr;

extern "C" {

size_t gsr_grad_norm_workspace(const int64_t* counts, int32_t tensors) {
    int64_t elements = 0;
    for (int32_t i = 0; counts && i < tensors; ++i) {
        if (counts[i] < 0 || counts[i] > ((int64_t)1 << 40) - elements) return 0;
        elements += counts[i];
    }
    return tensors < 0 ? 0 : norm_workspace(tensors, elements);
}

gsr_status_t gsr_grad_norm(const void* const* grads, const int64_t* counts, int32_t tensors, int32_t dtype, float* norm_out, void* workspace,
                           size_t workspace_bytes, void* stream) {
    int64_t elements;
    GSR_TRY(list_dtype(dtype));
    void* const* g = (void* const*)grads;
    GSR_TRY(check_list<1>({g}, {dtype_size(dtype)}, 0, counts, tensors, &elements));
    if (!norm_out || ((uintptr_t)norm_out & 3)) return fail(GSR_ERR_INVALID_ARG, "norm_out is null or not aligned");
    GSR_TRY(check_norm_workspace(tensors, elements, workspace, workspace_bytes));
    GSR_TRY(check_apart<1>(norm_out, workspace, {g}, {dtype_size(dtype)}, counts, tensors, elements));
    launch_norm(g, counts, tensors, dtype, norm_out, false, workspace, (hipStream_t)stream);
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

gsr_status_t gsr_grad_clip(void* const* grads, const int64_t* counts, int32_t tensors, int32_t dtype, float max_norm, float* norm_out,
                           void* const* out, int32_t out_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    int64_t elements;
    GSR_TRY(list_dtype(dtype));
    if (out) GSR_TRY(list_dtype(out_dtype));
    else out_dtype = dtype;
    if (!(max_norm >= 0.0f) || std::isinf(max_norm)) return fail(GSR_ERR_INVALID_ARG, "max_norm=%g is negative or not finite", (double)max_norm);
    const size_t w = dtype_size(dtype), wo = dtype_size(out_dtype);
    if (out) GSR_TRY(check_list<2>({grads, out}, {w, wo}, 2u, counts, tensors, &elements));
    else GSR_TRY(check_list<1>({grads}, {w}, 1u, counts, tensors, &elements));
    if ((uintptr_t)norm_out & 3) return fail(GSR_ERR_INVALID_ARG, "norm_out is not aligned");
    GSR_TRY(check_norm_workspace(tensors, elements, workspace, workspace_bytes));
    GSR_TRY(check_apart<2>(norm_out, workspace, {grads, out ? out : grads}, {w, wo}, counts, tensors, elements));
    hipStream_t s = (hipStream_t)stream;
    ClipNorm n = launch_norm(grads, counts, tensors, dtype, norm_out, true, workspace, s);
    n.max_norm = (double)max_norm;
    const bool in_place = !out;
    over_list<2, kUpdateChunk>({grads, out ? out : grads}, {w, wo}, counts, tensors, [&](const TensorTable<2>& t) {
        const dim3 grid(t.chunks), wg(256);
        if (dtype == GSR_F32 && out_dtype == GSR_F32) hipLaunchKernelGGL((k_clip<float, float>), grid, wg, 0, s, t, n, in_place);
        else if (dtype == GSR_F32) hipLaunchKernelGGL((k_clip<float, bf16_t>), grid, wg, 0, s, t, n, in_place);
        else if (out_dtype == GSR_F32) hipLaunchKernelGGL((k_clip<bf16_t, float>), grid, wg, 0, s, t, n, in_place);
        else hipLaunchKernelGGL((k_clip<bf16_t, bf16_t>), grid, wg, 0, s, t, n, in_place);
        n.norm_out = nullptr;           // written by the first launch
    });
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

gsr_status_t gsr_adam_update_list(float* const* w, const void* const* dw, float* const* m, float* const* v, const int64_t* counts,
                                  int32_t tensors, int32_t dw_dtype, const float* norm, float max_norm, int64_t t, double lr, double beta1,
                                  double beta2, double eps, double weight_decay, void* stream) {
    int64_t elements;
    GSR_TRY(list_dtype(dw_dtype));
    if (t < 1) return fail(GSR_ERR_INVALID_ARG, "Adam's step counter starts at 1");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return fail(GSR_ERR_INVALID_ARG, "beta outside [0,1)");
    if (norm && (!(max_norm >= 0.0f) || std::isinf(max_norm)))
        return fail(GSR_ERR_INVALID_ARG, "max_norm=%g is negative or not finite", (double)max_norm);
    if ((uintptr_t)norm & 3) return fail(GSR_ERR_INVALID_ARG, "norm is not aligned");
    void* const* lists[4] = {(void* const*)w, (void* const*)dw, (void* const*)m, (void* const*)v};
    const size_t width[4] = {4, dtype_size(dw_dtype), 4, 4};
    GSR_TRY(check_list<4>(lists, width, 13u, counts, tensors, &elements));
    if (elements == 0) return GSR_OK;
    if (norm && over_tensor<4>(norm, 4, lists, width, 13u, counts, tensors)) return fail(GSR_ERR_INVALID_ARG, "norm lies in a tensor that is written");
    const double c1 = 1.0 - std::pow(beta1, (double)t), c2 = 1.0 - std::pow(beta2, (double)t);
    const AdamParams p{(float)lr, (float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2), (float)eps, (float)weight_decay,
                       (float)(1.0 / c1), (float)(1.0 / c2)};
    hipStream_t s = (hipStream_t)stream;
    over_list<4, kUpdateChunk>(lists, width, counts, tensors, [&](const TensorTable<4>& table) {
        const dim3 grid(table.chunks), wg(256);
        if (dw_dtype == GSR_F32) hipLaunchKernelGGL((k_adam_list<float>), grid, wg, 0, s, table, norm, (double)max_norm, p);
        else hipLaunchKernelGGL((k_adam_list<bf16_t>), grid, wg, 0, s, table, norm, (double)max_norm, p);
    });
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

}  // extern "C"
