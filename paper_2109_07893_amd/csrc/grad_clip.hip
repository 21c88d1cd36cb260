// The norm over all gradients of a model and the gradients scaled to at most max_norm (between the gradients of a block, Section
// "Gradient Checkpoint", and the update of the weights; recurrent models are not trained without it):
//     norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / (norm + 1e-6)).
//
// Two passes over the gradients, the second of which finds what fits the 256 MB cache there.  The tensors of a launch (their addresses
// travel with it) are one long list of stretches of 32 KB, shared out evenly whatever the tensors' sizes.  Squares are formed
// and summed in 64 bits: in 32 they are infinite from 1.8e19 on and zero below 1e-23, and a multiply-add takes no longer.  A workgroup
// of the second pass adds up the workgroups' sums by itself, in one fixed order, instead of waiting for a launch that does, while its first
// stretch is on its way.  Bound by memory: 400 M elements in nine tensors of both types (1.33 GB) take 743 us, 3.6 TB/s of one read and one
// write, 5.4 with the second read, which the norm cannot do without (240 us the squares, 485 the scaling); 46 tensors of 90 K elements 4 + 5 us.
// In place under the bound, where nothing is scaled, the second pass still reads: 432 us, of which the norm is 221.
#include <algorithm>
#include <vector>

#include "common.hpp"

namespace {

using namespace dgnn;

constexpr int kThreads = 256;
constexpr int kTensors = 112;             // tensors of a launch
constexpr int kPer = 8;                   // 16-byte pieces of a stretch that a thread has
constexpr int kPieces = kThreads * kPer;  // ... of a stretch
constexpr int kBlocks = 1024;             // workgroups of a launch that leave a sum

struct Tensors {
    const void *g[kTensors];
    void *out[kTensors];
    int64_t count[kTensors];
    int64_t first[kTensors + 1];          // stretch at which a tensor begins
    uint8_t bf16[kTensors];
    int tensors;
};
static_assert(sizeof(Tensors) <= 4000, "kernel arguments");

// Elements [from, from + count) of a tensor: `head` of them ahead of the first 16-byte boundary, `pieces` whole pieces, and what is left
// from `tail` on (fewer than a piece each; a stretch that begins between two boundaries has both).
struct Stretch {
    int k, count, head, pieces, tail;
    int64_t from;
};

// Stretch s of the list: its tensor is the last one that begins at s or ahead of it (those without elements have no stretch).  All lanes
// look at once: a search step by step would go to the argument's memory seven times in a row.
__device__ __forceinline__ Stretch stretch_of(const Tensors &t, int64_t s) {
    const int lane = threadIdx.x % kWave;
    const int below = __popcll(__ballot(lane < t.tensors && t.first[min(lane, kTensors - 1)] <= s)) +
                      __popcll(__ballot(lane + kWave < t.tensors && t.first[min(lane + kWave, kTensors - 1)] <= s));
    Stretch r;
    r.k = below - 1;
    const int size = t.bf16[r.k] ? 2 : 4, per = kPieces * (16 / size);
    r.from = (s - t.first[r.k]) * per;
    r.count = (int)min((int64_t)per, t.count[r.k] - r.from);
    const uintptr_t at = reinterpret_cast<uintptr_t>(t.g[r.k]) + r.from * size;
    r.head = min((int)((16 - (at & 15)) & 15) / size, r.count);
    r.pieces = (r.count - r.head) * size / 16;
    r.tail = r.head + r.pieces * (16 / size);
    return r;
}

// Sum over the workgroup, every thread gets it; the same order in every workgroup.
__device__ __forceinline__ double block_sum(double v, double *s_sum) {
#pragma unroll
    for (int x = 1; x < kWave; x <<= 1) v += __shfl_xor(v, x);
    if (threadIdx.x % kWave == 0) s_sum[threadIdx.x / kWave] = v;
    __syncthreads();
    v = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    __syncthreads();
    return v;
}

template <bool BF16> struct Elem;
template <> struct Elem<false> {
    typedef float Type;
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<true> {
    typedef uint16_t Type;
    static __device__ __forceinline__ float get(uint16_t v) { return bf16_to_f32(v); }
    static __device__ __forceinline__ uint16_t put(float v) { return (uint16_t)pack_bf16(v, 0.0f); }
};

template <bool BF16> __device__ __forceinline__ const typename Elem<BF16>::Type *begin_of(const Tensors &t, const Stretch &s) {
    return as_global(static_cast<const typename Elem<BF16>::Type *>(t.g[s.k])) + s.from;
}

template <bool BF16> __device__ __forceinline__ void load(uintx4 (&r)[kPer], const Tensors &t, const Stretch &s) {
    const uintx4 *p = reinterpret_cast<const uintx4 *>(begin_of<BF16>(t, s) + s.head) + threadIdx.x;
#pragma unroll
    for (int u = 0; u < kPer; ++u) r[u] = (int)threadIdx.x + u * kThreads < s.pieces ? p[u * kThreads] : uintx4{0, 0, 0, 0};
}

template <bool BF16> __device__ __forceinline__ double squares(const Tensors &t, const Stretch &s) {
    constexpr int NV = Pack<BF16>::kVals;
    const auto *g = begin_of<BF16>(t, s);
    uintx4 r[kPer];
    load<BF16>(r, t, s);
    double sum = 0.0;
    auto one = [&](int i) { const double v = Elem<BF16>::get(g[i]); sum = fma(v, v, sum); };
    if ((int)threadIdx.x < s.head) one(threadIdx.x);
    if ((int)threadIdx.x < s.count - s.tail) one(s.tail + threadIdx.x);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        float v[NV];
        Pack<BF16>::unpack(v, r[u]);
#pragma unroll
        for (int e = 0; e < NV; ++e) sum = fma((double)v[e], (double)v[e], sum);
    }
    return sum;
}

__global__ __launch_bounds__(kThreads) void grad_squares_kernel(Tensors t, double *__restrict__ sums) {
    __shared__ double s_sum[kThreads / kWave];
    double sum = 0.0;
    for (int64_t i = blockIdx.x; i < t.first[t.tensors]; i += gridDim.x) {
        const Stretch s = stretch_of(t, i);
        sum += t.bf16[s.k] ? squares<true>(t, s) : squares<false>(t, s);
    }
    sum = block_sum(sum, s_sum);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double total_of(const double *__restrict__ sums, int count, double *s_sum) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < count; i += kThreads) sum += sums[i];
    return sqrt(block_sum(sum, s_sum));
}

// F: the type of the factor and of its product with a gradient.
template <bool BF16, typename F> __device__ __forceinline__ void scaled(const uintx4 (&r)[kPer], const Tensors &t, const Stretch &s, F factor) {
    constexpr int NV = Pack<BF16>::kVals;
    typedef typename Elem<BF16>::Type E;
    const E *g = begin_of<BF16>(t, s);
    E *out = as_global(static_cast<E *>(t.out[s.k])) + s.from;
    auto one = [&](int i) { out[i] = Elem<BF16>::put((float)((F)Elem<BF16>::get(g[i]) * factor)); };
    if ((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(out)) & 15) {       // no boundary in common
        for (int i = threadIdx.x; i < s.count; i += kThreads) one(i);
        return;
    }
    if ((int)threadIdx.x < s.head) one(threadIdx.x);
    if ((int)threadIdx.x < s.count - s.tail) one(s.tail + threadIdx.x);
    uintx4 *o = reinterpret_cast<uintx4 *>(out + s.head) + threadIdx.x;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        float v[NV];
        Pack<BF16>::unpack(v, r[u]);
#pragma unroll
        for (int e = 0; e < NV; ++e) v[e] = (float)((F)v[e] * factor);
        if ((int)threadIdx.x + u * kThreads < s.pieces) o[u * kThreads] = Pack<BF16>::pack(v);
    }
}

__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Tensors t, const double *__restrict__ sums, int count, double max_norm, float *__restrict__ norm) {
    __shared__ double s_sum[kThreads / kWave];
    const int64_t stretches = t.first[t.tensors];
    // from the end: what the first pass read last is what the cache still has
    int64_t i = stretches - 1 - blockIdx.x;
    Stretch s;
    uintx4 r[kPer];
    auto fetch = [&]() {
        s = stretch_of(t, i);
        if (t.bf16[s.k]) load<true>(r, t, s); else load<false>(r, t, s);
    };
    if (i >= 0) fetch();
    const double total = total_of(sums, count, s_sum);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    const double most = max_norm / (total + 1e-6);
    const bool clip = isfinite((float)total) && most < 1.0;  // a norm that *norm shows as no finite number: nothing to scale by
    const float factor = clip ? (float)most : 1.0f;
    // A factor below the normal numbers of 32 bits keeps few of its digits there, or none, where its product with a large gradient has all of them.
    const bool small = clip && most < 0x1p-126;
    while (i >= 0) {
        if (small) {
            if (t.bf16[s.k]) scaled<true>(r, t, s, most); else scaled<false>(r, t, s, most);
        } else if (clip || t.out[s.k] != t.g[s.k]) {
            if (t.bf16[s.k]) scaled<true>(r, t, s, factor); else scaled<false>(r, t, s, factor);
        }
        i -= gridDim.x;
        if (i >= 0) fetch();
    }
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double *__restrict__ sums, int count, float *__restrict__ norm) {
    __shared__ double s_sum[kThreads / kWave];
    const double total = total_of(sums, count, s_sum);
    if (threadIdx.x == 0) *norm = (float)total;
}

size_t size_of(const dgnn_grad_item &i) { return (size_t)i.count * (i.dt == DGNN_BF16 ? 2 : 4); }

int check(int32_t count, const dgnn_grad_item *items) {
    if (!items) return DGNN_ERR_NULL;
    if (count <= 0) return DGNN_ERR_SHAPE;
    for (int32_t i = 0; i < count; ++i) {
        if (items[i].count < 0 || (items[i].dt != DGNN_F32 && items[i].dt != DGNN_BF16)) return DGNN_ERR_SHAPE;
        if (items[i].count > (int64_t(1) << 40)) return DGNN_ERR_OVERFLOW;
    }
    return DGNN_OK;
}

int launches_of(int32_t count) { return (count + kTensors - 1) / kTensors; }

// What both passes are given of the items [from, from + kTensors).
Tensors tensors_of(int32_t count, const dgnn_grad_item *items, int32_t from) {
    Tensors t;
    t.tensors = std::min(kTensors, count - from);
    t.first[0] = 0;
    for (int i = 0; i < t.tensors; ++i) {
        const dgnn_grad_item &it = items[from + i];
        t.g[i] = it.g;
        t.out[i] = it.out;
        t.count[i] = it.count;
        t.bf16[i] = it.dt == DGNN_BF16;
        const int64_t per = (int64_t)kPieces * (it.dt == DGNN_BF16 ? 8 : 4);
        t.first[i + 1] = t.first[i] + (it.count + per - 1) / per;
    }
    return t;
}

int enqueue_squares(int32_t count, const dgnn_grad_item *items, double *sums, int &left, hipStream_t st) {
    left = 0;
    for (int32_t i = 0; i < count; i += kTensors) {
        const Tensors t = tensors_of(count, items, i);
        const int blocks = (int)std::min<int64_t>(kBlocks, std::max<int64_t>(t.first[t.tensors], 1));
        hipLaunchKernelGGL(grad_squares_kernel, dim3(blocks), dim3(kThreads), 0, st, t, sums + left);
        DGNN_RETURN_IF_LAUNCH_FAILED();
        left += blocks;
    }
    return DGNN_OK;
}

// Addresses: `out` = whether the gradients are written.  What is written (the norm and the sums too) meets nothing else that is written,
// and nothing that is read but, exactly, its own gradient.
int check_pointers(int32_t count, const dgnn_grad_item *items, bool out, const float *norm, const void *ws, size_t ws_bytes) {
    struct Range { uintptr_t from, to; int32_t item; };
    auto address = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if (!aligned16(ws) || address(norm) % sizeof(float)) return DGNN_ERR_ALIGN;
    for (int32_t i = 0; i < count; ++i) {
        const dgnn_grad_item &it = items[i];
        if (it.count == 0) continue;
        if (!it.g || (out && !it.out)) return DGNN_ERR_NULL;
        const size_t step = it.dt == DGNN_BF16 ? 2 : 4;
        if (address(it.g) % step || (out && address(it.out) % step)) return DGNN_ERR_ALIGN;
    }
    try {
        std::vector<Range> written{{address(ws), address(ws) + ws_bytes, -1}, {address(norm), address(norm) + sizeof(float), -1}};
        for (int32_t i = 0; out && i < count; ++i)
            if (items[i].count) written.push_back({address(items[i].out), address(items[i].out) + size_of(items[i]), i});
        std::sort(written.begin(), written.end(), [](const Range &a, const Range &b) { return a.from < b.from; });
        for (size_t i = 1; i < written.size(); ++i)
            if (written[i].from < written[i - 1].to) return DGNN_ERR_ALIAS;
        for (int32_t i = 0; i < count; ++i) {
            if (items[i].count == 0) continue;
            const uintptr_t from = address(items[i].g), to = from + size_of(items[i]);
            // the writes lie apart, so their ends are in order too: the first one that ends behind this gradient's start
            auto w = std::upper_bound(written.begin(), written.end(), from, [](uintptr_t at, const Range &b) { return at < b.to; });
            for (; w != written.end() && w->from < to; ++w)
                if (w->item != i || w->from != from) return DGNN_ERR_ALIAS;
        }
    } catch (...) {                       // no host memory for the lists
        return DGNN_ERR_CAPACITY;
    }
    return DGNN_OK;
}

}  // namespace

extern "C" int dgnn_grad_clip_workspace(int32_t count, size_t *bytes) {
    if (!bytes) return DGNN_ERR_NULL;
    if (count <= 0) return DGNN_ERR_SHAPE;
    *bytes = (size_t)launches_of(count) * kBlocks * sizeof(double);
    return DGNN_OK;
}

extern "C" int dgnn_grad_norm(int32_t count, const dgnn_grad_item *items, float *norm, void *ws, size_t ws_bytes, void *stream) {
    if (!norm || !ws) return DGNN_ERR_NULL;
    if (int rc = check(count, items)) return rc;
    if (int rc = check_pointers(count, items, false, norm, ws, ws_bytes)) return rc;
    if (ws_bytes < (size_t)launches_of(count) * kBlocks * sizeof(double)) return DGNN_ERR_CAPACITY;
    hipStream_t st = (hipStream_t)stream;
    int left = 0;
    if (int rc = enqueue_squares(count, items, static_cast<double *>(ws), left, st)) return rc;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kThreads), 0, st, static_cast<const double *>(ws), left, norm);
    DGNN_RETURN_IF_LAUNCH_FAILED();
    return DGNN_OK;
}

extern "C" int dgnn_grad_clip(int32_t count, const dgnn_grad_item *items, double max_norm, float *norm, void *ws, size_t ws_bytes, void *stream) {
    if (!norm || !ws) return DGNN_ERR_NULL;
    if (int rc = check(count, items)) return rc;
    if (!(max_norm > 0.0)) return DGNN_ERR_SHAPE;
    if (int rc = check_pointers(count, items, true, norm, ws, ws_bytes)) return rc;
    if (ws_bytes < (size_t)launches_of(count) * kBlocks * sizeof(double)) return DGNN_ERR_CAPACITY;
    hipStream_t st = (hipStream_t)stream;
    double *sums = static_cast<double *>(ws);
    int left = 0;
    if (int rc = enqueue_squares(count, items, sums, left, st)) return rc;
    for (int32_t i = 0; i < count; i += kTensors) {
        const Tensors t = tensors_of(count, items, i);
        const int blocks = (int)std::min<int64_t>(2 * kBlocks, std::max<int64_t>(t.first[t.tensors], 1));
        hipLaunchKernelGGL(grad_scale_kernel, dim3(blocks), dim3(kThreads), 0, st, t, (const double *)sums, left, max_norm, i == 0 ? norm : nullptr);
        DGNN_RETURN_IF_LAUNCH_FAILED();
    }
    return DGNN_OK;
}
