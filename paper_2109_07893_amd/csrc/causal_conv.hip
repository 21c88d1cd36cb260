// Causal convolution over time, one short filter per channel, and its adjoint (beside the M-transform, Section "TM-GCN", whose weights
// are the same for all channels and set by the window):
//     a[t] = bias + sum_{j<w} taps[j] x[t-j],  y[t] = a[t] or silu(a[t]);   frames ahead of the series are x_before's, or zero.
// Going back, with ga[t] = g_y[t] (silu'(a[t]) or 1):  dx[s] = sum_j taps[j] ga[s+j],  dtaps[j] = sum ga[t] x[t-j],  dbias = sum ga.
//
// Like the M-transform a lane owns one piece of a row and walks the time axis with the last w - 1 frames in registers, so that every
// frame is read and written once.  Few rows are shared out along the time axis too; a piece of it reads w - 1 frames ahead of it again
// (and, going back, w - 1 frames behind it, whose pre-activations it forms once more).
#include <algorithm>
#include <initializer_list>
#include <utility>

#include "common.hpp"

namespace {

using namespace dgnn;

constexpr int kThreads = 256;
constexpr int kMaxGrid = 1 << 22;         // workgroups of a launch: HIP counts its threads in 32 bits
constexpr int kAhead = 4;                 // frames fetched together
constexpr int kLeast = 16;                // timesteps of a piece of the time axis, at least
constexpr int64_t kMostPieces = 1 << 15;  // ... of which a launch has no more
constexpr int kBackBlocks = 1024;         // workgroups of the adjoint, each of which leaves sums
constexpr int kFlush = 64;                // timesteps summed up before they join the sums of the walk

struct Conv {
    const void *x, *x_before;
    const float *taps, *bias;
    void *y, *x_after;
    const int32_t *lengths;
    int64_t n, row_blocks;
    int T, f, ppr;                        // pieces per row
    int cols, rows_per_block;             // a row's pieces in `cols` parts of at most kThreads; rows of a workgroup
    int chunk, pieces;                    // the time axis in `pieces` pieces of `chunk` timesteps
};

struct ConvBack {
    Conv c;
    const void *g_y, *dx_after;
    void *dx, *dx_before;
    float *sums;                          // [slots][w + 1][f]
};

__device__ __forceinline__ int length_of(const int32_t *lengths, int64_t v, int T) { return lengths ? min(max(lengths[v], 0), T) : T; }

__device__ __forceinline__ float sigmoid_of(float a) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a * -1.44269504088896340736f)); }

// N consecutive parameters from p on, N and p's place among them multiples of four: `base` needs the alignment of a float only.
template <int N> __device__ __forceinline__ void load_parameters(float (&v)[N], const float *base, const float *p) {
    if ((reinterpret_cast<uintptr_t>(base) & 15) == 0) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const float4 t = *reinterpret_cast<const float4 *>(p + e);
            v[e] = t.x; v[e + 1] = t.y; v[e + 2] = t.z; v[e + 3] = t.w;
        }
    } else
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = p[e];
}

// ---- forward: pieces of 16 bytes ------------------------------------------------------------------------------------
// Bound by memory: 16 x 150001 x 64 bf16, four taps: 141 us for 0.73 GB, 5.2 TB/s.  Two frames fetched together instead of four: 7.2 us for 6.8
// at 32 x 512 x 128 fp32, 101 for 108 at 64 x 16384 x 64.
template <bool BF16, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_kernel(Conv c) {
    constexpr int NV = Pack<BF16>::kVals;
    const uintx4 *const x = static_cast<const uintx4 *>(c.x), *const before = static_cast<const uintx4 *>(c.x_before);
    uintx4 *const y = static_cast<uintx4 *>(c.y), *const after = static_cast<uintx4 *>(c.x_after);
    const int per = c.cols > 1 ? kThreads : c.ppr;
    const int col = blockIdx.x % c.cols, k = col * kThreads + threadIdx.x % per, sub = threadIdx.x / per;
    if (k >= c.ppr || sub >= c.rows_per_block) return;
    const int t0 = blockIdx.y * c.chunk, t1 = min(c.T, t0 + c.chunk);
    const int64_t frame = c.n * c.ppr;
    float taps[W][NV], bias[NV];
#pragma unroll
    for (int j = 0; j < W; ++j) load_parameters<NV>(taps[j], c.taps, c.taps + (int64_t)j * c.f + k * NV);
    if (c.bias) load_parameters<NV>(bias, c.bias, c.bias + (int64_t)k * NV);
    else
#pragma unroll
        for (int e = 0; e < NV; ++e) bias[e] = 0.0f;
    for (int64_t rb = blockIdx.x / c.cols; rb < c.row_blocks; rb += gridDim.x / c.cols) {
        const int64_t v = rb * c.rows_per_block + sub;
        if (v >= c.n) break;
        const int64_t at = v * c.ppr + k;
        const int len = length_of(c.lengths, v, c.T), t_end = min(t1, len);
        float ring[W][NV];                                   // ring[j] = x[t - j]
#pragma unroll
        for (int j = 1; j < W; ++j) {
            const int t = t0 - j;
            uintx4 r = {0, 0, 0, 0};
            if (t >= 0) r = x[t * frame + at];
            else if (before) r = before[(W - 1 + t) * frame + at];
            Pack<BF16>::unpack(ring[j - 1], r);
        }
        for (int t = t0; t < t_end; t += kAhead) {
            uintx4 next[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (t + i < t_end) next[i] = x[(t + i) * frame + at];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (t + i < t_end) {
#pragma unroll
                    for (int j = W - 1; j > 0; --j)
#pragma unroll
                        for (int e = 0; e < NV; ++e) ring[j][e] = ring[j - 1][e];
                    Pack<BF16>::unpack(ring[0], next[i]);
                    float out[NV];
#pragma unroll
                    for (int e = 0; e < NV; ++e) {
                        float a = bias[e];
#pragma unroll
                        for (int j = 0; j < W; ++j) a = fmaf(taps[j][e], ring[j][e], a);
                        out[e] = SILU ? a * sigmoid_of(a) : a;
                    }
                    y[(t + i) * frame + at] = Pack<BF16>::pack(out);
                }
        }
        for (int t = max(t0, t_end); t < t1; ++t) y[t * frame + at] = uintx4{0, 0, 0, 0};
        // The last W - 1 frames of the sequence.  x_after may be x_before: this lane alone has its piece, and only the first piece of the time
        // axis reads x_before.  Where that is all there is the frames are in the ring; else they are read again, frame j from a place that
        // is not yet written.
        if (after && blockIdx.y == 0)
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int t = len - (W - 1) + j;
                uintx4 r = {0, 0, 0, 0};
                if (c.pieces == 1) r = Pack<BF16>::pack(ring[W - 2 - j]);
                else if (t >= 0) r = x[t * frame + at];
                else if (before) r = before[(W - 1 + t) * frame + at];
                after[j * frame + at] = r;
            }
    }
}

// ---- backward: four values a lane, whatever they are stored in ------------------------------------------------------------
// Eight of bf16 would need twice the registers of ring, derivatives and sums.  Bound by memory: 24 x 60013 x 128 fp32, three taps, ragged: 398 us with the
// sums, 4.75 TB/s.  Half the workgroups: 643 us for 484 at 32 x 50000 x 128; twice as many: 497.
template <bool BF16> struct Four;
template <> struct Four<false> {
    typedef uintx4 Raw;
    static __device__ __forceinline__ void unpack(float (&v)[4], Raw r) { Pack<false>::unpack(v, r); }
    static __device__ __forceinline__ Raw pack(const float (&v)[4]) { return Pack<false>::pack(v); }
    static __device__ __forceinline__ Raw zero() { return Raw{0, 0, 0, 0}; }
};
template <> struct Four<true> {
    typedef uint2 Raw;
    static __device__ __forceinline__ void unpack(float (&v)[4], Raw r) {
        v[0] = __uint_as_float(r.x << 16); v[1] = __uint_as_float(r.x & 0xffff0000u);
        v[2] = __uint_as_float(r.y << 16); v[3] = __uint_as_float(r.y & 0xffff0000u);
    }
    static __device__ __forceinline__ Raw pack(const float (&v)[4]) { return make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])); }
    static __device__ __forceinline__ Raw zero() { return make_uint2(0, 0); }
};

template <bool BF16, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_back_kernel(ConvBack b) {
    typedef typename Four<BF16>::Raw Raw;
    const Conv &c = b.c;
    __shared__ float s_sum[kThreads][4];
    const Raw *const x = static_cast<const Raw *>(c.x), *const before = static_cast<const Raw *>(c.x_before), *const gy = static_cast<const Raw *>(b.g_y);
    const Raw *const d_after = static_cast<const Raw *>(b.dx_after);
    Raw *const dx = static_cast<Raw *>(b.dx), *const d_before = static_cast<Raw *>(b.dx_before);
    const int per = c.cols > 1 ? kThreads : c.ppr;
    const int col = blockIdx.x % c.cols, k = col * kThreads + threadIdx.x % per, sub = threadIdx.x / per;
    const int slot = blockIdx.x / c.cols, slots = gridDim.x / c.cols;
    const bool mine = k < c.ppr && sub < c.rows_per_block;
    const int64_t frame = c.n * c.ppr;
    float taps[W][4], bias[4], sums[W + 1][4];
    const int place = mine ? k : 0;
#pragma unroll
    for (int j = 0; j < W; ++j) load_parameters<4>(taps[j], c.taps, c.taps + (int64_t)j * c.f + place * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        bias[e] = 0.0f;
#pragma unroll
        for (int j = 0; j <= W; ++j) sums[j][e] = 0.0f;
    }
    if (c.bias) load_parameters<4>(bias, c.bias, c.bias + (int64_t)place * 4);
    for (int64_t item = slot; mine && item < c.row_blocks * c.pieces; item += slots) {
        const int64_t v = item / c.pieces * c.rows_per_block + sub;
        if (v >= c.n) continue;
        const int p = (int)(item % c.pieces), t0 = p * c.chunk, t1 = min(c.T, t0 + c.chunk);
        const int64_t at = v * c.ppr + k;
        const int len = length_of(c.lengths, v, c.T);
        float ring[W][4], ga[W][4], part[W + 1][4];          // ring[j] = x[t - j], ga[j] = ga[t - j]
#pragma unroll
        for (int j = 0; j < W; ++j) {
            Raw r = Four<BF16>::zero();
            const int t = t0 - 1 - j;
            if (j < W - 1) {
                if (t >= 0) r = x[t * frame + at];
                else if (before) r = before[(W - 1 + t) * frame + at];
            }
            Four<BF16>::unpack(ring[j], r);
#pragma unroll
            for (int e = 0; e < 4; ++e) ga[j][e] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j <= W; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[j][e] = 0.0f;
        // frame s = t - (W - 1) is complete when ga[t] is there; frames ahead of the series are x_before's
        const int last = t1 + W - 1, first_out = p == 0 ? -(W - 1) : t0;
        for (int t = t0; t < last; t += 2) {
            Raw xr[2], gr[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                xr[i] = gr[i] = Four<BF16>::zero();
                if (t + i < len && t + i < last) { xr[i] = x[(t + i) * frame + at]; gr[i] = gy[(t + i) * frame + at]; }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (t + i >= last) break;
#pragma unroll
                for (int j = W - 1; j > 0; --j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) { ring[j][e] = ring[j - 1][e]; ga[j][e] = ga[j - 1][e]; }
                Four<BF16>::unpack(ring[0], xr[i]);
                Four<BF16>::unpack(ga[0], gr[i]);
                if (SILU && t + i < len)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float a = bias[e];
#pragma unroll
                        for (int j = 0; j < W; ++j) a = fmaf(taps[j][e], ring[j][e], a);
                        const float sig = sigmoid_of(a);
                        ga[0][e] *= sig * fmaf(a, 1.0f - sig, 1.0f);
                    }
                if (t + i < t1 && t + i < len)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
#pragma unroll
                        for (int j = 0; j < W; ++j) part[j][e] = fmaf(ga[0][e], ring[j][e], part[j][e]);
                        part[W][e] += ga[0][e];
                    }
                const int s = t + i - (W - 1);
                if (s >= first_out && s < t1) {
                    float out[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        out[e] = 0.0f;
#pragma unroll
                        for (int j = 0; j < W; ++j) out[e] = fmaf(taps[j][e], ga[W - 1 - j][e], out[e]);
                    }
                    const int back = s - (len - (W - 1));     // the frame's place among those handed on
                    if (d_after && back >= 0 && back < W - 1) {
                        float more[4];
                        Four<BF16>::unpack(more, d_after[back * frame + at]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) out[e] += more[e];
                    }
                    if (s >= 0) dx[s * frame + at] = Four<BF16>::pack(out);
                    else if (d_before) d_before[(W - 1 + s) * frame + at] = Four<BF16>::pack(out);
                }
            }
            if (((t - t0) & (kFlush - 1)) == kFlush - 2 || t + 2 >= last)
#pragma unroll
                for (int j = 0; j <= W; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) { sums[j][e] += part[j][e]; part[j][e] = 0.0f; }
        }
    }
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) s_sum[threadIdx.x][e] = sums[j][e];
        __syncthreads();
        if (mine && sub == 0) {                               // the rows of a workgroup in order
            float total[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) total[e] = sums[j][e];
            for (int r = 1; r < c.rows_per_block; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) total[e] += s_sum[r * per + threadIdx.x][e];
#pragma unroll
            for (int e = 0; e < 4; ++e) b.sums[((int64_t)slot * (W + 1) + j) * c.f + k * 4 + e] = total[e];
        }
    }
}

// dtaps | dbias from the workgroups' sums: 64 strided parts of them, in 64 bits, in a fixed order.
__global__ __launch_bounds__(1024) void conv_sums_kernel(const float *__restrict__ sums, int slots, int width, int taps, float *__restrict__ dtaps, float *__restrict__ dbias,
                                                         int accumulate) {
    __shared__ double s_part[64][17];
    const int o = threadIdx.x % 16, r = threadIdx.x / 16, at = blockIdx.x * 16 + o;
    double sum = 0.0;
    if (at < width)
#pragma unroll 4
        for (int k = r; k < slots; k += 64) sum += (double)sums[(int64_t)k * width + at];
    s_part[r][o] = sum;
    __syncthreads();
    if (r == 0 && at < width) {
#pragma unroll 7
        for (int k = 1; k < 64; ++k) sum += s_part[k][o];
        float *to = at < taps ? dtaps + at : dbias ? dbias + (at - taps) : nullptr;
        if (to) *to = accumulate ? (float)((double)*to + sum) : (float)sum;
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------
int check(int64_t T, int64_t n, int32_t f, int32_t w) {
    if (T <= 0 || n <= 0 || f < 16 || f % 16 || f > DGNN_MAX_CHANNELS || w < 2 || w > 4) return DGNN_ERR_SHAPE;
    if (!fits_index(n) || T > (int64_t(1) << 30) || T > (int64_t(1) << 44) / n) return DGNN_ERR_OVERFLOW;   // a place behind the last piece still is an int
    return DGNN_OK;
}

// `lanes` = values of a lane; `wanted` = lanes that should have work before the time axis stays whole.
void shape_of(Conv &c, int64_t T, int64_t n, int32_t f, int lanes, int64_t wanted) {
    c.T = (int)T; c.n = n; c.f = f;
    c.ppr = f / lanes;
    c.cols = (c.ppr + kThreads - 1) / kThreads;
    c.rows_per_block = c.cols > 1 ? 1 : kThreads / c.ppr;
    c.row_blocks = (n + c.rows_per_block - 1) / c.rows_per_block;
    const int64_t pieces = std::max<int64_t>(1, std::min<int64_t>({T / kLeast, wanted / (n * c.ppr), kMostPieces}));
    c.chunk = (int)((T + pieces - 1) / pieces);
    c.pieces = (int)((T + c.chunk - 1) / c.chunk);
}

int64_t back_slots(const Conv &c) { return std::min<int64_t>(c.row_blocks * c.pieces, std::max(1, kBackBlocks / c.cols)); }

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const char *p = static_cast<const char *>(a), *q = static_cast<const char *>(b);
    return p && q && p < q + nb && q < p + na;
}

// Parameters, their gradients and lengths: 32-bit numbers at any address that those may have.
bool words_aligned(std::initializer_list<const void *> words) {
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) % 4) return false;
    return true;
}

// Lanes with work before the time axis stays whole, half of what the device holds at once: pieces read frames twice (64 x 16384 x 64 fp32 going
// back: 156 us whole, 179 in four pieces), fewer lanes leave loads unissued (128 x 8192 x 64 bf16 going back: 86 us with 2^18 lanes, 118 with 2^17).
constexpr int64_t kWanted = 1 << 18;

}  // namespace

extern "C" int dgnn_causal_conv(const void *x, const float *taps, const float *bias, const void *x_before, void *y, void *x_after, const int32_t *lengths, int64_t T,
                                int64_t n, int32_t f, int32_t w, uint32_t flags, dgnn_dtype dt, void *stream) {
    if (!x || !taps || !y) return DGNN_ERR_NULL;
    if (int rc = check(T, n, f, w)) return rc;
    if ((dt != DGNN_F32 && dt != DGNN_BF16) || (flags & ~DGNN_SILU)) return DGNN_ERR_SHAPE;
    for (const void *p : {x, x_before, (const void *)y, (const void *)x_after})
        if (p && !aligned16(p)) return DGNN_ERR_ALIGN;
    if (!words_aligned({taps, bias, lengths})) return DGNN_ERR_ALIGN;
    const size_t row = (size_t)n * f * (dt == DGNN_F32 ? 4 : 2), all = row * T, edge = row * (w - 1);
    for (auto o : {std::pair<const void *, size_t>{y, all}, {x_after, edge}})
        if (overlap(o.first, o.second, taps, sizeof(float) * w * f) || overlap(o.first, o.second, bias, sizeof(float) * f) ||
            overlap(o.first, o.second, lengths, sizeof(int32_t) * n))
            return DGNN_ERR_ALIAS;
    if (overlap(y, all, x, all) || overlap(y, all, x_before, edge) || overlap(y, all, x_after, edge) || overlap(x_after, edge, x, all) ||
        (x_after != x_before && overlap(x_after, edge, x_before, edge)))
        return DGNN_ERR_ALIAS;
    Conv c{x, x_before, taps, bias, y, x_after, lengths};
    shape_of(c, T, n, f, dt == DGNN_F32 ? 4 : 8, kWanted);
    const int64_t blocks = std::min<int64_t>(c.row_blocks, std::max(1, kMaxGrid / (c.pieces * c.cols)));
    const dim3 grid((unsigned)(blocks * c.cols), (unsigned)c.pieces);
    hipStream_t st = (hipStream_t)stream;
    auto launch = [&](auto plain, auto silu) {
        if (flags & DGNN_SILU) hipLaunchKernelGGL(silu, grid, dim3(kThreads), 0, st, c);
        else hipLaunchKernelGGL(plain, grid, dim3(kThreads), 0, st, c);
    };
    if (dt == DGNN_BF16) {
        if (w == 2) launch(conv_kernel<true, 2, false>, conv_kernel<true, 2, true>);
        else if (w == 3) launch(conv_kernel<true, 3, false>, conv_kernel<true, 3, true>);
        else launch(conv_kernel<true, 4, false>, conv_kernel<true, 4, true>);
    } else {
        if (w == 2) launch(conv_kernel<false, 2, false>, conv_kernel<false, 2, true>);
        else if (w == 3) launch(conv_kernel<false, 3, false>, conv_kernel<false, 3, true>);
        else launch(conv_kernel<false, 4, false>, conv_kernel<false, 4, true>);
    }
    DGNN_RETURN_IF_LAUNCH_FAILED();
    return DGNN_OK;
}

extern "C" int dgnn_causal_conv_backward_workspace(int64_t T, int64_t n, int32_t f, int32_t w, size_t *bytes) {
    if (!bytes) return DGNN_ERR_NULL;
    if (int rc = check(T, n, f, w)) return rc;
    Conv c{};
    shape_of(c, T, n, f, 4, kWanted);
    *bytes = (size_t)back_slots(c) * (w + 1) * f * sizeof(float);
    return DGNN_OK;
}

extern "C" int dgnn_causal_conv_backward(const void *x, const float *taps, const float *bias, const void *x_before, const void *g_y, const void *dx_after, void *dx,
                                         void *dx_before, float *dtaps, float *dbias, const int32_t *lengths, int64_t T, int64_t n, int32_t f, int32_t w, uint32_t flags,
                                         int32_t accumulate, dgnn_dtype dt, void *ws, size_t ws_bytes, void *stream) {
    if (!x || !taps || !g_y || !dx || !dtaps || !ws || (bias && !dbias)) return DGNN_ERR_NULL;
    if (int rc = check(T, n, f, w)) return rc;
    if ((dt != DGNN_F32 && dt != DGNN_BF16) || (flags & ~DGNN_SILU)) return DGNN_ERR_SHAPE;
    for (const void *p : {x, x_before, g_y, dx_after, (const void *)dx, (const void *)dx_before, (const void *)ws})
        if (p && !aligned16(p)) return DGNN_ERR_ALIGN;
    if (!words_aligned({taps, bias, lengths, dtaps, dbias})) return DGNN_ERR_ALIGN;
    size_t need = 0;
    dgnn_causal_conv_backward_workspace(T, n, f, w, &need);
    if (ws_bytes < need) return DGNN_ERR_CAPACITY;
    const size_t row = (size_t)n * f * (dt == DGNN_F32 ? 4 : 2), all = row * T, edge = row * (w - 1);
    const size_t parameters = sizeof(float) * w * f, vector = sizeof(float) * f;
    const std::pair<const void *, size_t> in[] = {{x, all}, {x_before, edge}, {g_y, all}, {dx_after, edge}, {taps, parameters}, {bias, vector}, {lengths, sizeof(int32_t) * n}};
    const std::pair<const void *, size_t> out[] = {{dx, all}, {dx_before, edge}, {ws, ws_bytes}, {dtaps, parameters}, {dbias, vector}};
    for (size_t i = 0; i < sizeof(out) / sizeof(*out); ++i) {
        for (auto o : in)
            if (overlap(out[i].first, out[i].second, o.first, o.second)) return DGNN_ERR_ALIAS;
        for (size_t k = 0; k < i; ++k)
            if (overlap(out[i].first, out[i].second, out[k].first, out[k].second)) return DGNN_ERR_ALIAS;
    }
    ConvBack b{};
    b.c = Conv{x, x_before, taps, bias, nullptr, nullptr, lengths};
    shape_of(b.c, T, n, f, 4, kWanted);
    b.g_y = g_y; b.dx_after = dx_after; b.dx = dx; b.dx_before = dx_before;
    b.sums = static_cast<float *>(ws);
    const int slots = (int)back_slots(b.c);
    hipStream_t st = (hipStream_t)stream;
    auto launch = [&](auto plain, auto silu) {
        const dim3 grid((unsigned)(slots * b.c.cols));
        if (flags & DGNN_SILU) hipLaunchKernelGGL(silu, grid, dim3(kThreads), 0, st, b);
        else hipLaunchKernelGGL(plain, grid, dim3(kThreads), 0, st, b);
    };
    if (dt == DGNN_BF16) {
        if (w == 2) launch(conv_back_kernel<true, 2, false>, conv_back_kernel<true, 2, true>);
        else if (w == 3) launch(conv_back_kernel<true, 3, false>, conv_back_kernel<true, 3, true>);
        else launch(conv_back_kernel<true, 4, false>, conv_back_kernel<true, 4, true>);
    } else {
        if (w == 2) launch(conv_back_kernel<false, 2, false>, conv_back_kernel<false, 2, true>);
        else if (w == 3) launch(conv_back_kernel<false, 3, false>, conv_back_kernel<false, 3, true>);
        else launch(conv_back_kernel<false, 4, false>, conv_back_kernel<false, 4, true>);
    }
    DGNN_RETURN_IF_LAUNCH_FAILED();
    const int width = (w + 1) * f;
    hipLaunchKernelGGL(conv_sums_kernel, dim3((unsigned)((width + 15) / 16)), dim3(1024), 0, st, b.sums, slots, width, w * f, dtaps, dbias, accumulate);
    DGNN_RETURN_IF_LAUNCH_FAILED();
    return DGNN_OK;
}
