// Selective state-space scan over a series of timesteps, and its adjoint: a temporal layer beside the LSTM (Section "CD-GCN") whose
// recurrence is linear in its state and gated by its input.  Per sequence v, channel c and state s
//     dt = softplus(delta[t][v][c] + dt_bias[c]),   e = exp(dt a[c][s]),   h = e h + dt x[t][v][c] B[t][v][s],
//     y[t][v][c] = (sum_s C[t][v][s] h[c][s] + d[c] x[t][v][c]) silu(z[t][v][c])
// and going back, with g = g_y silu(z) and k = dL/dh as it comes from the timestep behind,
//     gh = k + C g,   dC += h g,   dB += gh dt x,   dx = d g + dt sum_s gh B,   u = gh e,   k <- u,
//     d(dt) = sum_s u h_before a + x sum_s gh B,   da += u h_before dt,   ddelta = d(dt) sig(delta + dt_bias).
//
// A wavefront owns sixteen channels of one sequence and walks the time axis; four lanes share a channel and hold a quarter of its
// states each, in registers.  Timesteps go by fours: lane q of a channel loads x, delta and z of timestep 4 i + q and forms dt for it,
// so that nothing is loaded or computed twice, and the four hand their values round with quad permutations, which are operand
// modifiers.  Sums over a channel's states stay inside the four lanes; four timesteps' sums are exchanged at once and end in the lane
// whose timestep they are.  Sums over channels (dB, dC) run across the sixteen groups of four, again many at a time, so that every step
// of the exchange halves the number of registers; the wavefronts of a sequence then meet in LDS.
#include <algorithm>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "common.hpp"

namespace {

using namespace dgnn;

constexpr int kChannels = 16;             // channels of a wavefront
constexpr int kTile = 16;                 // timesteps between two kept states (and of a piece of the time axis at least)
constexpr int kWaves = 4;                 // wavefronts of a workgroup of the kernels without sums over channels
constexpr int kBackWaves = 8;             // ... of the adjoint, at most
constexpr int kMaxGrid = 1 << 22;         // workgroups of a launch: HIP counts its threads in 32 bits
constexpr int kMaxSlots = 1024;           // workgroups of the adjoint that leave sums over time and sequences
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eLow = 1.92596299112661746887e-8f;
constexpr float kLn2 = 0.693147180559945309417f;

struct Scan {
    const void *x, *delta, *bc, *z;
    const float *a, *d, *dt_bias, *h_before;
    void *y;
    float *h_after, *checkpoints;
    const int32_t *lengths;
    int64_t n;
    int T, f, groups;                     // groups of kChannels channels
    int chunk, pieces;                    // the time axis in `pieces` pieces of `chunk` timesteps, a multiple of kTile
    float *piece_state, *piece_time;      // [pieces][n][f][N], [pieces][n][f]
};

struct ScanBack {
    Scan s;
    const void *g_y;
    const float *dh_after;
    void *dx, *ddelta, *dbc, *dz;
    float *dh_before;
    float *dbc_part;                      // [blocks of channel groups][T][n][2 N], where a sequence has more than one workgroup
    double *sums;                         // [slots][f (N + 2)]: da, dd, ddt_bias
    int blocks_of_groups, sequences;      // workgroups of a sequence; sequences of a workgroup
};

// ---- arithmetic ---------------------------------------------------------------------------------------------------
// 2^x and 1 / x by the hardware's instructions, 1 unit in the last place each.
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_of(float x) { return __builtin_amdgcn_rcpf(x); }

// exp(v) for v <= 0 with the product v log2(e) in two parts: the error of a rounded product grows with |v| otherwise.
__device__ __forceinline__ float exp_of(float v) {
    const float p = v * kLog2e, e = exp2_of(p);
    const float low = fmaf(v, kLog2eLow, fmaf(v, kLog2e, -p));
    return p < -160.0f ? 0.0f : fmaf(e, low * kLn2, e);
}

// softplus(v) = max(v, 0) + log(1 + e), e = exp(-|v|), and sig(v).  log(1 + e) = 2 artanh(e / (2 + e)) by its power series: the argument
// is at most 1/3, eight terms leave 1.4e-9 of the result, and a small e loses no digits, which 1 + e would.
__device__ __forceinline__ float softplus_of(float v, float &sig) {
    const float e = exp_of(-fabsf(v));
    const float r = e * rcp_of(2.0f + e), q = r * r;
    float p = fmaf(q, 1.0f / 15, 1.0f / 13);
    p = fmaf(p, q, 1.0f / 11);
    p = fmaf(p, q, 1.0f / 9);
    p = fmaf(p, q, 1.0f / 7);
    p = fmaf(p, q, 1.0f / 5);
    p = fmaf(p, q, 1.0f / 3);
    p = fmaf(p, q, 1.0f);
    sig = (v >= 0.0f ? 1.0f : e) * rcp_of(1.0f + e);
    return fmaxf(v, 0.0f) + 2.0f * r * p;
}
__device__ __forceinline__ float sigmoid_of(float v) { return rcp_of(1.0f + exp2_of(-v * kLog2e)); }

// ---- lanes --------------------------------------------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// The value of lane J of the four.
template <int J> __device__ __forceinline__ float of_lane(float v) { return dpp<J * 0x55>(v); }

__device__ __forceinline__ float quad_sum(float v) {
    v += dpp<0xb1>(v);
    return v + dpp<0x4e>(v);
}

// Lane q of the four gets the sum over the four of v[q]: an exchange with the lane two further leaves two values, one with the
// neighbour the last.
__device__ __forceinline__ float quad_sums(const float (&v)[4], int q) {
    const bool hi = q & 2, odd = q & 1;
    const float a = (hi ? v[2] : v[0]) + dpp<0x4e>(hi ? v[0] : v[2]);
    const float b = (hi ? v[3] : v[1]) + dpp<0x4e>(hi ? v[1] : v[3]);
    return (odd ? b : a) + dpp<0xb1>(odd ? a : b);
}

// Sums of M values over the sixteen channels of a wavefront, lanes with equal lane % 4 among themselves: v[0 .. M / 16) then hold the
// sums of the values i + (M / 16) k, k = the lane's place (lane / 4) with its bits in reverse.  Rows of 16 lanes and halves of the
// wavefront change places by one instruction for two registers, then neighbours within a row by data-parallel moves.
template <int M> __device__ __forceinline__ void channel_sums(float (&v)[M], int lane) {
#pragma unroll
    for (int i = 0; i < M / 2; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + M / 2]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
#pragma unroll
    for (int i = 0; i < M / 4; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + M / 4]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    const bool b3 = lane & 8, b2 = lane & 4;
#pragma unroll
    for (int i = 0; i < M / 8; ++i) v[i] = (b3 ? v[i + M / 8] : v[i]) + dpp<0x128>(b3 ? v[i] : v[i + M / 8]);      // row_ror:8
#pragma unroll
    for (int i = 0; i < M / 16; ++i) {
        const int give = __float_as_int(b2 ? v[i] : v[i + M / 16]);
        int got = __builtin_amdgcn_update_dpp(0, give, 0x104, 0xf, 0x5, false);          // row_shl:4 into groups 0 and 2
        got = __builtin_amdgcn_update_dpp(got, give, 0x114, 0xf, 0xa, false);            // row_shr:4 into groups 1 and 3
        v[i] = (b2 ? v[i + M / 16] : v[i]) + __int_as_float(got);
    }
}
// Which of the M values v[0] holds afterwards, in units of M / 16.
__device__ __forceinline__ int place_of(int lane) { return (lane & 32 ? 8 : 0) + (lane & 16 ? 4 : 0) + (lane & 8 ? 2 : 0) + (lane & 4 ? 1 : 0); }

// ---- storage ------------------------------------------------------------------------------------------------------
template <bool BF16> struct Elem;
template <> struct Elem<false> {
    typedef float Type;
    static __device__ __forceinline__ float get(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
    template <int S> static __device__ __forceinline__ void row(float (&v)[S], const float *p) {
        typedef float Vec __attribute__((ext_vector_type(S < 4 ? S : 4)));
#pragma unroll
        for (int i = 0; i < S; i += 4) {
            const Vec t = *reinterpret_cast<const Vec *>(p + i);
#pragma unroll
            for (int k = 0; k < (S < 4 ? S : 4); ++k) v[i + k] = t[k];
        }
    }
};
template <> struct Elem<true> {
    typedef uint16_t Type;
    static __device__ __forceinline__ float get(const uint16_t *p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ void put(uint16_t *p, float v) { *p = (uint16_t)pack_bf16(v, 0.0f); }
    template <int S> static __device__ __forceinline__ void row(float (&v)[S], const uint16_t *p) {
        typedef uint32_t Vec __attribute__((ext_vector_type(S / 2)));
        uint32_t w[S / 2];
        if constexpr (S == 2) w[0] = *reinterpret_cast<const uint32_t *>(p);
        else {
            const Vec t = *reinterpret_cast<const Vec *>(p);
#pragma unroll
            for (int k = 0; k < S / 2; ++k) w[k] = t[k];
        }
#pragma unroll
        for (int k = 0; k < S / 2; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
    }
};

template <int S> __device__ __forceinline__ void load_state(float (&h)[S], const float *p) { Elem<false>::row<S>(h, p); }
template <int S> __device__ __forceinline__ void store_state(float *p, const float (&h)[S]) {
    typedef float Vec __attribute__((ext_vector_type(S < 4 ? S : 4)));
#pragma unroll
    for (int i = 0; i < S; i += 4) {
        Vec t;
#pragma unroll
        for (int k = 0; k < (S < 4 ? S : 4); ++k) t[k] = h[i + k];
        *reinterpret_cast<Vec *>(p + i) = t;
    }
}

// Item i = sequence * groups + group of channels.
__device__ __forceinline__ void split_item(int64_t i, int groups, int64_t &v, int &g) {
    if ((i >> 32) == 0) { v = (uint32_t)i / (uint32_t)groups; g = (uint32_t)i % (uint32_t)groups; }
    else { v = i / groups; g = (int)(i % groups); }
}

__device__ __forceinline__ int length_of(const int32_t *lengths, int64_t v, int T) {
    return lengths ? min(max(uniform(lengths[v]), 0), T) : T;
}

// What a wavefront's lane has of one sequence: its channel, its states, where its rows lie.
template <bool BF16, int S> struct Lane {
    typedef typename Elem<BF16>::Type E;
    static constexpr int N = 4 * S;
    int q, ch;
    int64_t v, n, f;
    __device__ __forceinline__ Lane(const Scan &s, int64_t v_, int g, int lane) : q(lane & 3), ch(g * kChannels + (lane >> 2)), v(v_), n(s.n), f(s.f) {}
    __device__ __forceinline__ int64_t at(int t) const { return ((int64_t)t * n + v) * f + ch; }                     // of a frame [T][n][f]
    __device__ __forceinline__ const E *b_row(const void *bc, int t) const { return static_cast<const E *>(bc) + ((int64_t)t * n + v) * 2 * N + q * S; }
    __device__ __forceinline__ int64_t state(int64_t piece) const { return (((piece * n + v) * f) + ch) * N + q * S; }
    __device__ __forceinline__ int64_t channel(int64_t piece) const { return (piece * n + v) * f + ch; }
};

// a log2(e) of a lane's states: e = 2^(dt a2).
template <int S> __device__ __forceinline__ void load_decay(float (&a2)[S], const float *a, int ch, int q) {
#pragma unroll
    for (int s = 0; s < S; ++s) a2[s] = a[(int64_t)ch * 4 * S + q * S + s] * kLog2e;
}

// The state ahead of piece p: what its predecessors leave, each taken from zero by scan_piece_kernel (the first from h_before).
template <bool BF16, int S>
__device__ __forceinline__ void join_pieces(float (&h)[S], const float (&a2)[S], const Scan &s, const Lane<BF16, S> &l, int p) {
    if (p == 0) { load_state(h, s.piece_state + l.state(s.pieces - 1)); return; }
    load_state(h, s.piece_state + l.state(0));
    for (int k = 1; k < p; ++k) {
        float part[S];
        load_state(part, s.piece_state + l.state(k));
        const float time = s.piece_time[l.channel(k)];
#pragma unroll
        for (int i = 0; i < S; ++i) h[i] = fmaf(exp2_of(time * a2[i]), h[i], part[i]);
    }
}

// ---- forward ------------------------------------------------------------------------------------------------------
// Four timesteps of a wavefront as they lie in memory.
template <bool BF16, int S> struct Four {
    float x, delta, z, b[4][S], c[4][S];
};

// Y = whether outputs are formed (else only the state is carried along); `steps` of the four exist.
template <bool BF16, int S, bool Y>
__device__ __forceinline__ void load_four(Four<BF16, S> &r, const Scan &s, const Lane<BF16, S> &l, int t, int steps) {
    typedef typename Elem<BF16>::Type E;
    const int64_t at = l.at(t + min(l.q, steps - 1));
    r.x = Elem<BF16>::get(static_cast<const E *>(s.x) + at);
    r.delta = Elem<BF16>::get(static_cast<const E *>(s.delta) + at);
    if (Y) r.z = s.z ? Elem<BF16>::get(static_cast<const E *>(s.z) + at) : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const E *row = l.b_row(s.bc, t + min(j, steps - 1));
        Elem<BF16>::template row<S>(r.b[j], row);
        if (Y) Elem<BF16>::template row<S>(r.c[j], row + 4 * S);
    }
}

template <bool BF16, int S, bool Y, int J>
__device__ __forceinline__ void one_step(float (&h)[S], float &out, const float (&a2)[S], const Four<BF16, S> &r, float dt, float dtx) {
    const float dt_j = of_lane<J>(dt), dtx_j = of_lane<J>(dtx);
    float acc = 0.0f;
#pragma unroll
    for (int i = 0; i < S; ++i) {
        h[i] = fmaf(exp2_of(dt_j * a2[i]), h[i], dtx_j * r.b[J][i]);
        if (Y) acc = fmaf(r.c[J][i], h[i], acc);
    }
    out = acc;
}

template <bool BF16, int S, bool Y>
__device__ __forceinline__ void four_steps(float (&h)[S], float &time, const float (&a2)[S], const Scan &s, const Lane<BF16, S> &l, const Four<BF16, S> &r, int t,
                                           int steps, float bias, float d) {
    typedef typename Elem<BF16>::Type E;
    float sig;
    const float dt = softplus_of(r.delta + bias, sig), dtx = dt * r.x;
    float out[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    one_step<BF16, S, Y, 0>(h, out[0], a2, r, dt, dtx);
    if (steps > 1) one_step<BF16, S, Y, 1>(h, out[1], a2, r, dt, dtx);
    if (steps > 2) one_step<BF16, S, Y, 2>(h, out[2], a2, r, dt, dtx);
    if (steps > 3) one_step<BF16, S, Y, 3>(h, out[3], a2, r, dt, dtx);
    if (!Y) time += l.q < steps ? dt : 0.0f;
    else {
        float y = fmaf(d, r.x, quad_sums(out, l.q));
        if (s.z) y *= r.z * sigmoid_of(r.z);
        if (l.q < steps) Elem<BF16>::put(static_cast<E *>(s.y) + l.at(t + l.q), y);
    }
}

// One sequence's sixteen channels over [t0, t_end), the states of four timesteps ahead of their use.
template <bool BF16, int S, bool Y>
__device__ __forceinline__ void walk(float (&h)[S], float &time, const float (&a2)[S], const Scan &s, const Lane<BF16, S> &l, int t0, int t_end, float bias, float d) {
    if (t0 >= t_end) return;
    Four<BF16, S> now, next;
    load_four<BF16, S, Y>(now, s, l, t0, min(4, t_end - t0));
    for (int t = t0; t < t_end; t += 4) {
        if (Y && s.checkpoints && (t & (kTile - 1)) == 0) store_state(s.checkpoints + l.state(t / kTile), h);
        const int left = t_end - t;
        if (left > 4) load_four<BF16, S, Y>(next, s, l, t + 4, min(4, left - 4));
        if (left >= 4) four_steps<BF16, S, Y>(h, time, a2, s, l, now, t, 4, bias, d);
        else four_steps<BF16, S, Y>(h, time, a2, s, l, now, t, left, bias, d);
        now = next;
    }
}

template <bool BF16, int S>
__global__ __launch_bounds__(kWaves *kWave) void scan_kernel(Scan s) {
    typedef typename Elem<BF16>::Type E;
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), p = blockIdx.y;
    const int t0 = p * s.chunk, t1 = min(s.T, t0 + s.chunk);
    for (int64_t i = (int64_t)blockIdx.x * kWaves + wave; i < s.n * s.groups; i += (int64_t)gridDim.x * kWaves) {
        int64_t v;
        int g;
        split_item(i, s.groups, v, g);
        const Lane<BF16, S> l(s, v, g, lane);
        const int t_end = min(t1, length_of(s.lengths, v, s.T));
        float a2[S], h[S], time = 0.0f;
        load_decay(a2, s.a, l.ch, l.q);
        const float bias = s.dt_bias ? s.dt_bias[l.ch] : 0.0f, d = s.d ? s.d[l.ch] : 0.0f;
        if (s.pieces > 1) join_pieces<BF16, S>(h, a2, s, l, p);
        else if (s.h_before) load_state(h, s.h_before + l.state(0));
        else
#pragma unroll
            for (int k = 0; k < S; ++k) h[k] = 0.0f;
        walk<BF16, S, true>(h, time, a2, s, l, t0, t_end, bias, d);
        for (int t = max(t0, t_end) + l.q; t < t1; t += 4) Elem<BF16>::put(static_cast<E *>(s.y) + l.at(t), 0.0f);
        if (s.h_after && p == s.pieces - 1) store_state(s.h_after + l.state(0), h);
    }
}

// Where there are few sequences the time axis is cut into pieces: what each leaves when it starts from zero (the first: from h_before),
// and the sum of its step sizes, which gives the decay across it, exp(a sum dt).  The last piece's place takes a copy of h_before: the
// last piece's wavefront may write h_after over it before the first one's has read it.
template <bool BF16, int S>
__global__ __launch_bounds__(kWaves *kWave) void scan_piece_kernel(Scan s) {
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), p = blockIdx.y;
    const int t0 = p * s.chunk, t1 = min(s.T, t0 + s.chunk);
    for (int64_t i = (int64_t)blockIdx.x * kWaves + wave; i < s.n * s.groups; i += (int64_t)gridDim.x * kWaves) {
        int64_t v;
        int g;
        split_item(i, s.groups, v, g);
        const Lane<BF16, S> l(s, v, g, lane);
        const int t_end = min(t1, length_of(s.lengths, v, s.T));
        float a2[S], h[S], time = 0.0f;
        load_decay(a2, s.a, l.ch, l.q);
        if (p == 0 && s.h_before) load_state(h, s.h_before + l.state(0));
        else
#pragma unroll
            for (int k = 0; k < S; ++k) h[k] = 0.0f;
        if (p == 0) store_state(s.piece_state + l.state(s.pieces - 1), h);
        walk<BF16, S, false>(h, time, a2, s, l, t0, t_end, s.dt_bias ? s.dt_bias[l.ch] : 0.0f, 0.0f);
        time = quad_sum(time);
        store_state(s.piece_state + l.state(p), h);
        if (l.q == 0) s.piece_time[l.channel(p)] = time;
    }
}

// ---- backward -----------------------------------------------------------------------------------------------------
// dL/dh as a piece hands it to its predecessor when nothing reaches it from behind, and the sum of its step sizes.
template <bool BF16, int S>
__global__ __launch_bounds__(kWaves *kWave) void scan_back_piece_kernel(ScanBack b) {
    typedef typename Elem<BF16>::Type E;
    const Scan &s = b.s;
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), p = blockIdx.y + 1;
    const int t0 = p * s.chunk, t1 = min(s.T, t0 + s.chunk);
    for (int64_t i = (int64_t)blockIdx.x * kWaves + wave; i < s.n * s.groups; i += (int64_t)gridDim.x * kWaves) {
        int64_t v;
        int g;
        split_item(i, s.groups, v, g);
        const Lane<BF16, S> l(s, v, g, lane);
        const int t_end = min(t1, length_of(s.lengths, v, s.T));
        const float bias = s.dt_bias ? s.dt_bias[l.ch] : 0.0f;
        float a2[S], k[S], time = 0.0f;
        load_decay(a2, s.a, l.ch, l.q);
#pragma unroll
        for (int i2 = 0; i2 < S; ++i2) k[i2] = 0.0f;
        auto four = [&](int t, int steps) {
            const bool there = l.q < steps;
            const int64_t at = l.at(t + min(l.q, steps - 1));
            float sig, gy = Elem<BF16>::get(static_cast<const E *>(b.g_y) + at);
            if (s.z) {
                const float z = Elem<BF16>::get(static_cast<const E *>(s.z) + at);
                gy *= z * sigmoid_of(z);
            }
            const float dt = softplus_of(Elem<BF16>::get(static_cast<const E *>(s.delta) + at) + bias, sig);
            time += there ? dt : 0.0f;
            auto step = [&](float dt_j, float g_j, int j) {
                float c[S];
                Elem<BF16>::template row<S>(c, l.b_row(s.bc, t + j) + 4 * S);
#pragma unroll
                for (int m = 0; m < S; ++m) k[m] = exp2_of(dt_j * a2[m]) * fmaf(c[m], g_j, k[m]);
            };
            if (steps > 3) step(of_lane<3>(dt), of_lane<3>(gy), 3);
            if (steps > 2) step(of_lane<2>(dt), of_lane<2>(gy), 2);
            if (steps > 1) step(of_lane<1>(dt), of_lane<1>(gy), 1);
            step(of_lane<0>(dt), of_lane<0>(gy), 0);
        };
        int t = t0 + ((t_end - t0 - 1) & ~3);
        if (t_end > t0) {
            if (t_end - t < 4) { four(t, t_end - t); t -= 4; }
            for (; t >= t0; t -= 4) four(t, 4);
        }
        time = quad_sum(time);
        store_state(s.piece_state + l.state(p), k);
        if (l.q == 0) s.piece_time[l.channel(p)] = time;
    }
}

// Timesteps that a wavefront holds the states of: as many as fit its registers.
template <int S> constexpr int kHeld = S <= 4 ? 16 : 8;

template <bool BF16, int S>
__global__ __launch_bounds__(kBackWaves *kWave) void scan_back_kernel(ScanBack b) {
    typedef typename Elem<BF16>::Type E;
    constexpr int N = 4 * S, K = kHeld<S>, R = K / 4, V = K * 2 * N;      // V: values of dB and dC of a tile
    extern __shared__ float s_bc[];                                       // [2][wavefronts][V]
    const Scan &s = b.s;
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int part = blockIdx.x % b.blocks_of_groups, slot = blockIdx.x / b.blocks_of_groups, slots = gridDim.x / b.blocks_of_groups;
    const int own = b.sequences > 1 ? s.groups : waves;                   // wavefronts of one sequence in this workgroup
    const int g = b.blocks_of_groups > 1 ? part * kBackWaves + wave : wave % own, which = wave / own;
    const bool in_width = g < s.groups;
    const int ch = g * kChannels + (lane >> 2), q = lane & 3;
    float a2[S], a[S], acc_a[S];
    double sum_a[S], sum_d = 0.0, sum_bias = 0.0;
#pragma unroll
    for (int i = 0; i < S; ++i) {
        a[i] = in_width ? s.a[(int64_t)ch * N + q * S + i] : 0.0f;
        a2[i] = a[i] * kLog2e;
        sum_a[i] = 0.0;
    }
    const float bias = s.dt_bias && in_width ? s.dt_bias[ch] : 0.0f, d = s.d && in_width ? s.d[ch] : 0.0f;
    const int64_t items = (s.n + b.sequences - 1) / b.sequences * s.pieces;
    int buffer = 0;
    for (int64_t item = slot; item < items; item += slots) {
        const int p = (int)(item % s.pieces);
        const int64_t first = item / s.pieces * b.sequences, v = first + which;
        const int t0 = p * s.chunk, t1 = min(s.T, t0 + s.chunk);
        const bool mine = in_width && v < s.n;
        const Lane<BF16, S> l(s, mine ? v : 0, mine ? g : 0, lane);
        const int t_end = mine ? min(t1, length_of(s.lengths, v, s.T)) : t0;
        float k[S];                                                       // dL/dh from behind
#pragma unroll
        for (int i = 0; i < S; ++i) k[i] = 0.0f;
        if (mine) {
            if (b.dh_after) load_state(k, b.dh_after + l.state(0));
            for (int o = s.pieces - 1; o > p; --o) {
                float there[S];
                load_state(there, s.piece_state + l.state(o));
                const float time = s.piece_time[l.channel(o)];
#pragma unroll
                for (int i = 0; i < S; ++i) k[i] = fmaf(exp2_of(time * a2[i]), k[i], there[i]);
            }
        }
        for (int t = t0 + (t1 - t0 - 1) / K * K; t >= t0; t -= K, buffer ^= 1) {
            float *const out = s_bc + (buffer * waves + wave) * V;
            if (t < t_end) {
                const int steps = min(K, t_end - t);
                // the lane's own timesteps: t + 4 i + q
                float x[R], dt[R], sig[R], gp[R], gz[R], y[R];
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const bool there = 4 * i + q < steps;
                    const int64_t at = l.at(t + min(4 * i + q, steps - 1));
                    x[i] = Elem<BF16>::get(static_cast<const E *>(s.x) + at);
                    const float delta = Elem<BF16>::get(static_cast<const E *>(s.delta) + at), gy = Elem<BF16>::get(static_cast<const E *>(b.g_y) + at);
                    dt[i] = softplus_of(delta + bias, sig[i]);
                    gp[i] = gy;
                    gz[i] = 0.0f;
                    if (s.z) {
                        const float z = Elem<BF16>::get(static_cast<const E *>(s.z) + at), sz = sigmoid_of(z);
                        gp[i] = gy * z * sz;
                        gz[i] = gy * sz * fmaf(z, 1.0f - sz, 1.0f);
                    }
                    if (!there) x[i] = dt[i] = gp[i] = 0.0f;
                }
                // forward over the tile, its states kept
                float h[S], held[K][S];
                int64_t from = l.state(t / kTile);
                load_state(h, s.checkpoints + from);
                auto rows = [&](float (&r)[4][S], int i, int column) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (4 * i + j < steps) Elem<BF16>::template row<S>(r[j], l.b_row(s.bc, t + 4 * i + j) + column);
                        else
#pragma unroll
                            for (int m = 0; m < S; ++m) r[j][m] = 0.0f;
                    }
                };
                auto ahead = [&](float (&h)[S], const float (&row)[S], float dt_j, float dtx_j) {
#pragma unroll
                    for (int m = 0; m < S; ++m) h[m] = fmaf(exp2_of(dt_j * a2[m]), h[m], dtx_j * row[m]);
                };
                if (K < kTile && (t & (kTile - 1))) {                     // the kept state lies K timesteps back
                    float dt0[R], dtx0[R], sig0;
#pragma unroll
                    for (int i = 0; i < R; ++i) {
                        const int64_t at = l.at(t - K + 4 * i + q);
                        dt0[i] = softplus_of(Elem<BF16>::get(static_cast<const E *>(s.delta) + at) + bias, sig0);
                        dtx0[i] = dt0[i] * Elem<BF16>::get(static_cast<const E *>(s.x) + at);
                    }
#pragma unroll
                    for (int i = 0; i < R; ++i) {
                        float rb[4][S];
#pragma unroll
                        for (int j = 0; j < 4; ++j) Elem<BF16>::template row<S>(rb[j], l.b_row(s.bc, t - K + 4 * i + j));
                        ahead(h, rb[0], of_lane<0>(dt0[i]), of_lane<0>(dtx0[i]));
                        ahead(h, rb[1], of_lane<1>(dt0[i]), of_lane<1>(dtx0[i]));
                        ahead(h, rb[2], of_lane<2>(dt0[i]), of_lane<2>(dtx0[i]));
                        ahead(h, rb[3], of_lane<3>(dt0[i]), of_lane<3>(dtx0[i]));
                    }
                }
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    float rb[4][S], rc[4][S], part_y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    rows(rb, i, 0);
                    if (s.z) rows(rc, i, N);
                    const float dtx = dt[i] * x[i];
                    auto step = [&](int j, float dt_j, float dtx_j) {
#pragma unroll
                        for (int m = 0; m < S; ++m) held[4 * i + j][m] = h[m];
                        ahead(h, rb[j], dt_j, dtx_j);
                        if (s.z)
#pragma unroll
                            for (int m = 0; m < S; ++m) part_y[j] = fmaf(rc[j][m], h[m], part_y[j]);
                    };
                    step(0, of_lane<0>(dt[i]), of_lane<0>(dtx));
                    step(1, of_lane<1>(dt[i]), of_lane<1>(dtx));
                    step(2, of_lane<2>(dt[i]), of_lane<2>(dtx));
                    step(3, of_lane<3>(dt[i]), of_lane<3>(dtx));
                    y[i] = fmaf(d, x[i], quad_sums(part_y, q));
                }
                // ... and back
#pragma unroll
                for (int m = 0; m < S; ++m) acc_a[m] = 0.0f;
                float acc_d = 0.0f, acc_bias = 0.0f;
#pragma unroll
                for (int i = R - 1; i >= 0; --i) {
                    float rb[4][S], rc[4][S], bc[8 * S], ghb[4], sa[4];
                    rows(rb, i, 0);
                    rows(rc, i, N);
                    const float dtx = dt[i] * x[i];
                    auto step = [&](int j, float dt_j, float dtx_j, float g_j) {
                        ghb[j] = sa[j] = 0.0f;
#pragma unroll
                        for (int m = 0; m < S; ++m) {
                            const float gh = fmaf(rc[j][m], g_j, k[m]);
                            bc[j * 2 * S + m] = gh * dtx_j;
                            bc[j * 2 * S + S + m] = h[m] * g_j;
                            ghb[j] = fmaf(gh, rb[j][m], ghb[j]);
                            h[m] = held[4 * i + j][m];
                            k[m] = gh * exp2_of(dt_j * a2[m]);
                            const float u = k[m] * h[m];
                            sa[j] = fmaf(u, a[m], sa[j]);
                            acc_a[m] = fmaf(u, dt_j, acc_a[m]);
                        }
                    };
                    step(3, of_lane<3>(dt[i]), of_lane<3>(dtx), of_lane<3>(gp[i]));
                    step(2, of_lane<2>(dt[i]), of_lane<2>(dtx), of_lane<2>(gp[i]));
                    step(1, of_lane<1>(dt[i]), of_lane<1>(dtx), of_lane<1>(gp[i]));
                    step(0, of_lane<0>(dt[i]), of_lane<0>(dtx), of_lane<0>(gp[i]));
                    const float gb = quad_sums(ghb, q), da = quad_sums(sa, q);
                    const float ddelta = fmaf(x[i], gb, da) * sig[i];
                    if (4 * i + q < steps) {
                        const int64_t at = l.at(t + 4 * i + q);
                        Elem<BF16>::put(static_cast<E *>(b.dx) + at, fmaf(d, gp[i], dt[i] * gb));
                        Elem<BF16>::put(static_cast<E *>(b.ddelta) + at, ddelta);
                        if (s.z) Elem<BF16>::put(static_cast<E *>(b.dz) + at, gz[i] * y[i]);
                        acc_d = fmaf(gp[i], x[i], acc_d);
                        acc_bias += ddelta;
                    }
                    // value i = step * 2 S + (B or C) * S + state; a lane ends up with 8 S / 16 of them
                    channel_sums<8 * S>(bc, lane);
#pragma unroll
                    for (int m = 0; m < S / 2; ++m) {
                        const int at = m + (S / 2) * place_of(lane), j = at / (2 * S), rest = at % (2 * S);
                        out[(4 * i + j) * 2 * N + (rest / S) * N + q * S + rest % S] = bc[m];
                    }
                }
#pragma unroll
                for (int m = 0; m < S; ++m) sum_a[m] += (double)acc_a[m];
                sum_d += (double)acc_d;
                sum_bias += (double)acc_bias;
            } else
                for (int i = lane; i < V; i += kWave) out[i] = 0.0f;
            if (mine)
                for (int o = max(t, t_end) + q; o < min(t + K, t1); o += 4) {
                    const int64_t at = l.at(o);
                    Elem<BF16>::put(static_cast<E *>(b.dx) + at, 0.0f);
                    Elem<BF16>::put(static_cast<E *>(b.ddelta) + at, 0.0f);
                    if (s.z) Elem<BF16>::put(static_cast<E *>(b.dz) + at, 0.0f);
                }
            __syncthreads();                                              // two buffers: the next tile's values do not meet this one's readers
            const float *const all = s_bc + buffer * waves * V;
            for (int i = threadIdx.x; i < b.sequences * V; i += blockDim.x) {
                const int r = i / V, e = i % V, j = e / (2 * N), column = e % (2 * N);
                float sum = all[r * own * V + e];
                for (int w = 1; w < own; ++w) sum += all[(r * own + w) * V + e];
                if (first + r < s.n && t + j < t1) {
                    const int64_t at = ((int64_t)(t + j) * s.n + first + r) * 2 * N + column;
                    if (b.dbc_part) b.dbc_part[(int64_t)part * s.T * s.n * 2 * N + at] = sum;
                    else Elem<BF16>::put(static_cast<E *>(b.dbc) + at, sum);
                }
            }
        }
        if (mine && b.dh_before && p == 0) store_state(b.dh_before + l.state(0), k);
    }
    // sums over time and sequences: one place per workgroup and sequence beside others
    if (in_width) {
        double *to = b.sums + ((int64_t)slot * b.sequences + which) * s.f * (N + 2);
#pragma unroll
        for (int i = 0; i < S; ++i) to[(int64_t)ch * N + q * S + i] = sum_a[i];
        sum_d += __shfl_xor(sum_d, 1);
        sum_d += __shfl_xor(sum_d, 2);
        sum_bias += __shfl_xor(sum_bias, 1);
        sum_bias += __shfl_xor(sum_bias, 2);
        if (q == 0) { to[(int64_t)s.f * N + ch] = sum_d; to[(int64_t)s.f * (N + 1) + ch] = sum_bias; }
    }
}

// da | dd | ddt_bias from the workgroups' sums, sixteen at a time and in a fixed order.
__global__ __launch_bounds__(256) void scan_sums_kernel(const double *__restrict__ sums, int slots, int states, int rest, float *__restrict__ da, float *__restrict__ dd,
                                                        float *__restrict__ ddt_bias, int accumulate) {
    __shared__ double s_part[16][17];
    const int o = threadIdx.x % 16, r = threadIdx.x / 16, at = blockIdx.x * 16 + o, width = states + 2 * rest;
    double sum = 0.0;
    if (at < width)
        for (int k = r; k < slots; k += 16) sum += sums[(int64_t)k * width + at];
    s_part[r][o] = sum;
    __syncthreads();
    if (r == 0 && at < width) {
        for (int k = 1; k < 16; ++k) sum += s_part[k][o];
        float *to = at < states ? da + at : at < states + rest ? (dd ? dd + (at - states) : nullptr) : ddt_bias ? ddt_bias + (at - states - rest) : nullptr;
        if (to) *to = accumulate ? (float)((double)*to + sum) : (float)sum;
    }
}

// dbc of sequences that several workgroups share.
template <bool BF16>
__global__ __launch_bounds__(256) void scan_rows_kernel(const float *__restrict__ part, int parts, int64_t count, void *dbc) {
    typedef typename Elem<BF16>::Type E;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        float sum = part[i];
        for (int k = 1; k < parts; ++k) sum += part[(int64_t)k * count + i];
        Elem<BF16>::put(static_cast<E *>(dbc) + i, sum);
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------
bool scan_states(int32_t N) { return N == 8 || N == 16 || N == 32; }

int check_shape(int64_t T, int64_t n, int32_t f, int32_t N) {
    if (T <= 0 || n <= 0 || f < kChannels || f % kChannels || f > DGNN_MAX_CHANNELS || !scan_states(N)) return DGNN_ERR_SHAPE;
    if (!fits_index(n) || !fits_index(T) || T > (int64_t(1) << 44) / n) return DGNN_ERR_OVERFLOW;
    return DGNN_OK;
}

struct Pieces { int chunk, count; };

Pieces pieces_of(int64_t T, int64_t items, int64_t wanted) {
    const int64_t tiles = (T + kTile - 1) / kTile;
    int64_t count = std::min<int64_t>(tiles / 2, wanted / std::max<int64_t>(items, 1));
    if (count < 4) return {(int)(tiles * kTile), 1};
    const int64_t chunk = (tiles + count - 1) / count * kTile;
    return {(int)chunk, (int)((T + chunk - 1) / chunk)};
}

Pieces forward_pieces(int64_t T, int64_t n, int32_t f) { return pieces_of(T, n * (f / kChannels), 4096); }

struct BackShape { int groups, blocks_of_groups, sequences, waves; int64_t rows; Pieces pieces; int64_t slots; };

BackShape back_shape(int64_t T, int64_t n, int32_t f) {
    BackShape b;
    b.groups = f / kChannels;
    b.blocks_of_groups = (b.groups + kBackWaves - 1) / kBackWaves;
    b.sequences = b.groups < kBackWaves ? kBackWaves / b.groups : 1;
    b.waves = b.blocks_of_groups > 1 ? kBackWaves : b.sequences * b.groups;
    b.rows = (n + b.sequences - 1) / b.sequences;
    b.pieces = pieces_of(T, b.rows * b.blocks_of_groups, 512);
    b.slots = std::max<int64_t>(1, std::min<int64_t>(b.rows * b.pieces.count, kMaxSlots / 2 / b.blocks_of_groups));
    return b;
}

size_t piece_bytes(const Pieces &p, int64_t n, int32_t f, int32_t N) {
    return p.count > 1 ? round_up((size_t)p.count * n * f * N * sizeof(float), 256) + round_up((size_t)p.count * n * f * sizeof(float), 256) : 0;
}

void place_pieces(Scan &s, const Pieces &p, int32_t N, void *ws) {
    s.chunk = p.chunk;
    s.pieces = p.count;
    s.piece_state = s.piece_time = nullptr;
    if (p.count > 1) {
        s.piece_state = static_cast<float *>(ws);
        s.piece_time = reinterpret_cast<float *>(static_cast<char *>(ws) + round_up((size_t)p.count * s.n * s.f * N * sizeof(float), 256));
    }
}

dim3 walk_grid(const Scan &s, int pieces) {
    return dim3((unsigned)std::min<int64_t>((s.n * s.groups + kWaves - 1) / kWaves, std::max(1, kMaxGrid / pieces)), (unsigned)pieces);
}

// kernel<BF16, S> by storage type and state size
template <typename F> int by_kind(dgnn_dtype dt, int32_t N, F &&launch) {
    const bool wide = dt == DGNN_BF16;
    if (N == 8) { if (wide) launch(std::integral_constant<bool, true>{}, std::integral_constant<int, 2>{}); else launch(std::integral_constant<bool, false>{}, std::integral_constant<int, 2>{}); }
    else if (N == 16) { if (wide) launch(std::integral_constant<bool, true>{}, std::integral_constant<int, 4>{}); else launch(std::integral_constant<bool, false>{}, std::integral_constant<int, 4>{}); }
    else { if (wide) launch(std::integral_constant<bool, true>{}, std::integral_constant<int, 8>{}); else launch(std::integral_constant<bool, false>{}, std::integral_constant<int, 8>{}); }
    DGNN_RETURN_IF_LAUNCH_FAILED();
    return DGNN_OK;
}

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const char *p = static_cast<const char *>(a), *q = static_cast<const char *>(b);
    return p && q && p < q + nb && q < p + na;
}

}  // namespace

extern "C" int dgnn_selective_scan_checkpoints(int64_t T, int64_t n, int32_t f, int32_t states, size_t *bytes) {
    if (!bytes) return DGNN_ERR_NULL;
    if (int rc = check_shape(T, n, f, states)) return rc;
    *bytes = (size_t)((T + kTile - 1) / kTile) * n * f * states * sizeof(float);
    return DGNN_OK;
}

extern "C" int dgnn_selective_scan_workspace(int64_t T, int64_t n, int32_t f, int32_t states, size_t *bytes) {
    if (!bytes) return DGNN_ERR_NULL;
    if (int rc = check_shape(T, n, f, states)) return rc;
    *bytes = std::max<size_t>(256, piece_bytes(forward_pieces(T, n, f), n, f, states));
    return DGNN_OK;
}

extern "C" int dgnn_selective_scan(const void *x, const void *delta, const void *bc, const void *z, const float *a, const float *d, const float *dt_bias,
                                   const float *h_before, void *y, float *h_after, float *checkpoints, const int32_t *lengths, int64_t T, int64_t n, int32_t f,
                                   int32_t states, dgnn_dtype dt, void *ws, size_t ws_bytes, void *stream) {
    if (!x || !delta || !bc || !a || !y || !ws) return DGNN_ERR_NULL;
    if (int rc = check_shape(T, n, f, states)) return rc;
    if (dt != DGNN_F32 && dt != DGNN_BF16) return DGNN_ERR_SHAPE;
    for (const void *p : {x, delta, bc, z, (const void *)h_before, (const void *)y, (const void *)h_after, (const void *)checkpoints, (const void *)ws})
        if (p && !aligned16(p)) return DGNN_ERR_ALIGN;
    const size_t frame = (size_t)T * n * f * (dt == DGNN_F32 ? 4 : 2), rows = (size_t)T * n * 2 * states * (dt == DGNN_F32 ? 4 : 2);
    const size_t state = (size_t)n * f * states * sizeof(float), kept = (size_t)((T + kTile - 1) / kTile) * state;
    for (auto o : {std::pair<const void *, size_t>{y, frame}, {h_after, state}, {checkpoints, kept}, {ws, ws_bytes}}) {
        for (auto i : {std::pair<const void *, size_t>{x, frame}, {delta, frame}, {bc, rows}, {z, frame}})
            if (overlap(o.first, o.second, i.first, i.second)) return DGNN_ERR_ALIAS;
        if (!(o.first == h_after && h_after == h_before) && overlap(o.first, o.second, h_before, state)) return DGNN_ERR_ALIAS;
    }
    if (overlap(y, frame, h_after, state) || overlap(y, frame, checkpoints, kept) || overlap(h_after, state, checkpoints, kept) || overlap(ws, ws_bytes, y, frame) ||
        overlap(ws, ws_bytes, h_after, state) || overlap(ws, ws_bytes, checkpoints, kept))
        return DGNN_ERR_ALIAS;
    const Pieces p = forward_pieces(T, n, f);
    if (ws_bytes < piece_bytes(p, n, f, states)) return DGNN_ERR_CAPACITY;
    Scan s{x, delta, bc, z, a, d, dt_bias, h_before, y, h_after, checkpoints, lengths, n, (int)T, f, f / kChannels, 0, 0, nullptr, nullptr};
    place_pieces(s, p, states, ws);
    hipStream_t st = (hipStream_t)stream;
    if (s.pieces > 1) {
        const int rc = by_kind(dt, states, [&](auto bf16, auto per) {
            hipLaunchKernelGGL((scan_piece_kernel<decltype(bf16)::value, decltype(per)::value>), walk_grid(s, s.pieces - 1), dim3(kWaves * kWave), 0, st, s);
        });
        if (rc) return rc;
    }
    return by_kind(dt, states, [&](auto bf16, auto per) {
        hipLaunchKernelGGL((scan_kernel<decltype(bf16)::value, decltype(per)::value>), walk_grid(s, s.pieces), dim3(kWaves * kWave), 0, st, s);
    });
}

extern "C" int dgnn_selective_scan_backward_workspace(int64_t T, int64_t n, int32_t f, int32_t states, size_t *bytes) {
    if (!bytes) return DGNN_ERR_NULL;
    if (int rc = check_shape(T, n, f, states)) return rc;
    const BackShape b = back_shape(T, n, f);
    *bytes = piece_bytes(b.pieces, n, f, states) + round_up((size_t)b.slots * b.sequences * f * (states + 2) * sizeof(double), 256) +
             (b.blocks_of_groups > 1 ? (size_t)b.blocks_of_groups * T * n * 2 * states * sizeof(float) : 0);
    return DGNN_OK;
}

extern "C" int dgnn_selective_scan_backward(const void *x, const void *delta, const void *bc, const void *z, const float *a, const float *d, const float *dt_bias,
                                            const float *checkpoints, const void *g_y, const float *dh_after, void *dx, void *ddelta, void *dbc, void *dz,
                                            float *da, float *dd, float *ddt_bias, float *dh_before, const int32_t *lengths, int64_t T, int64_t n, int32_t f,
                                            int32_t states, int32_t accumulate, dgnn_dtype dt, void *ws, size_t ws_bytes, void *stream) {
    if (!x || !delta || !bc || !a || !checkpoints || !g_y || !dx || !ddelta || !dbc || !da || !ws || (z && !dz) || (d && !dd) || (dt_bias && !ddt_bias))
        return DGNN_ERR_NULL;
    if (int rc = check_shape(T, n, f, states)) return rc;
    if (dt != DGNN_F32 && dt != DGNN_BF16) return DGNN_ERR_SHAPE;
    if ((!z && dz) || (!d && dd) || (!dt_bias && ddt_bias)) return DGNN_ERR_SHAPE;       // a gradient of what is not there
    for (const void *p : {x, delta, bc, z, (const void *)checkpoints, g_y, (const void *)dh_after, (const void *)dx, (const void *)ddelta, (const void *)dbc, (const void *)dz,
                          (const void *)dh_before, (const void *)ws})
        if (p && !aligned16(p)) return DGNN_ERR_ALIGN;
    size_t need = 0;
    dgnn_selective_scan_backward_workspace(T, n, f, states, &need);
    if (ws_bytes < need) return DGNN_ERR_CAPACITY;
    const size_t frame = (size_t)T * n * f * (dt == DGNN_F32 ? 4 : 2), rows = (size_t)T * n * 2 * states * (dt == DGNN_F32 ? 4 : 2);
    const size_t state = (size_t)n * f * states * sizeof(float), kept = (size_t)((T + kTile - 1) / kTile) * state;
    const std::pair<const void *, size_t> in[] = {{x, frame}, {delta, frame}, {bc, rows}, {z, frame}, {checkpoints, kept}, {g_y, frame}, {dh_after, state}};
    const std::pair<const void *, size_t> out[] = {{dx, frame}, {ddelta, frame}, {dbc, rows}, {dz, frame}, {dh_before, state}, {ws, ws_bytes}};
    for (size_t i = 0; i < sizeof(out) / sizeof(*out); ++i) {
        for (auto o : in)
            if (overlap(out[i].first, out[i].second, o.first, o.second)) return DGNN_ERR_ALIAS;
        for (size_t k = 0; k < i; ++k)
            if (overlap(out[i].first, out[i].second, out[k].first, out[k].second)) return DGNN_ERR_ALIAS;
    }
    const BackShape shape = back_shape(T, n, f);
    ScanBack b{};
    b.s = Scan{x, delta, bc, z, a, d, dt_bias, nullptr, nullptr, nullptr, const_cast<float *>(checkpoints), lengths, n, (int)T, f, shape.groups, 0, 0, nullptr, nullptr};
    place_pieces(b.s, shape.pieces, states, ws);
    b.g_y = g_y; b.dh_after = dh_after; b.dx = dx; b.ddelta = ddelta; b.dbc = dbc; b.dz = dz; b.dh_before = dh_before;
    b.blocks_of_groups = shape.blocks_of_groups;
    b.sequences = shape.sequences;
    char *at = static_cast<char *>(ws) + piece_bytes(shape.pieces, n, f, states);
    b.sums = reinterpret_cast<double *>(at);
    at += round_up((size_t)shape.slots * shape.sequences * f * (states + 2) * sizeof(double), 256);
    b.dbc_part = shape.blocks_of_groups > 1 ? reinterpret_cast<float *>(at) : nullptr;
    hipStream_t st = (hipStream_t)stream;
    if (b.s.pieces > 1) {
        const int rc = by_kind(dt, states, [&](auto bf16, auto per) {
            hipLaunchKernelGGL((scan_back_piece_kernel<decltype(bf16)::value, decltype(per)::value>), walk_grid(b.s, b.s.pieces - 1), dim3(kWaves * kWave), 0, st, b);
        });
        if (rc) return rc;
    }
    int rc = by_kind(dt, states, [&](auto bf16, auto per) {
        constexpr int S = decltype(per)::value;
        const unsigned lds = 2u * shape.waves * kHeld<S> * 8 * S * sizeof(float);
        hipLaunchKernelGGL((scan_back_kernel<decltype(bf16)::value, S>), dim3((unsigned)(shape.slots * shape.blocks_of_groups)), dim3(shape.waves * kWave), lds, st, b);
    });
    if (rc) return rc;
    const int width = f * (states + 2);
    hipLaunchKernelGGL(scan_sums_kernel, dim3((unsigned)((width + 15) / 16)), dim3(256), 0, st, b.sums, (int)(shape.slots * shape.sequences), f * states, f, da, dd, ddt_bias,
                       accumulate);
    DGNN_RETURN_IF_LAUNCH_FAILED();
    if (b.dbc_part) {
        const int64_t count = T * n * 2 * states;
        const unsigned blocks = (unsigned)std::min<int64_t>((count + 255) / 256, kMaxGrid);
        if (dt == DGNN_BF16) hipLaunchKernelGGL(scan_rows_kernel<true>, dim3(blocks), dim3(256), 0, st, b.dbc_part, shape.blocks_of_groups, count, dbc);
        else hipLaunchKernelGGL(scan_rows_kernel<false>, dim3(blocks), dim3(256), 0, st, b.dbc_part, shape.blocks_of_groups, count, dbc);
        DGNN_RETURN_IF_LAUNCH_FAILED();
    }
    return DGNN_OK;
}
