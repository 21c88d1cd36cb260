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
//
// The time axis goes by tiles of sixteen steps (eight in short series).  B and C of a tile are the same for all channels: a wavefront fetches them as whole
// 16-byte pieces and reads them back from LDS, four addresses a read, where a load per timestep would keep the 64 lanes of the
// cache's port busy for 64 bytes.  Wavefronts stay, keep their channels (and so a, d and the bias) and take one sequence after the other;
// the loads of the next tile, be it of the next sequence, are under way while a tile is computed.
#include <algorithm>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "common.hpp"

namespace {

using namespace dgnn;

constexpr int kChannels = 16;             // channels of a wavefront
constexpr int kTile = 16;                 // timesteps of a tile, but for short series
constexpr int kPiece = 16;                // ... of a piece of the time axis, at least; pieces are multiples of it
// ... between two kept states: the adjoint holds the states of so many timesteps in registers (sixteen would be 32 registers more with 16 states,
// beyond the 256 there are); the forward pass writes 4 N / 8 bytes a value for them.
constexpr int kHeld = 8;
constexpr int kWaves = 4;                 // wavefronts of a workgroup of the kernels without sums over channels
// Wavefronts of a workgroup of the adjoint at most, and of all its workgroups: two on a SIMD, and three with 8 states, whose registers
// allow it (16 x 8192 x 128 fp32: 225 us with two, 187 with three); workgroups of four then, for three times eight do not fit.
constexpr int back_waves(int states) { return states == 8 ? 4 : 8; }
constexpr int back_resident(int states) { return (states == 8 ? 3 : 2) * 4 * 256; }   // of 4 SIMDs on 256 CUs
constexpr int kMaxGrid = 1 << 22;         // workgroups of a launch: HIP counts its threads in 32 bits
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
    int chunk, pieces;                    // the time axis in `pieces` pieces of `chunk` timesteps, a multiple of kPiece
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
    int blocks_of_groups;                 // workgroups of a sequence
};

// ---- arithmetic ---------------------------------------------------------------------------------------------------
// 2^x and 1 / x by the hardware's instructions, 1 unit in the last place each; 2^x is zero below 2^-126, and so are decays.
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_of(float x) { return __builtin_amdgcn_rcpf(x); }

// exp(v) for v <= 0 with the product v log2(e) in two parts: the error of a rounded product grows with |v| otherwise.
__device__ __forceinline__ float exp_of(float v) {
    const float p = v * kLog2e, e = exp2_of(p);
    const float low = fmaf(v, kLog2eLow, fmaf(v, kLog2e, -p));
    return p < -160.0f ? 0.0f : fmaf(e, low * kLn2, e);
}

// softplus(v) = max(v, 0) + log(1 + e), e = exp(-|v|), and sig(v).  log(1 + e) = 2 artanh(r) with r = e / (2 + e) <= 1/3, an odd series:
// r P(r^2) with the polynomial of degree 4 that meets it at the Chebyshev nodes of [0, 1/9], 8e-9 of the result off (an eighth of fp32's half
// step) with its coefficients rounded to fp32.  A small e loses no
// digits, which 1 + e would.
__device__ __forceinline__ float softplus_of(float v, float &sig) {
    const float e = exp_of(-fabsf(v));
    const float r = e * rcp_of(2.0f + e), q = r * r;
    float p = fmaf(q, 0.28157778f, 0.27965158f);
    p = fmaf(p, q, 0.40024595f);
    p = fmaf(p, q, 0.66666322f);
    p = fmaf(p, q, 2.00000001f);
    sig = (v >= 0.0f ? 1.0f : e) * rcp_of(1.0f + e);
    return fmaf(r, p, fmaxf(v, 0.0f));
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

__device__ __forceinline__ int length_of(const int32_t *lengths, int64_t v, int T) {
    return lengths ? min(max(as_constant(lengths)[v], 0), T) : T;
}

// What a wavefront's lane is: its channel, its quarter of the states, and where its values lie in the frames.
template <int S> struct Lane {
    static constexpr int N = 4 * S;
    int q, ch, lane;
    int64_t n, f, own;                    // own: the lane's place relative to the first of four timesteps in [T][n][f]
    __device__ __forceinline__ Lane(const Scan &s, int g, int lane_) : q(lane_ & 3), ch(g * kChannels + (lane_ >> 2)), lane(lane_), n(s.n), f(s.f) {
        own = (int64_t)q * n * f + ch;
    }
    __device__ __forceinline__ int64_t at(int64_t v, int t) const { return ((int64_t)t * n + v) * f + own; }          // of timestep t + q
    __device__ __forceinline__ int64_t state(int64_t piece, int64_t v) const { return (((piece * n + v) * f) + ch) * N + q * S; }
    __device__ __forceinline__ int64_t channel(int64_t piece, int64_t v) const { return (piece * n + v) * f + ch; }
};

// a log2(e) of a lane's states: e = 2^(dt a2).
template <int S> __device__ __forceinline__ void load_decay(float (&a2)[S], const float *a, int ch, int q) {
    const float *const p = a + (int64_t)ch * 4 * S + q * S;
    if ((reinterpret_cast<uintptr_t>(a) & 15) == 0) load_state(a2, p);            // a needs the alignment of a float only
    else
#pragma unroll
        for (int s = 0; s < S; ++s) a2[s] = p[s];
#pragma unroll
    for (int s = 0; s < S; ++s) a2[s] *= kLog2e;
}
// The same going back, the largest number of its sign where that is infinite: a state that is forgotten at once (a of minus infinity) has a decay of
// zero, which meets a2 there, and timesteps that are not there have a step size of zero; zero times infinity is NaN.
template <int S> __device__ __forceinline__ void load_decay_back(float (&a2)[S], const float *a, int ch, int q) {
    load_decay(a2, a, ch, q);
#pragma unroll
    for (int s = 0; s < S; ++s) a2[s] = fabsf(a2[s]) == __builtin_inff() ? copysignf(3.402823466e38f, a2[s]) : a2[s];
}

// Sequence v in piece p of the time axis: timesteps [t0, t1), of which the sequence has those ahead of t_end.
struct Place {
    int64_t v;
    int p, t0, t1, t_end;
    __device__ __forceinline__ bool settle(const Scan &s, int pieces) {          // after v was moved on
        if (v >= s.n) {                   // both below 2^32; one step at a time, many pieces of one sequence took 30 us to count
            const uint32_t on = (uint32_t)v / (uint32_t)s.n;
            v -= (int64_t)on * s.n;
            p += (int)on;
        }
        if (p >= pieces) return false;
        t0 = p * s.chunk;
        t1 = min(s.T, t0 + s.chunk);
        t_end = min(t1, length_of(s.lengths, v, s.T));
        return true;
    }
};

// B and C of a tile of K timesteps on their way to LDS: 16-byte pieces of its rows, in order over the lanes.
template <bool BF16, int S, int K> struct Rows {
    typedef typename Elem<BF16>::Type E;
    static constexpr int kValues = 16 / sizeof(E), kRow = 8 * S / kValues;        // values of a piece, pieces of a row
    static constexpr int kPieces = K * kRow, kLoads = (kPieces + kWave - 1) / kWave;
    uintx4 r[kLoads];
    __device__ __forceinline__ void load(const void *bc, int64_t n, int64_t v, int t, int steps, int lane) {
        const uintx4 *const p = static_cast<const uintx4 *>(bc) + ((int64_t)t * n + v) * kRow;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = i * kWave + lane, row = at / kRow;
            r[i] = uintx4{0, 0, 0, 0};                                            // rows behind the sequence: nothing
            if (row < steps) r[i] = p[(int64_t)row * n * kRow + at % kRow];
        }
    }
    // The same without a branch: rows behind the sequence are fetched from the last one's place and left out of the stage.
    __device__ __forceinline__ void load_all(const void *bc, int64_t n, int64_t v, int t, int steps, int lane) {
        const uintx4 *const p = static_cast<const uintx4 *>(bc) + ((int64_t)t * n + v) * kRow;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = i * kWave + lane;
            r[i] = p[min(at / kRow, steps - 1) * (n * kRow) + at % kRow];
        }
    }
    template <bool ALL> __device__ __forceinline__ void stage(float *to, int lane, int steps) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = i * kWave + lane;
            if (kPieces % kWave == 0 || at < kPieces) {
                float v[kValues];
                Pack<BF16>::unpack(v, !ALL || at / kRow < steps ? r[i] : uintx4{0, 0, 0, 0});
#pragma unroll
                for (int k = 0; k < kValues; k += 4) *reinterpret_cast<uintx4 *>(to + at * kValues + k) = Pack<false>::pack({v[k], v[k + 1], v[k + 2], v[k + 3]});
            }
        }
    }
};

// ---- forward ------------------------------------------------------------------------------------------------------
// What bounds it: vector instructions, then memory.  A state takes five a timestep (two products, the exponential, which holds the pipe for
// two, two multiply-adds), a lane's four 24 slots of some 34; the rest is the step sizes (25 instructions for four timesteps), the exchange of
// four timesteps' sums (9), the gate, addresses.  16 x 100003 x 64 fp32, 16 states, gated: 571 - 583 us, vector instructions in 81 % of the cycles at
// five wavefronts per SIMD, 3.9 TB/s of the 4.5 - 5.4 that copies reach; bf16 at half the bytes, bound by instructions alone, 509.
template <bool BF16, int S, int K> struct Tile {
    Rows<BF16, S, K> rows;
    float x[K / 4], delta[K / 4], z[K / 4], h[S];
};

// The tile of `steps` timesteps from t on; the state ahead of it where it is the first one of a series that is not cut into pieces.
template <bool BF16, int S, int K, bool Y, bool GATE>
__device__ __forceinline__ void load_tile(Tile<BF16, S, K> &r, const Scan &s, const Lane<S> &l, int64_t v, int t, int steps, bool first) {
    typedef typename Elem<BF16>::Type E;
    const int64_t first_at = l.at(v, t), four = 4 * s.n * s.f;
    auto values = [&](int i) {
        r.x[i] = Elem<BF16>::get(static_cast<const E *>(s.x) + first_at + i * four);
        r.delta[i] = Elem<BF16>::get(static_cast<const E *>(s.delta) + first_at + i * four);
        if (GATE) r.z[i] = Elem<BF16>::get(static_cast<const E *>(s.z) + first_at + i * four);
    };
    // No lane stands aside in a whole tile: nothing for the compiler to wait for ahead of the loads (4 - 7 %, 16 x 8192 x 128 bf16 with 32 states 148
    // us against 159; with 32 states in fp32, whose rows take twice the registers, it costs that).
    if ((S <= 4 || BF16) && steps == K) {
        r.rows.load_all(s.bc, s.n, v, t, K, l.lane);
#pragma unroll
        for (int i = 0; i < K / 4; ++i) values(i);
    } else {
        r.rows.load(s.bc, s.n, v, t, steps, l.lane);
#pragma unroll
        for (int i = 0; i < K / 4; ++i)
            if (4 * i + l.q < steps) values(i);
    }
    if (first && s.h_before && (Y ? s.pieces == 1 : t == 0)) load_state(r.h, s.h_before + l.state(0, v));
    else if (first)
#pragma unroll
        for (int k = 0; k < S; ++k) r.h[k] = 0.0f;
}

template <int S, bool Y, int J>
__device__ __forceinline__ float one_step(float (&h)[S], const float (&a2)[S], const float *row, float dt, float dtx) {
    float b[S], c[S], acc = 0.0f;
    load_state(b, row);
    if (Y) load_state(c, row + 4 * S);
    const float dt_j = of_lane<J>(dt), dtx_j = of_lane<J>(dtx);
#pragma unroll
    for (int i = 0; i < S; ++i) {
        h[i] = fmaf(exp2_of(dt_j * a2[i]), h[i], dtx_j * b[i]);
        if (Y) acc = fmaf(c[i], h[i], acc);
    }
    return acc;
}

// Y: outputs are formed (GATE: under z).  Else only what a piece of the time axis leaves behind when it starts from zero (the first: from h_before), and
// the sum of its step sizes, which gives the decay across it, exp(a sum dt).
template <bool BF16, int S, int K, bool Y, bool GATE> __device__ __forceinline__ void scan_tiles(const Scan &s, float *s_rows) {
    typedef typename Elem<BF16>::Type E;
    constexpr int N = 4 * S;
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), pieces = Y ? s.pieces : s.pieces - 1;
    const int w = blockIdx.x * kWaves + wave, stride = (int)(gridDim.x * kWaves) / s.groups;
    if (w / s.groups >= stride) return;
    float *const rows = s_rows + wave * 2 * K * 2 * N;
    const Lane<S> l(s, w % s.groups, lane);
    float a2[S], h[S], time = 0.0f;
    load_decay(a2, s.a, l.ch, l.q);
    const float bias = s.dt_bias ? s.dt_bias[l.ch] : 0.0f, d = s.d ? s.d[l.ch] : 0.0f;
    Place here{w / s.groups, 0, 0, 0, 0};
    if (!here.settle(s, pieces)) return;
    int t = here.t0, buffer = 0;
    // Loads of a tile -> what is computed with.  Loads and stores leave a wavefront in one order and are counted in it, so waiting for a
    // load is waiting for every store ahead of it too: the next tile's loads go out first, are taken up after all of this tile's arithmetic,
    // and this tile's stores follow.
    Tile<BF16, S, K> r;
    float x[K / 4], z[K / 4], dt[K / 4], start[S];
    auto take = [&](int steps, int to) {
        r.rows.template stage<false>(rows + to * K * 2 * N, lane, steps);
#pragma unroll
        for (int i = 0; i < K / 4; ++i)
            if (4 * i < steps) {
                float sig;
                x[i] = r.x[i];
                if (GATE) z[i] = r.z[i];
                dt[i] = softplus_of(r.delta[i] + bias, sig);
            }
#pragma unroll
        for (int k = 0; k < S; ++k) start[k] = r.h[k];
    };
    load_tile<BF16, S, K, Y, GATE>(r, s, l, here.v, t, min(K, here.t_end - t), true);
    take(min(K, here.t_end - t), 0);
    for (;;) {
        const int steps = min(K, here.t_end - t);
        Place next = here;
        int t_next = t + K;
        bool more = true;
        if (t_next >= here.t_end) {
            next.v += stride;
            more = next.settle(s, pieces);
            t_next = next.t0;
        }
        if (t == here.t0) {
            if (Y && s.pieces > 1) {      // what its predecessors leave (join_kernel)
                load_state(h, s.piece_state + l.state(here.p == 0 ? s.pieces - 1 : here.p - 1, here.v));
            } else
#pragma unroll
                for (int k = 0; k < S; ++k) h[k] = start[k];
            // A copy of the first piece's state ahead lies where the last one's would: the last piece's wavefront may write h_after over
            // h_before before the first one's reads it.
            if (!Y && here.p == 0) store_state(s.piece_state + l.state(s.pieces - 1, here.v), h);
            time = 0.0f;
        }
        if (Y && s.checkpoints && steps > 0) store_state(s.checkpoints + l.state(t / kHeld, here.v), h);
        if (more) load_tile<BF16, S, K, Y, GATE>(r, s, l, next.v, t_next, min(K, next.t_end - t_next), t_next == next.t0);
        wave_lds_sync();
        float y[K / 4], half[S];
        auto group = [&](int i, int left) {                 // four timesteps, of which `left` are there
            const float *const row = rows + buffer * K * 2 * N + 4 * i * 2 * N + l.q * S;
            const float dtx = dt[i] * x[i];
            if (kHeld < K && i == 2)
#pragma unroll
                for (int k = 0; k < S; ++k) half[k] = h[k];
            float out[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            out[0] = one_step<S, Y, 0>(h, a2, row, dt[i], dtx);
            if (left > 1) out[1] = one_step<S, Y, 1>(h, a2, row + 2 * N, dt[i], dtx);
            if (left > 2) out[2] = one_step<S, Y, 2>(h, a2, row + 4 * N, dt[i], dtx);
            if (left > 3) out[3] = one_step<S, Y, 3>(h, a2, row + 6 * N, dt[i], dtx);
            if (Y) {
                y[i] = fmaf(d, x[i], quad_sums(out, l.q));
                if (GATE) y[i] *= z[i] * sigmoid_of(z[i]);
            } else time += l.q < left ? dt[i] : 0.0f;
        };
        if (steps == K) {
#pragma unroll
            for (int i = 0; i < K / 4; ++i) group(i, 4);
        } else
#pragma unroll
            for (int i = 0; i < K / 4; ++i)
                if (4 * i < steps) group(i, steps - 4 * i);
        if (more) take(min(K, next.t_end - t_next), buffer ^ 1);
        if (Y) {
            const int64_t at = l.at(here.v, t), four = 4 * s.n * s.f;
            if (steps == K) {
#pragma unroll
                for (int i = 0; i < K / 4; ++i) Elem<BF16>::put(static_cast<E *>(s.y) + at + i * four, y[i]);
            } else
#pragma unroll
                for (int i = 0; i < K / 4; ++i)
                    if (4 * i + l.q < steps) Elem<BF16>::put(static_cast<E *>(s.y) + at + i * four, y[i]);
            if (kHeld < K && s.checkpoints && steps > kHeld) store_state(s.checkpoints + l.state(t / kHeld + 1, here.v), half);
        }
        if (t + K >= here.t_end) {    // the sequence ends here, or this piece of it
            if (Y) {
                for (int o = max(here.t0, here.t_end); o < here.t1; o += 4)
                    if (o + l.q < here.t1) Elem<BF16>::put(static_cast<E *>(s.y) + l.at(here.v, o), 0.0f);
                if (s.h_after && here.p == s.pieces - 1) store_state(s.h_after + l.state(0, here.v), h);
            } else {
                time = quad_sum(time);
                store_state(s.piece_state + l.state(here.p, here.v), h);
                if (l.q == 0) s.piece_time[l.channel(here.p, here.v)] = time;
            }
        }
        if (!more) return;
        here = next;
        t = t_next;
        buffer ^= 1;
    }
}

template <bool BF16, int S, bool GATE, int K> __global__ __launch_bounds__(kWaves *kWave) void scan_kernel(Scan s) {
    __shared__ float s_rows[kWaves * 2 * K * 8 * S];
    scan_tiles<BF16, S, K, true, GATE>(s, s_rows);
}
// Where there are few sequences the time axis is cut into pieces, and this goes ahead over all but the last one: 3 x 16411 x 128 bf16 in 147
// pieces takes 31 us here, 7 to join and 40 for the outputs, where one wavefront per sixteen channels would walk 1026 tiles, 2 us each.
template <bool BF16, int S> __global__ __launch_bounds__(kWaves *kWave) void scan_piece_kernel(Scan s) {
    __shared__ float s_rows[kWaves * 2 * kTile * 8 * S];
    scan_tiles<BF16, S, kTile, false, false>(s, s_rows);
}

// One timestep, the step of a model that follows a running series: a wavefront per sixteen channels of a sequence and no more.  The state
// comes and goes (8 N bytes a channel against 4 x 2 or 4 of everything else), and what streams it is many wavefronts that are soon done:
// 100000 x 128 fp32 350 us against 479 by the kernel that walks, 16 x 128 3.5 against 4.7.  60013 x 64 bf16: 107 us, 4.9 TB/s.
template <bool BF16, int S, bool GATE> __global__ __launch_bounds__(kWaves *kWave) void scan_step_kernel(Scan s) {
    typedef typename Elem<BF16>::Type E;
    constexpr int N = 4 * S;
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
    for (int64_t i = (int64_t)blockIdx.x * kWaves + wave; i < s.n * s.groups; i += (int64_t)gridDim.x * kWaves) {
        const bool narrow = i >> 32 == 0;
        const int64_t v = narrow ? (uint32_t)i / (uint32_t)s.groups : i / s.groups;
        const Lane<S> l(s, (int)(i - v * s.groups), lane);
        const int64_t at = v * s.f + l.ch;
        float h[S], a2[S], b[S], c[S];
        if (s.h_before) load_state(h, s.h_before + l.state(0, v));
        else
#pragma unroll
            for (int k = 0; k < S; ++k) h[k] = 0.0f;
        if (length_of(s.lengths, v, 1) == 0) {
            if (l.q == 0) Elem<BF16>::put(static_cast<E *>(s.y) + at, 0.0f);
            if (s.h_after) store_state(s.h_after + l.state(0, v), h);
            continue;
        }
        const E *const row = static_cast<const E *>(s.bc) + v * 2 * N + l.q * S;
        Elem<BF16>::template row<S>(b, row);
        Elem<BF16>::template row<S>(c, row + N);
        const float x = Elem<BF16>::get(static_cast<const E *>(s.x) + at), delta = Elem<BF16>::get(static_cast<const E *>(s.delta) + at);
        const float z = GATE ? Elem<BF16>::get(static_cast<const E *>(s.z) + at) : 0.0f;
        load_decay(a2, s.a, l.ch, l.q);
        if (s.checkpoints) store_state(s.checkpoints + l.state(0, v), h);
        float sig, y = 0.0f;
        const float dt = softplus_of(delta + (s.dt_bias ? s.dt_bias[l.ch] : 0.0f), sig), dtx = dt * x;
#pragma unroll
        for (int k = 0; k < S; ++k) {
            h[k] = fmaf(exp2_of(dt * a2[k]), h[k], dtx * b[k]);
            y = fmaf(c[k], h[k], y);
        }
        // the sum in the order of quad_sums, so that a series taken step by step gives the same bits
        y += dpp<0x4e>(y);
        y += dpp<0xb1>(y);
        y = fmaf(s.d ? s.d[l.ch] : 0.0f, x, y);
        if (GATE) y *= z * sigmoid_of(z);
        if (s.h_after) store_state(s.h_after + l.state(0, v), h);
        if (l.q == 0) Elem<BF16>::put(static_cast<E *>(s.y) + at, y);
    }
}

// The states between the pieces, in place.  Forward (STEP 1): piece p left part[p] behind when it started from zero, part[0] from h_before;
// the state ahead of piece p takes the place p - 1.  Backward (STEP -1): the same from the last piece on, which dh_after reaches; what
// reaches piece p from behind takes the place p + 1.  A thread has one state of one of RUNS runs of at most kJoin pieces, which are fetched
// together: what a run does to a state (its own part, its decay) first, then the same of all runs up to each, twice as many with every step,
// then its pieces.  147 pieces of 6144 states: 7 us; the memory trips (the pieces' states come from other dies' wavefronts) are what it takes.
// As few runs as hold the pieces: loads that a run has no piece for cost as much as others (16 sequences of 4096 x 128 in 32 pieces: 80 us with
// four runs, 93 with 32; 128 of 64 x 128 in two: 36 with one, 43 with four).
constexpr int kJoin = 16, kJoinRuns = 32;
constexpr int join_states(int runs) { return runs == 1 ? 256 : runs == 4 ? 64 : 32; }         // of a workgroup
// 2^(time a2) h.  The exponent goes in last: across pieces of a series whose states may grow (a > 0) the factor alone leaves fp32 where the
// state does not, and no timestep leaves it as it is whatever a is.
__device__ __forceinline__ float across(float h, float time, float a2) {
    const float p = time == 0.0f ? 0.0f : fminf(fmaxf(time * a2, -4096.0f), 4096.0f), whole = floorf(p);
    return ldexpf(h * exp2_of(p - whole), (int)whole);
}
template <int STEP, int RUNS> __global__ __launch_bounds__(RUNS *join_states(RUNS)) void join_kernel(Scan s, const float *behind, uint32_t states) {
    constexpr int STATES = join_states(RUNS);
    __shared__ float s_part[RUNS][STATES], s_time[RUNS][STATES];
    // Series in pieces are few: a place among the states of all of them is a 32-bit number.  Beyond the last state: that one once more.
    const uint32_t channels = (uint32_t)s.n * (uint32_t)s.f, width = channels * states;
    const int o = threadIdx.x % STATES, run = threadIdx.x / STATES;
    const uint32_t at = blockIdx.x * STATES + o, i = min(at, width - 1), c = i / states;
    const float a2 = s.a[i % ((uint32_t)s.f * states)] * kLog2e;
    const int first = STEP > 0 ? 1 : s.pieces - 1, count = s.pieces - (STEP > 0 ? 2 : 1), per = (count + RUNS - 1) / RUNS;
    const int k0 = run * per, k1 = min(count, k0 + per);
    float part[kJoin], step[kJoin];
#pragma unroll
    for (int j = 0; j < kJoin; ++j) {
        const uint64_t p = first + STEP * min(k0 + j, count - 1);
        part[j] = s.piece_state[p * width + i];
        step[j] = s.piece_time[p * channels + c];
    }
    float h = STEP > 0 ? s.piece_state[i] : behind ? behind[i] : 0.0f;
    if (RUNS > 1) {
        float own = 0.0f, time = 0.0f;
#pragma unroll
        for (int j = 0; j < kJoin; ++j)
            if (k0 + j < k1) { own = across(own, step[j], a2) + part[j]; time += step[j]; }
#pragma unroll
        for (int d = 1; d < RUNS; d <<= 1) {
            s_part[run][o] = own;
            s_time[run][o] = time;
            __syncthreads();
            const float before = run >= d ? s_part[run - d][o] : 0.0f, time_before = run >= d ? s_time[run - d][o] : 0.0f;
            __syncthreads();
            own += across(before, time, a2);
            time += time_before;
        }
        s_part[run][o] = own;
        s_time[run][o] = time;
        __syncthreads();
        if (run > 0) h = across(h, s_time[run - 1][o], a2) + s_part[run - 1][o];
    }
#pragma unroll
    for (int j = 0; j < kJoin; ++j)
        if (k0 + j < k1) {
            h = across(h, step[j], a2) + part[j];
            if (at < width) s.piece_state[(uint64_t)(first + STEP * (k0 + j)) * width + i] = h;
        }
}

// ---- backward -----------------------------------------------------------------------------------------------------
// dL/dh as a piece hands it to its predecessor when nothing reaches it from behind, and the sum of its step sizes (4 x 1025 x 1536 bf16: 40 us
// against the 112 of the kernel below).
template <bool BF16, int S>
__global__ __launch_bounds__(kWaves *kWave) void scan_back_piece_kernel(ScanBack b) {
    typedef typename Elem<BF16>::Type E;
    constexpr int N = 4 * S, R = kTile / 4;
    __shared__ float s_rows[kWaves * kTile * 2 * N];
    const Scan &s = b.s;
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
    const int w = blockIdx.x * kWaves + wave, stride = (int)(gridDim.x * kWaves) / s.groups;
    if (w / s.groups >= stride) return;
    float *const rows = s_rows + wave * kTile * 2 * N;
    const Lane<S> l(s, w % s.groups, lane);
    const float bias = s.dt_bias ? s.dt_bias[l.ch] : 0.0f;
    float a2[S];
    load_decay_back(a2, s.a, l.ch, l.q);
    for (Place here{w / s.groups, 1, 0, 0, 0}; here.settle(s, s.pieces); here.v += stride) {
        Rows<BF16, S, kTile> bc;
        float k[S], time = 0.0f, delta[R], gy[R], z[R];
#pragma unroll
        for (int i = 0; i < S; ++i) k[i] = 0.0f;
        auto load = [&](int t) {
            const int steps = here.t_end - t;
            bc.load(s.bc, s.n, here.v, t, steps, lane);
            const int64_t at = l.at(here.v, t), four = 4 * s.n * s.f;
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (4 * i + l.q < steps) {
                    delta[i] = Elem<BF16>::get(static_cast<const E *>(s.delta) + at + i * four);
                    gy[i] = Elem<BF16>::get(static_cast<const E *>(b.g_y) + at + i * four);
                    if (s.z) z[i] = Elem<BF16>::get(static_cast<const E *>(s.z) + at + i * four);
                }
        };
        int t = here.t0 + (here.t_end - here.t0 - 1) / kTile * kTile;
        if (here.t_end > here.t0) load(t);
        else t = here.t0 - 1;
        for (; t >= here.t0; t -= kTile) {
            const int steps = min(kTile, here.t_end - t);
            float dt[R], g[R];
            bc.template stage<false>(rows, lane, steps);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float sig;
                dt[i] = softplus_of(delta[i] + bias, sig);
                g[i] = gy[i];
                if (s.z) g[i] *= z[i] * sigmoid_of(z[i]);
                if (4 * i + l.q >= steps) dt[i] = g[i] = 0.0f;            // decay 1, nothing added: rows behind the sequence are zero
                time += dt[i];
            }
            wave_lds_sync();
            if (t > here.t0) load(t - kTile);
            auto four = [&](int i) {
                auto step = [&](int j, float dt_j, float g_j) {
                    float c[S];
                    load_state(c, rows + (4 * i + j) * 2 * N + N + l.q * S);
#pragma unroll
                    for (int m = 0; m < S; ++m) k[m] = exp2_of(dt_j * a2[m]) * fmaf(c[m], g_j, k[m]);
                };
                step(3, of_lane<3>(dt[i]), of_lane<3>(g[i]));
                step(2, of_lane<2>(dt[i]), of_lane<2>(g[i]));
                step(1, of_lane<1>(dt[i]), of_lane<1>(g[i]));
                step(0, of_lane<0>(dt[i]), of_lane<0>(g[i]));
            };
#pragma unroll
            for (int i = R - 1; i >= 0; --i)
                if (4 * i < steps) four(i);
            wave_lds_sync();
        }
        time = quad_sum(time);
        store_state(s.piece_state + l.state(here.p, here.v), k);
        if (l.q == 0) s.piece_time[l.channel(here.p, here.v)] = time;
    }
}

// Timesteps of a tile of the adjoint at most: what a wavefront fetches ahead.  Sixteen with 16 states (256 x 512 x 128 bf16: 268 us against 294 with eight;
// 16 x 8192 x 128 fp32 276 against 271); with 8 states, at three wavefronts per SIMD, eight (187 against 216).  With 32 the registers are short with
// eight already: all 256 are in use and 38 - 60 values a lane go through scratch memory; with sixteen it is 180 - 268 (16 x 4096 x 128 fp32: 281 us
// against 929).
template <int S> constexpr int kBackTile = S == 4 ? 16 : 8;
// Whether a tile's loads are all made, whatever is there of it.  With 32 states, where the registers are short, the loads that a branch may
// pass over cost more (16 x 8192 x 128 fp32: 859 us against 556), and with 16 in bf16 (256 x 512 x 128: 299 against 268); with 16 in fp32 and with
// 8 it makes no difference in whole tiles (16 x 8192 x 128: 276 and 280; 7 x 20000 x 64: 186 and 187; 8 states 187 and 185), and nothing is loaded that is not there.
template <bool BF16, int S> constexpr bool kAllLoads = S > 4 || (BF16 && S == 4);

template <bool BF16, int S, int K> struct BackTile {
    Rows<BF16, S, K> rows;
    float x[K / 4], delta[K / 4], gy[K / 4], z[K / 4], h[K / kHeld][S], k[S];
};

// `k`: what reaches the last tile of a piece from behind.
template <bool BF16, int S, int K, bool GATE>
__device__ __forceinline__ void load_back_tile(BackTile<BF16, S, K> &r, const ScanBack &b, const Lane<S> &l, const Place &p, int t, int steps, bool last) {
    typedef typename Elem<BF16>::Type E;
    const Scan &s = b.s;
    const int64_t first = l.at(p.v, t), frame = s.n * s.f;
    auto values = [&](int i, int64_t at) {
        r.x[i] = Elem<BF16>::get(static_cast<const E *>(s.x) + at);
        r.delta[i] = Elem<BF16>::get(static_cast<const E *>(s.delta) + at);
        r.gy[i] = Elem<BF16>::get(static_cast<const E *>(b.g_y) + at);
        if (GATE) r.z[i] = Elem<BF16>::get(static_cast<const E *>(s.z) + at);
    };
    if (kAllLoads<BF16, S>) {
        steps = min(max(steps, 1), K);
        r.rows.load_all(s.bc, s.n, p.v, t, steps, l.lane);
#pragma unroll
        for (int i = 0; i < K / 4; ++i) values(i, first + (min(4 * i + l.q, steps - 1) - l.q) * frame);
#pragma unroll
        for (int i = 0; i < K / kHeld; ++i) load_state(r.h[i], s.checkpoints + l.state(t / kHeld + (i * kHeld < steps ? i : 0), p.v));
    } else {
        r.rows.load(s.bc, s.n, p.v, t, steps, l.lane);
#pragma unroll
        for (int i = 0; i < K / 4; ++i)
            if (4 * i + l.q < steps) values(i, first + 4 * i * frame);
#pragma unroll
        for (int i = 0; i < K / kHeld; ++i)
            if (i * kHeld < steps) load_state(r.h[i], s.checkpoints + l.state(t / kHeld + i, p.v));
    }
    if (last && p.p < s.pieces - 1) load_state(r.k, s.piece_state + l.state(p.p + 1, p.v));
    else if (last && b.dh_after) load_state(r.k, b.dh_after + l.state(0, p.v));
    else if (last)
#pragma unroll
        for (int i = 0; i < S; ++i) r.k[i] = 0.0f;
}

// A workgroup has all channels of a sequence, or a part of them (of back_waves() wavefronts).  Eight timesteps are walked ahead from a kept state
// (five instructions a state and timestep) and back again (eight, and 4 for the sums over channels): some 108 a timestep and lane with 16
// states, and they are what bounds it: 16 x 50021 x 32 fp32 takes 425 us with vector instructions in 80 % of the cycles at two wavefronts per SIMD, 2.9
// TB/s with the forward pass.  The exchange over channels is 16 of them, its cost when left out 19 %; the matrix cores would take the sums at the same number of
// issue slots.  16 x 8192 x 128 fp32: 187 us with 8 states, 276 with 16; 16 x 4096 x 128 with 32 (which spill): 281, bf16 276.
template <bool BF16, int S, bool GATE, int K>
__global__ __launch_bounds__(back_waves(4 * S) * kWave) void scan_back_kernel(ScanBack b) {
    typedef typename Elem<BF16>::Type E;
    constexpr int N = 4 * S, R = K / 4, V = K * 2 * N;  // V: values of dB and dC of a tile
    constexpr int J = S <= 4 ? 4 : 2;                                     // timesteps whose sums over channels are exchanged together
    // With 32 states in fp32 what two fours have in flight together does not fit the registers: they stay apart (16 x 4096 x 128: 281 us against 294);
    // in bf16 they do not (276 against 289).
    constexpr bool kFence = S > 4 && !BF16;
    // [3][wavefronts][V], the three by turns: B and C of a tile, where dB and dC take their place timestep by timestep (the next tile's B
    // and C are laid down when a slower wavefront may still be adding up this one's dB and dC); 64-bit sums.  Decays are formed twice: kept here
    // on the way ahead they took 2 - 4 % longer.
    extern __shared__ float s_mem[];
    const Scan &s = b.s;
    const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int part = blockIdx.x % b.blocks_of_groups, slot = blockIdx.x / b.blocks_of_groups, slots = gridDim.x / b.blocks_of_groups;
    const int g = part * back_waves(N) + wave, active = min(waves, s.groups - part * back_waves(N));
    if (wave >= active) return;                                           // the last part may be narrower; a barrier waits for those that are left
    const Lane<S> l(s, g, lane);
    const int q = l.q, turn = waves * V;
    float a2[S], acc[S + 2];                                              // sums over a few tiles: da of the lane's states, dd, ddt_bias
    load_decay_back(a2, s.a, l.ch, q);
    double *const sums = reinterpret_cast<double *>(s_mem + 3 * turn) + wave * (S + 2) * kWave + lane;
#pragma unroll
    for (int i = 0; i < S + 2; ++i) { sums[i * kWave] = 0.0; acc[i] = 0.0f; }
    const float bias = s.dt_bias ? s.dt_bias[l.ch] : 0.0f, d = s.d ? s.d[l.ch] : 0.0f;
    const int at_place = J * 2 * S / 16 * place_of(lane);                 // the first value a lane has after the exchange, and where it belongs
    const int to_place = at_place / (2 * S) * 2 * N + at_place % (2 * S) / S * N + q * S + at_place % S;
    // the thread's first value among a tile's dB and dC; values kWave further on are whole rows further on, or the same row's
    const int row_first = threadIdx.x / (2 * N);
    const int64_t row_at = (int64_t)row_first * s.n * 2 * N + threadIdx.x % (2 * N);
    float *const part_out = b.dbc_part ? b.dbc_part + (int64_t)part * s.T * s.n * 2 * N : nullptr;
    auto last_tile = [&](const Place &p) { return p.t0 + (p.t1 - p.t0 - 1) / K * K; };
    Place here{slot, 0, 0, 0, 0};
    bool more = here.settle(s, s.pieces);
    int t = more ? last_tile(here) : 0, buffer = 0;
    // the lane's own timesteps: t + 4 i + q
    float x[R], dt[R], sig[R], gp[R], gz[R], h0[K / kHeld][S], k[S], from_behind[S];
    BackTile<BF16, S, K> r;
    auto take = [&](int steps, float *to) {
        r.rows.template stage<kAllLoads<BF16, S>>(to, lane, steps);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            x[i] = r.x[i];
            dt[i] = softplus_of(r.delta[i] + bias, sig[i]);
            gp[i] = r.gy[i];
            if (GATE) {
                const float z = r.z[i], sz = sigmoid_of(z);
                gz[i] = gp[i] * sz * fmaf(z, 1.0f - sz, 1.0f);
                gp[i] *= z * sz;
            }
            if (4 * i + q >= steps) x[i] = dt[i] = gp[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < K / kHeld; ++i)
#pragma unroll
            for (int m = 0; m < S; ++m) h0[i][m] = r.h[i][m];
#pragma unroll
        for (int i = 0; i < S; ++i) from_behind[i] = r.k[i];
    };
    if (more) {
        load_back_tile<BF16, S, K, GATE>(r, b, l, here, t, min(K, here.t_end - t), true);
        take(min(K, here.t_end - t), s_mem + wave * V);
    }
    while (more) {
        const int steps = min(K, here.t_end - t);
        float *const rows = s_mem + buffer * turn + wave * V;
        const int ahead_buffer = buffer == 2 ? 0 : buffer + 1;
        Place next = here;
        int t_next = t - K;
        if (t_next < here.t0) {
            next.v += slots;
            more = next.settle(s, s.pieces);
            t_next = more ? last_tile(next) : 0;
        }
        if (t == last_tile(here))
#pragma unroll
            for (int i = 0; i < S; ++i) k[i] = from_behind[i];
        // The next tile's loads go out now and are taken up behind this one's stores, whose number is known: loads and stores are counted in
        // one order, and waiting for the loads is waiting until no more than the stores are left.
        const int steps_next = min(K, next.t_end - t_next);
        if (more) load_back_tile<BF16, S, K, GATE>(r, b, l, next, t_next, steps_next, t_next == last_tile(next));
        const int64_t at = l.at(here.v, t), four = 4 * s.n * s.f;
        wave_lds_sync();
        float h[S], held[kHeld][S];
        auto ahead = [&](auto whole, int i) {         // forward over four timesteps of the tile, their states kept
            float part_y[4];
            const float dtx = dt[i] * x[i];
            auto step = [&](int j, float dt_j, float dtx_j) {
                const float *const row = rows + (4 * i + j) * 2 * N;
                float rb[S], rc[S];
                load_state(rb, row + q * S);
                if (GATE) load_state(rc, row + N + q * S);
                part_y[j] = 0.0f;
#pragma unroll
                for (int m = 0; m < S; ++m) {
                    held[(4 * i + j) % kHeld][m] = h[m];
                    h[m] = fmaf(exp2_of(dt_j * a2[m]), h[m], dtx_j * rb[m]);
                    if (GATE) part_y[j] = fmaf(rc[m], h[m], part_y[j]);
                }
            };
            step(0, of_lane<0>(dt[i]), of_lane<0>(dtx));
            step(1, of_lane<1>(dt[i]), of_lane<1>(dtx));
            step(2, of_lane<2>(dt[i]), of_lane<2>(dtx));
            step(3, of_lane<3>(dt[i]), of_lane<3>(dtx));
            if (GATE) {
                const float dz = gz[i] * fmaf(d, x[i], quad_sums(part_y, q));
                if (decltype(whole)::value || 4 * i + q < steps) Elem<BF16>::put(static_cast<E *>(b.dz) + at + i * four, dz);
            }
            if (kFence) __builtin_amdgcn_sched_barrier(0);
        };
        auto back = [&](auto whole, int i) {          // ... and back over them
            float bc[J * 2 * S], ghb[4], sa[4];
            const float dtx = dt[i] * x[i];
            auto step = [&](int j, float dt_j, float dtx_j, float g_j) {
                const float *const row = rows + (4 * i + j) * 2 * N;
                float rb[S], rc[S];
                load_state(rb, row + q * S);
                load_state(rc, row + N + q * S);
                ghb[j] = sa[j] = 0.0f;
#pragma unroll
                for (int m = 0; m < S; ++m) {
                    const float gh = fmaf(rc[m], g_j, k[m]);
                    bc[j % J * 2 * S + m] = gh * dtx_j;
                    bc[j % J * 2 * S + S + m] = h[m] * g_j;
                    ghb[j] = fmaf(gh, rb[m], ghb[j]);
                    h[m] = held[(4 * i + j) % kHeld][m];
                    k[m] = gh * exp2_of(dt_j * a2[m]);
                    const float u = k[m] * h[m];
                    sa[j] = fmaf(u, a2[m], sa[j]);
                    acc[m] = fmaf(u, dt_j, acc[m]);
                }
            };
            // value v of the exchange = step * 2 S + (B or C) * S + state; a lane ends up with J 2 S / 16 of them
            auto leave = [&](int j0) {
                channel_sums<J * 2 * S>(bc, lane);
#pragma unroll
                for (int m = 0; m < J * 2 * S / 16; ++m) rows[(4 * i + j0) * 2 * N + to_place + m] = bc[m];
            };
            step(3, of_lane<3>(dt[i]), of_lane<3>(dtx), of_lane<3>(gp[i]));
            step(2, of_lane<2>(dt[i]), of_lane<2>(dtx), of_lane<2>(gp[i]));
            if (J == 2) leave(2);
            step(1, of_lane<1>(dt[i]), of_lane<1>(dtx), of_lane<1>(gp[i]));
            step(0, of_lane<0>(dt[i]), of_lane<0>(dtx), of_lane<0>(gp[i]));
            leave(0);
            const float gb = quad_sums(ghb, q), da = quad_sums(sa, q) * kLn2;
            const float ddelta = fmaf(x[i], gb, da) * sig[i];
            if (decltype(whole)::value || 4 * i + q < steps) {
                Elem<BF16>::put(static_cast<E *>(b.dx) + at + i * four, fmaf(d, gp[i], dt[i] * gb));
                Elem<BF16>::put(static_cast<E *>(b.ddelta) + at + i * four, ddelta);
                acc[S] = fmaf(gp[i], x[i], acc[S]);
                acc[S + 1] += ddelta;
            }
            if (kFence) __builtin_amdgcn_sched_barrier(0);
        };
        auto start = [&](int half) {
#pragma unroll
            for (int m = 0; m < S; ++m) h[m] = h0[half][m];
        };
        if (steps == K) {
            const std::true_type whole;
            start(K / kHeld - 1);
            ahead(whole, R - 2);
            ahead(whole, R - 1);
            back(whole, R - 1);
            back(whole, R - 2);
            if (K > kHeld) {
                start(0);
                ahead(whole, 0);
                ahead(whole, 1);
                back(whole, 1);
                back(whole, 0);
            }
            if (more) take(steps_next, s_mem + ahead_buffer * turn + wave * V);
        } else {                          // fours of which nothing is there are left out; what is missing of the last one is zero
            const std::false_type whole;
#pragma unroll
            for (int half = K / kHeld - 1; half >= 0; --half)
                if (half * kHeld < steps) {
                    start(half);
                    ahead(whole, 2 * half);
                    if (half * kHeld + 4 < steps) {
                        ahead(whole, 2 * half + 1);
                        back(whole, 2 * half + 1);
                    }
                    back(whole, 2 * half);
                }
            for (int o = max(steps, 0); o < K; o += 4)
                if (o + q < K && t + o + q < here.t1) {
                    const int64_t to = l.at(here.v, t + o);
                    Elem<BF16>::put(static_cast<E *>(b.dx) + to, 0.0f);
                    Elem<BF16>::put(static_cast<E *>(b.ddelta) + to, 0.0f);
                    if (GATE) Elem<BF16>::put(static_cast<E *>(b.dz) + to, 0.0f);
                }
            if (more) take(steps_next, s_mem + ahead_buffer * turn + wave * V);
        }
        if ((t & 63) == 0 || t == here.t0)
#pragma unroll
            for (int i = 0; i < S + 2; ++i) { sums[i * kWave] += (double)acc[i]; acc[i] = 0.0f; }
        block_lds_sync();
        // dB and dC of the tile over the workgroup's channels: reads by fours, those beyond the last wavefront of its own
        const float *const all = s_mem + buffer * turn + threadIdx.x;
        const int64_t tile_at = ((int64_t)t * s.n + here.v) * 2 * N + row_at;
#pragma unroll 2
        for (int i = 0; i < V / kWave; i += active)
            if (i * kWave + (int)threadIdx.x < V && t + row_first + i * kWave / (2 * N) < here.t1) {
                float sum = 0.0f;
                for (int o = 0; o < active; o += 4) {
                    float v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = all[min(o + u, active - 1) * V + i * kWave];
#pragma unroll
                    for (int u = 0; u < 4; ++u) sum += o + u < active ? v[u] : 0.0f;
                }
                if (row_first + i * kWave / (2 * N) >= steps) sum = 0.0f;
                const int64_t to = tile_at + i * (kWave * s.n);
                if (b.dbc_part) part_out[to] = sum;
                else Elem<BF16>::put(static_cast<E *>(b.dbc) + to, sum);
            }
        if (b.dh_before && here.p == 0 && t == here.t0) store_state(b.dh_before + l.state(0, here.v), k);
        buffer = ahead_buffer;
        here = next;
        t = t_next;
    }
    // sums over time and sequences
    double *to = b.sums + (int64_t)slot * s.f * (N + 2);
#pragma unroll
    for (int i = 0; i < S; ++i) to[(int64_t)l.ch * N + q * S + i] = sums[i * kWave];
    double sum_d = sums[S * kWave], sum_bias = sums[(S + 1) * kWave];
    sum_d += __shfl_xor(sum_d, 1);
    sum_d += __shfl_xor(sum_d, 2);
    sum_bias += __shfl_xor(sum_bias, 1);
    sum_bias += __shfl_xor(sum_bias, 2);
    if (q == 0) { to[(int64_t)s.f * N + l.ch] = sum_d; to[(int64_t)s.f * (N + 1) + l.ch] = sum_bias; }
}

// da | dd | ddt_bias from the workgroups' sums, 64 strided parts of them added up in a fixed order.
__global__ __launch_bounds__(1024) void scan_sums_kernel(const double *__restrict__ sums, int slots, int states, int rest, float *__restrict__ da, float *__restrict__ dd,
                                                         float *__restrict__ ddt_bias, int accumulate) {
    __shared__ double s_part[64][17];
    const int o = threadIdx.x % 16, r = threadIdx.x / 16, at = blockIdx.x * 16 + o, width = states + 2 * rest;
    double sum = 0.0;
    if (at < width)
#pragma unroll 4
        for (int k = r; k < slots; k += 64) sum += sums[(int64_t)k * width + at];
    s_part[r][o] = sum;
    __syncthreads();
    if (r == 0 && at < width) {
#pragma unroll 7
        for (int k = 1; k < 64; ++k) sum += s_part[k][o];
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
    if (!fits_index(n) || T > (int64_t(1) << 30) || T > (int64_t(1) << 44) / n) return DGNN_ERR_OVERFLOW;
    return DGNN_OK;                       // a place behind the last piece still is an int
}

// Tiles of eight timesteps where the series is short: half the loads that nothing is there for, fewer registers, more wavefronts (fp32, 16 x 100003 x
// 64 with the state handed on: 650 us against 691; 40 x 3200 x 64 42 against 46; 57 x 1501 x 48 the same; 256 x 256 x 128 53 against 49).  bf16 from
// twelve timesteps down (8 x 16000 x 64 48 us against 57, 12 x 11000 x 64 51 against 54; 16 x 100003 x 64 591 against 563).
bool short_ahead(int64_t T, dgnn_dtype dt) { return T <= (dt == DGNN_F32 ? 48 : 12); }
// The adjoint with 16 states likewise: 8 x 16000 x 64 145 us against 171, bf16 142 against 178; 12 x 11000 x 64 156 against 162, bf16 164 against
// 157; 16 x 50021 x 32 447 against 413.
bool short_back(int64_t T) { return T <= 8; }

struct Pieces { int chunk, count; };

// The time axis in pieces of whole tiles where there is less work across it than the device holds: `items` walks side by side (going ahead a wavefront's,
// going back a workgroup's) out of `wanted`.  Every piece is walked twice, so going ahead fewer than four do not pay (2^17 x 128 channels, two pieces: 226
// us against 198); going back, where the first walk is a quarter of the second, two do (128 sequences of 256 x 128: 106 us against 140).
// The fewest timesteps weigh the second walk against the launches: 64 ahead (80 of 16 sequences 10.9 us against 11.9, 64 of them 12.2 against
// 11.1), 32 back (48 of two: 20 against 29 us, 32 of a hundred: 24.7 against 22.6).  Twice as many tiles to a piece cost 10 - 20 % at a few hundred
// timesteps (16 sequences of 128 x 64: 14.5 us for 12.1); no more pieces than one join takes.
Pieces pieces_of(int64_t T, int64_t items, int64_t wanted, int64_t least, int64_t least_tiles) {
    const int64_t tiles = (T + kPiece - 1) / kPiece;
    const int64_t count = std::min<int64_t>({tiles, wanted / items, kJoinRuns * kJoin});
    if (count < least || tiles < least_tiles) return {(int)(tiles * kPiece), 1};
    const int64_t chunk = (tiles + count - 1) / count * kPiece;
    return {(int)chunk, (int)((T + chunk - 1) / chunk)};
}

Pieces forward_pieces(int64_t T, int64_t n, int32_t f) { return pieces_of(T, n * (f / kChannels), 4096, 4, 5); }

struct BackShape { int groups, blocks_of_groups, waves; Pieces pieces; int64_t slots; };

BackShape back_shape(int64_t T, int64_t n, int32_t f, int32_t N) {
    BackShape b;
    b.groups = f / kChannels;
    b.blocks_of_groups = (b.groups + back_waves(N) - 1) / back_waves(N);
    b.waves = std::min(b.groups, back_waves(N));
    const int64_t blocks = std::max(1, back_resident(N) / (b.waves * b.blocks_of_groups));
    b.pieces = pieces_of(T, n, blocks, 2, 3);
    b.slots = std::min<int64_t>(n * b.pieces.count, blocks);
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

// Wavefronts that stay: as many workgroups as the device holds, or as there is work for.  All channels of a sequence have one (there are
// at most 1024 groups of them, and never fewer than 256 workgroups at once).
template <typename K> dim3 walk_grid(K kernel, const Scan &s, int pieces) {
    const int64_t work = (s.n * s.groups * pieces + kWaves - 1) / kWaves;
    return dim3((unsigned)std::min<int64_t>(work, std::max<int64_t>(DGNN_MAX_CHANNELS / kChannels / kWaves, resident_workgroups(kernel, kWaves * kWave, 1024))));
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

template <int STEP> int join_pieces(const Scan &s, const float *behind, int32_t states, hipStream_t st) {
    const int64_t width = s.n * s.f * states;
    auto launch = [&](auto runs) {
        constexpr int RUNS = decltype(runs)::value, STATES = join_states(RUNS);
        hipLaunchKernelGGL((join_kernel<STEP, RUNS>), dim3((unsigned)((width + STATES - 1) / STATES)), dim3(RUNS * STATES), 0, st, s, behind, (uint32_t)states);
    };
    if (s.pieces > 4 * kJoin) launch(std::integral_constant<int, kJoinRuns>{});
    else if (s.pieces > kJoin) launch(std::integral_constant<int, 4>{});
    else launch(std::integral_constant<int, 1>{});
    DGNN_RETURN_IF_LAUNCH_FAILED();
    return DGNN_OK;
}

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

}  // namespace

extern "C" int dgnn_selective_scan_checkpoints(int64_t T, int64_t n, int32_t f, int32_t states, size_t *bytes) {
    if (!bytes) return DGNN_ERR_NULL;
    if (int rc = check_shape(T, n, f, states)) return rc;
    *bytes = (size_t)((T + kHeld - 1) / kHeld) * n * f * states * sizeof(float);
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
    if (!words_aligned({a, d, dt_bias, lengths})) return DGNN_ERR_ALIGN;
    const size_t vector = sizeof(float) * f, ends = sizeof(int32_t) * n;
    const size_t frame = (size_t)T * n * f * (dt == DGNN_F32 ? 4 : 2), rows = (size_t)T * n * 2 * states * (dt == DGNN_F32 ? 4 : 2);
    const size_t state = (size_t)n * f * states * sizeof(float), kept = (size_t)((T + kHeld - 1) / kHeld) * state;
    for (auto o : {std::pair<const void *, size_t>{y, frame}, {h_after, state}, {checkpoints, kept}, {ws, ws_bytes}}) {
        for (auto i : {std::pair<const void *, size_t>{x, frame}, {delta, frame}, {bc, rows}, {z, frame}, {a, vector * states}, {d, vector}, {dt_bias, vector}, {lengths, ends}})
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
            const auto kernel = scan_piece_kernel<decltype(bf16)::value, decltype(per)::value>;
            hipLaunchKernelGGL(kernel, walk_grid(kernel, s, s.pieces - 1), dim3(kWaves * kWave), 0, st, s);
        });
        if (rc) return rc;
        if (s.pieces > 2) {
            if (const int failed = join_pieces<1>(s, nullptr, states, st)) return failed;
        }
    }
    if (T == 1)
        return by_kind(dt, states, [&](auto bf16, auto per) {
            const auto kernel = z ? scan_step_kernel<decltype(bf16)::value, decltype(per)::value, true> : scan_step_kernel<decltype(bf16)::value, decltype(per)::value, false>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((n * s.groups + kWaves - 1) / kWaves, kMaxGrid)), dim3(kWaves * kWave), 0, st, s);
        });
    return by_kind(dt, states, [&](auto bf16, auto per) {
        auto launch = [&](auto tile) {
            constexpr int K = decltype(tile)::value;
            const auto kernel = z ? scan_kernel<decltype(bf16)::value, decltype(per)::value, true, K> : scan_kernel<decltype(bf16)::value, decltype(per)::value, false, K>;
            hipLaunchKernelGGL(kernel, walk_grid(kernel, s, s.pieces), dim3(kWaves * kWave), 0, st, s);
        };
        if (short_ahead(T, dt)) launch(std::integral_constant<int, kHeld>{});
        else launch(std::integral_constant<int, kTile>{});
    });
}

extern "C" int dgnn_selective_scan_backward_workspace(int64_t T, int64_t n, int32_t f, int32_t states, size_t *bytes) {
    if (!bytes) return DGNN_ERR_NULL;
    if (int rc = check_shape(T, n, f, states)) return rc;
    const BackShape b = back_shape(T, n, f, states);
    *bytes = piece_bytes(b.pieces, n, f, states) + round_up((size_t)b.slots * f * (states + 2) * sizeof(double), 256) +
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
    if (!words_aligned({a, d, dt_bias, lengths, da, dd, ddt_bias})) return DGNN_ERR_ALIGN;
    size_t need = 0;
    dgnn_selective_scan_backward_workspace(T, n, f, states, &need);
    if (ws_bytes < need) return DGNN_ERR_CAPACITY;
    const size_t frame = (size_t)T * n * f * (dt == DGNN_F32 ? 4 : 2), rows = (size_t)T * n * 2 * states * (dt == DGNN_F32 ? 4 : 2);
    const size_t state = (size_t)n * f * states * sizeof(float), kept = (size_t)((T + kHeld - 1) / kHeld) * state;
    const size_t vector = sizeof(float) * f;
    const std::pair<const void *, size_t> in[] = {{x, frame}, {delta, frame}, {bc, rows}, {z, frame}, {checkpoints, kept}, {g_y, frame}, {dh_after, state},
                                                  {a, vector * states}, {d, vector}, {dt_bias, vector}, {lengths, sizeof(int32_t) * n}};
    const std::pair<const void *, size_t> out[] = {{dx, frame}, {ddelta, frame}, {dbc, rows}, {dz, frame}, {dh_before, state}, {ws, ws_bytes},
                                                   {da, vector * states}, {dd, vector}, {ddt_bias, vector}};
    for (size_t i = 0; i < sizeof(out) / sizeof(*out); ++i) {
        for (auto o : in)
            if (overlap(out[i].first, out[i].second, o.first, o.second)) return DGNN_ERR_ALIAS;
        for (size_t k = 0; k < i; ++k)
            if (overlap(out[i].first, out[i].second, out[k].first, out[k].second)) return DGNN_ERR_ALIAS;
    }
    const BackShape shape = back_shape(T, n, f, states);
    ScanBack b{};
    b.s = Scan{x, delta, bc, z, a, d, dt_bias, nullptr, nullptr, nullptr, const_cast<float *>(checkpoints), lengths, n, (int)T, f, shape.groups, 0, 0, nullptr, nullptr};
    place_pieces(b.s, shape.pieces, states, ws);
    b.g_y = g_y; b.dh_after = dh_after; b.dx = dx; b.ddelta = ddelta; b.dbc = dbc; b.dz = dz; b.dh_before = dh_before;
    b.blocks_of_groups = shape.blocks_of_groups;
    char *at = static_cast<char *>(ws) + piece_bytes(shape.pieces, n, f, states);
    b.sums = reinterpret_cast<double *>(at);
    at += round_up((size_t)shape.slots * f * (states + 2) * sizeof(double), 256);
    b.dbc_part = shape.blocks_of_groups > 1 ? reinterpret_cast<float *>(at) : nullptr;
    hipStream_t st = (hipStream_t)stream;
    if (b.s.pieces > 1) {
        const int rc = by_kind(dt, states, [&](auto bf16, auto per) {
            const auto kernel = scan_back_piece_kernel<decltype(bf16)::value, decltype(per)::value>;
            hipLaunchKernelGGL(kernel, walk_grid(kernel, b.s, b.s.pieces - 1), dim3(kWaves * kWave), 0, st, b);
        });
        if (rc) return rc;
        if (const int failed = join_pieces<-1>(b.s, dh_after, states, st)) return failed;
    }
    int rc = by_kind(dt, states, [&](auto bf16, auto per) {
        constexpr int S = decltype(per)::value;
        auto launch = [&](auto tile) {
            constexpr int K = decltype(tile)::value;
            const unsigned lds = shape.waves * (3u * K * 8 * S * sizeof(float) + (S + 2) * kWave * sizeof(double));
            const auto kernel = z ? scan_back_kernel<decltype(bf16)::value, S, true, K> : scan_back_kernel<decltype(bf16)::value, S, false, K>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(shape.slots * shape.blocks_of_groups)), dim3(shape.waves * kWave), lds, st, b);
        };
        if (short_back(T)) launch(std::integral_constant<int, kHeld>{});
        else launch(std::integral_constant<int, kBackTile<S>>{});
    });
    if (rc) return rc;
    const int width = f * (states + 2);
    hipLaunchKernelGGL(scan_sums_kernel, dim3((unsigned)((width + 15) / 16)), dim3(1024), 0, st, b.sums, (int)shape.slots, f * states, f, da, dd, ddt_bias,
                       accumulate);
    DGNN_RETURN_IF_LAUNCH_FAILED();
    if (b.dbc_part) {
        const int64_t count = T * n * 2 * states;
        const unsigned blocks = (unsigned)std::min<int64_t>((count + 255) / 256, 1 << 20);
        if (dt == DGNN_BF16) hipLaunchKernelGGL(scan_rows_kernel<true>, dim3(blocks), dim3(256), 0, st, b.dbc_part, shape.blocks_of_groups, count, dbc);
        else hipLaunchKernelGGL(scan_rows_kernel<false>, dim3(blocks), dim3(256), 0, st, b.dbc_part, shape.blocks_of_groups, count, dbc);
        DGNN_RETURN_IF_LAUNCH_FAILED();
    }
    return DGNN_OK;
}
