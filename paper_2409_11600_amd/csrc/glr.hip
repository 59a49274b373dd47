// Gated linear recurrence: for every sequence and channel
//   f = sigmoid(gi_f + b_f), c = gi_c + b_c, o = sigmoid(gi_o + b_o),  h_t = f h_{t-1} + (1 - f) c,  y_t = o h_t,
// all steps in one call in both directions, and one token for each of many sequences.  Backwards, with G_t the gradient of h_t:
//   G_t = dy_t o_t + f_{t+1} G_{t+1},  dc = G (1 - f),  d gi_f = G (h_{t-1} - c) f (1 - f),  d gi_o = dy h o (1 - o),  dh0 = f_1 G_1.
#include <math.h>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

// sigmoid(a) and 1 - sigmoid(a), both to the last places: near 1 the difference from it would keep none of the small one's.  The hardware's exponential (1 ulp) and
// its reciprocal with a Newton step: a product of hundreds of gates adds up a rounding that leans to one side (2000 steps of 256 channels, dh0 against 64 bits: 3.5e-7
// without the step, 2.0e-7 with it; no difference in time).
__device__ inline void sigmoid2(float a, float &s, float &rest)
{
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(a)), x = 1.f + e, y = __builtin_amdgcn_rcpf(x);
    const float big = fmaf(fmaf(-x, y, 1.f), y, y), small = e * big;
    s = a >= 0.f ? big : small;
    rest = a >= 0.f ? small : big;
}
__device__ inline float sigmoid(float a)
{
    float s, rest;
    sigmoid2(a, s, rest);
    return s;
}

// How the work is laid out.  A lane has one channel of one sequence, a wavefront 64 of them (a tile) and a stretch of 16 steps, whose values it keeps in registers:
// they are read once.  A stretch by itself takes a state h to A h + B; the wavefronts of a block take consecutive stretches, exchange (A, B) through LDS,
// and each then goes through its steps again from the state that enters them.  A block goes on like this to the end of its segment.  Where tiles are few
// and steps many, the steps are shared out to several segments; a launch before the main one finds (A, B) of each.
constexpr int kStretch = NSK_GLR_STRETCH;
constexpr int kMostWaves = 16;
struct Sizes {
    int T, N, H;
    int stretches;          // of the whole sequence
    int per;                // of a segment
    int segments;
    unsigned tiles;
    int together;           // neighbouring tiles on one XCD (place)
    int flat;               // tiles go on across sequences (1), or each sequence has tiles of its own (0)
    long long gi_t, gi_n, y_t, y_n;
};
// Blocks are handed to the eight XCDs in turn.  Where rows are not whole cache lines, neighbouring tiles share those at their ends and are given to the same XCD
// (T=777, N=33, bf16 200 channels, us forward / backward: 23 / 29, otherwise 25 / 33); where they are, it costs a little (T=4096, N=4, fp32 256 channels: 22.4 / 33.8
// and 21.0 / 30.1).
__device__ inline void place(const Sizes &z, unsigned &tile, unsigned &segment)
{
    const unsigned g = blockIdx.x, n = gridDim.x, x = g % 8, each = n / 8, more = n % 8;
    const unsigned at = z.together ? x * each + (x < more ? x : more) + g / 8 : g;
    segment = at / z.tiles;
    tile = at - segment * z.tiles;
}
// The channel of this lane.
struct Lane {
    long long q;            // n * H + c; that of the last channel in lanes beyond it
    bool there;
    int n, c;
    unsigned gi, y;         // bytes from (t, first sequence of the tile, 0) on; kNowhere in lanes without a channel
};
// Rows are reached through buffer descriptors: a base in scalar registers, moved on from step to step, and one offset a lane.  An access at kNowhere, or
// through a descriptor of no bytes (a step behind the end), reads zeros and writes nothing.  Offsets and gates stay below 2^30 bytes each (plan_of).
constexpr unsigned kNowhere = 0x80000000u;
template <typename T> __device__ inline Lane lane_of(const Sizes &z, unsigned tile, long long &gi0, long long &y0)
{
    Lane l;
    const int lane = threadIdx.x & 63;
    if (z.flat) {
        const long long all = (long long)z.N * z.H, q = (long long)tile * 64 + lane;
        l.there = q < all;
        l.q = l.there ? q : all - 1;
        l.n = (int)(l.q / z.H);
        l.c = (int)(l.q - (long long)l.n * z.H);
    } else {
        const unsigned tiles = (unsigned)(z.H + 63) / 64;
        l.n = (int)(tile / tiles);
        const int c = (int)(tile - (unsigned)l.n * tiles) * 64 + lane;
        l.there = c < z.H;
        l.c = l.there ? c : z.H - 1;
        l.q = (long long)l.n * z.H + l.c;
    }
    const int n0 = __builtin_amdgcn_readfirstlane(l.n);
    gi0 = n0 * z.gi_n;
    y0 = n0 * z.y_n;
    l.gi = l.there ? ((unsigned)((l.n - n0) * z.gi_n) + (unsigned)l.c) * (unsigned)sizeof(T) : kNowhere;
    l.y = l.there ? ((unsigned)((l.n - n0) * z.y_n) + (unsigned)l.c) * (unsigned)sizeof(T) : kNowhere;
    return l;
}
// The rows of a stretch, one after the other: at() is the present one's descriptor, of no bytes where there is no such step.
template <typename T> struct Rows {
    T *p;
    int left;       // steps from the present one to the end of the sequence
    __device__ __amdgpu_buffer_rsrc_t at() const { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, left > 0 ? (int)kNowhere : 0, 0x00020000); }
    // `steps` on.  (Opaque: the compiler would keep the addresses and ends of all steps, for which there are not enough scalar registers.)
    __device__ void move(long long by, int steps = 1)
    {
        p += by;
        left -= steps;
        asm("" : "+s"(p), "+s"(left));
    }
};
template <typename T> __device__ inline float load(__amdgpu_buffer_rsrc_t r, unsigned lane, unsigned at)
{
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, (unsigned)__builtin_amdgcn_raw_buffer_load_b16(r, lane, at, 0) << 16);
    else return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, lane, at, 0));
}
template <typename T> __device__ inline void store(float v, __amdgpu_buffer_rsrc_t r, unsigned lane, unsigned at)
{
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (T)v), r, lane, at, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), r, lane, at, 0);
}
__device__ inline int steps_of(const int *lengths, const Lane &l, int T)
{
    if (!lengths) return T;
    const int len = lengths[l.n];
    return len < 0 ? 0 : len > T ? T : len;
}
__device__ inline int wave_of_block() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ inline bool any(bool b) { return __builtin_amdgcn_ballot_w64(b) != 0; }
struct Bias {
    float f, c, o;
};
__device__ inline Bias bias_of(const float *bias, const Sizes &z, const Lane &l)
{
    if (!bias) return {0.f, 0.f, 0.f};
    return {bias[l.c], bias[z.H + (long long)l.c], bias[2LL * z.H + l.c]};
}

// Loads of a stretch: gates f and c into f and x, o if asked for, biases added.
template <typename T, bool WITH_O>
__device__ inline void load_gates(const T *gi, const Sizes &z, const Lane &l, const Bias &b, int t0, float (&f)[kStretch], float (&x)[kStretch], float (&o)[kStretch])
{
    const unsigned gate = (unsigned)z.H * (unsigned)sizeof(T);
    Rows<const T> in{gi, z.T - t0};
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        const __amdgpu_buffer_rsrc_t r = in.at();
        f[i] = load<T>(r, l.gi, 0);
        x[i] = load<T>(r, l.gi, gate);
        if (WITH_O) o[i] = load<T>(r, l.gi, 2 * gate);
        in.move(z.gi_t);
    }
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        f[i] += b.f;
        x[i] += b.c;
        if (WITH_O) o[i] += b.o;
    }
}
// Steps from `live` on leave the state: f = sigmoid(inf) = 1, (1 - f) c = 0.
__device__ inline void leave_state(int live, float (&f)[kStretch], float (&x)[kStretch])
{
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        f[i] = i < live ? f[i] : INFINITY;
        x[i] = i < live ? x[i] : 0.f;
    }
}
// Arguments into f, x = (1 - f) c and o.
template <bool WITH_O> __device__ inline void apply_gates(float (&f)[kStretch], float (&x)[kStretch], float (&o)[kStretch])
{
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        float s, keep;
        sigmoid2(f[i], s, keep);
        x[i] *= keep;
        f[i] = s;
        if (WITH_O) o[i] = sigmoid(o[i]);
    }
}
// Zeros into the steps of a stretch that a lane's sequence does not have, behind what went there before.
template <typename T> __device__ inline void store_zeros(T *p, long long by, int from, int to, unsigned lane, unsigned gate, int gates)
{
#pragma unroll 1
    for (int i = 0; i < to; ++i) {
        const unsigned at = i < from ? kNowhere : lane;
        const __amdgpu_buffer_rsrc_t r = Rows<T>{p + i * by, 1}.at();
        for (int g = 0; g < gates; ++g) store<T>(0.f, r, at, g * gate);
    }
}
// (A, B) of this lane's stretch: the step is h = f h + x.
__device__ inline void fold(const float (&f)[kStretch], const float (&x)[kStretch], float &A, float &B)
{
    A = f[0];
    B = x[0];
#pragma unroll
    for (int i = 1; i < kStretch; ++i) {
        A *= f[i];
        B = f[i] * B + x[i];
    }
}

// (A, B) of a segment into ab[segment][2][N * H].
template <typename T>
__global__ __launch_bounds__(1024) void glr_fwd_fold_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths, float *__restrict__ ab)
{
    __shared__ float part[kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    unsigned tile, segment;
    place(z, tile, segment);
    long long gi0, y0;
    const Lane l = lane_of<T>(z, tile, gi0, y0);
    const int len = steps_of(lengths, l, z.T);
    const Bias b = bias_of(bias, z, l);
    const int begin = segment * z.per;
    float A = 1.f, B = 0.f;
    // a wavefront takes a run of the segment's stretches, the runs are joined once
    const int each = (z.per + waves - 1) / waves, first = begin + wave * each, most = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    const int last = first + each < most ? first + each : most;
    for (int s = first; s < last; ++s) {
        const int t0 = s * kStretch;
        if (!any(t0 < len)) break;
        float f[kStretch], x[kStretch], p, q;
        load_gates<T, false>(gi + gi0 + t0 * z.gi_t, z, l, b, t0, f, x, f);
        if (any(t0 + kStretch > len)) leave_state(len - t0, f, x);
        apply_gates<false>(f, x, f);
        fold(f, x, p, q);
        A *= p;
        B = p * B + q;
    }
    part[wave][0][lane] = A;
    part[wave][1][lane] = B;
    __syncthreads();
    if (wave == 0 && l.there) {
        for (int w = 1; w < waves; ++w) {
            A *= part[w][0][lane];
            B = part[w][0][lane] * B + part[w][1][lane];
        }
        const long long all = (long long)z.N * z.H;
        ab[(2LL * segment) * all + l.q] = A;
        ab[(2LL * segment + 1) * all + l.q] = B;
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void glr_fwd_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                      const float *__restrict__ h0, const float *__restrict__ ab, T *__restrict__ y, float *__restrict__ h_last,
                                                      float *__restrict__ saved)
{
    __shared__ float part[2][kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    unsigned tile, segment;
    place(z, tile, segment);
    long long gi0, y0;
    const Lane l = lane_of<T>(z, tile, gi0, y0);
    const long long all = (long long)z.N * z.H;
    const int len = steps_of(lengths, l, z.T);
    const Bias b = bias_of(bias, z, l);
    const int begin = segment * z.per, end = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    float carry = h0 ? h0[l.q] : 0.f;
    for (int s = 0; s < (int)segment; ++s) carry = ab[2LL * s * all + l.q] * carry + ab[(2LL * s + 1) * all + l.q];
    for (int k = begin, turn = 0; k < end; k += waves, turn ^= 1) {
        const int s = k + wave, t0 = s * kStretch;
        float f[kStretch], x[kStretch], o[kStretch], A = 1.f, B = 0.f;
        const bool some = s < end && any(t0 < len), ends = any(t0 + kStretch > len);
        if (some) {
            load_gates<T, true>(gi + gi0 + t0 * z.gi_t, z, l, b, t0, f, x, o);
            if (ends) leave_state(len - t0, f, x);
            apply_gates<true>(f, x, o);
            fold(f, x, A, B);
        }
        part[turn][wave][0][lane] = A;
        part[turn][wave][1][lane] = B;
        // (a wavefront writes a buffer again only after the barrier of the next turn, which all pass behind their reads of this one)
        lds_barrier();
        float h = carry;
        for (int w = 0; w < waves; ++w) {
            if (w == wave) h = carry;
            carry = part[turn][w][0][lane] * carry + part[turn][w][1][lane];
        }
        if (s >= end) continue;
        if (saved && l.there) saved[s * all + l.q] = h;
        if (!y) continue;
        T *out = y + y0 + t0 * z.y_t;
        if (some) {
            Rows<T> rows{out, z.T - t0};
#pragma unroll
            for (int i = 0; i < kStretch; ++i) {
                h = f[i] * h + x[i];
                store<T>(o[i] * h, rows.at(), l.y, 0);
                rows.move(z.y_t);
            }
        }
        if (ends) store_zeros(out, z.y_t, len - t0, z.T - t0 < kStretch ? z.T - t0 : kStretch, l.y, 0, 1);
    }
    if (h_last && end == z.stretches && wave == 0 && l.there) h_last[l.q] = carry;
}

// Backwards a stretch takes E, the gradient of the state that leaves it, to A E + B.  What a step needs for that: f, u = dy o, and with the states, which
// come from the saved one, k = 1 - f and d = (h_{t-1} - c) f (1 - f).  The gradient of the gate o depends on nothing later.
template <typename T>
__global__ __launch_bounds__(1024) void glr_bwd_fold_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                           const T *__restrict__ dy, float *__restrict__ ab)
{
    __shared__ float part[kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    unsigned tile, segment;
    place(z, tile, segment);
    long long gi0, y0;
    const Lane l = lane_of<T>(z, tile, gi0, y0);
    const int len = steps_of(lengths, l, z.T);
    const Bias b = bias_of(bias, z, l);
    const unsigned gate = (unsigned)z.H * (unsigned)sizeof(T);
    const int begin = ++segment * z.per;       // (nothing comes before the first)
    float A = 1.f, B = 0.f;
    const int each = (z.per + waves - 1) / waves, first = begin + wave * each, most = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    const int last = first + each < most ? first + each : most;
    for (int s = last - 1; s >= first; --s) {
        const int t0 = s * kStretch;
        if (!any(t0 < len)) continue;
        float f[kStretch], o[kStretch], up[kStretch];
        Rows<const T> in{gi + gi0 + t0 * z.gi_t, z.T - t0}, above{dy + y0 + t0 * z.y_t, dy ? z.T - t0 : 0};
#pragma unroll
        for (int i = 0; i < kStretch; ++i) {
            const __amdgpu_buffer_rsrc_t r = in.at();
            f[i] = load<T>(r, l.gi, 0);
            o[i] = load<T>(r, l.gi, 2 * gate);
            up[i] = load<T>(above.at(), l.y, 0);
            in.move(z.gi_t);
            above.move(z.y_t);
        }
#pragma unroll
        for (int i = kStretch - 1; i >= 0; --i) {
            const bool live = t0 + i < len;
            const float g = live ? sigmoid(f[i] + b.f) : 1.f, u = live ? up[i] * sigmoid(o[i] + b.o) : 0.f;
            B = g * (B + u);
            A *= g;
        }
    }
    part[wave][0][lane] = A;
    part[wave][1][lane] = B;
    __syncthreads();
    if (wave == 0 && l.there) {
        A = 1.f;
        B = 0.f;
        for (int w = waves - 1; w >= 0; --w) {
            A *= part[w][0][lane];
            B = part[w][0][lane] * B + part[w][1][lane];
        }
        const long long all = (long long)z.N * z.H;
        ab[(2LL * segment) * all + l.q] = A;
        ab[(2LL * segment + 1) * all + l.q] = B;
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void glr_bwd_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                      const float *__restrict__ saved, const T *__restrict__ dy, const float *__restrict__ dh_last,
                                                      const float *__restrict__ ab, T *__restrict__ dgi, float *__restrict__ dh0)
{
    __shared__ float part[2][kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    unsigned tile, segment;
    place(z, tile, segment);
    long long gi0, y0;
    const Lane l = lane_of<T>(z, tile, gi0, y0);
    const long long all = (long long)z.N * z.H;
    const int len = steps_of(lengths, l, z.T);
    const Bias b = bias_of(bias, z, l);
    const unsigned gate = (unsigned)z.H * (unsigned)sizeof(T);
    const int begin = segment * z.per, end = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    float carry = dh_last ? dh_last[l.q] : 0.f;
    for (int s = z.segments - 1; s > (int)segment; --s) carry = ab[2LL * s * all + l.q] * carry + ab[(2LL * s + 1) * all + l.q];
    for (int k = end, turn = 0; k > begin; k -= waves, turn ^= 1) {
        const int s = k - 1 - wave, t0 = s * kStretch;       // wavefront 0 has the last stretch
        const bool mine = s >= begin, some = mine && any(t0 < len), ends = any(t0 + kStretch > len);
        float f[kStretch], keep[kStretch], u[kStretch], d[kStretch], A = 1.f, B = 0.f;
        const long long at = gi0 + t0 * z.gi_t;
        if (some) {
            // (arguments of f and o, c and dy are in f, keep, d and u until their step)
            float h = saved[s * all + l.q];
            Rows<const T> in{gi + at, z.T - t0}, above{dy + y0 + t0 * z.y_t, dy ? z.T - t0 : 0};
#pragma unroll
            for (int i = 0; i < kStretch; ++i) {
                const __amdgpu_buffer_rsrc_t r = in.at();
                f[i] = load<T>(r, l.gi, 0);
                d[i] = load<T>(r, l.gi, gate);
                keep[i] = load<T>(r, l.gi, 2 * gate);
                u[i] = load<T>(above.at(), l.y, 0);
                in.move(z.gi_t);
                above.move(z.y_t);
            }
#pragma unroll
            for (int i = 0; i < kStretch; ++i) {
                f[i] += b.f;
                d[i] += b.c;
                keep[i] += b.o;
            }
            if (ends) {
                leave_state(len - t0, f, d);
#pragma unroll
                for (int i = 0; i < kStretch; ++i) {
                    keep[i] = t0 + i < len ? keep[i] : 0.f;
                    u[i] = t0 + i < len ? u[i] : 0.f;
                }
            }
            Rows<T> out{dgi + at, z.T - t0};
#pragma unroll
            for (int i = 0; i < kStretch; ++i) {
                const float c = d[i];
                float o, shut, s, rest;
                sigmoid2(keep[i], o, shut);
                sigmoid2(f[i], s, rest);
                f[i] = s;
                keep[i] = rest;
                d[i] = (h - c) * (s * rest);
                h = s * h + rest * c;
                u[i] *= o;
                store<T>(u[i] * shut * h, out.at(), l.gi, 2 * gate);
                out.move(z.gi_t);
            }
#pragma unroll
            for (int i = kStretch - 1; i >= 0; --i) {
                A *= f[i];
                B = f[i] * (B + u[i]);
            }
        }
        part[turn][wave][0][lane] = A;
        part[turn][wave][1][lane] = B;
        lds_barrier();
        float E = carry;
        for (int w = 0; w < waves; ++w) {
            if (w == wave) E = carry;
            carry = part[turn][w][0][lane] * carry + part[turn][w][1][lane];
        }
        if (!mine) continue;
        if (some) {
            Rows<T> out{dgi + at + (kStretch - 1) * z.gi_t, z.T - t0 - (kStretch - 1)};
#pragma unroll
            for (int i = kStretch - 1; i >= 0; --i) {
                const __amdgpu_buffer_rsrc_t r = out.at();
                const float G = E + u[i];
                store<T>(G * d[i], r, l.gi, 0);
                store<T>(G * keep[i], r, l.gi, gate);
                E = f[i] * G;
                out.move(-z.gi_t, -1);
            }
        }
        if (ends) store_zeros(dgi + at, z.gi_t, len - t0, z.T - t0 < kStretch ? z.T - t0 : kStretch, l.gi, gate, 3);
    }
    if (dh0 && begin == 0 && wave == 0 && l.there) dh0[l.q] = carry;
}

template <typename T>
__global__ __launch_bounds__(64) void glr_step_kernel(int H, int S, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ slots,
                                                      float *__restrict__ state, T *__restrict__ y, unsigned tiles)
{
    const unsigned n = blockIdx.x / tiles;
    const int c = (int)(blockIdx.x - n * tiles) * 64 + threadIdx.x;
    if (c >= H) return;
    const int slot = slots ? slots[n] : (int)n;
    float out = 0.f;
    if (slot >= 0 && slot < S) {
        const T *g = gi + (size_t)n * 3 * H + c;
        float f, keep;
        sigmoid2((float)g[0] + (bias ? bias[c] : 0.f), f, keep);
        float *h = state + (size_t)slot * H + c;
        const float hn = f * *h + keep * ((float)g[H] + (bias ? bias[H + c] : 0.f));
        *h = hn;
        out = sigmoid((float)g[2 * (size_t)H] + (bias ? bias[2 * (size_t)H + c] : 0.f)) * hn;
    }
    if (y) y[(size_t)n * H + c] = (T)out;
}

// Rows of `width` elements at t * st + n * sn that do not overlap, and do not lie between each other's; both strides 0: [T,N,width].
bool rows_apart(int T, int N, long long width, long long &st, long long &sn)
{
    if (st == 0 && sn == 0) {
        sn = width;
        st = width * N;
    }
    const long long most = 1LL << 60;
    if ((T > 1 && (st < width || st > most / T)) || (N > 1 && (sn < width || sn > most / N))) return false;
    return T == 1 || N == 1 || st >= sn * (N - 1) + width || sn >= st * (T - 1) + width;
}
// Checks a descriptor and fills in the strides that are left open.
int check(const nsk_glr_desc_t *desc, nsk_glr_desc_t &d)
{
    if (!desc) return NSK_ERR_NULL;
    d = *desc;
    if (d.T <= 0 || d.N <= 0 || d.H <= 0 || d.H > (1 << 26) || (d.dtype != NSK_F32 && d.dtype != NSK_BF16)) return NSK_ERR_BAD_DESC;
    if ((long long)d.N * d.H > (1LL << 60) / d.T) return NSK_ERR_BAD_DESC;
    if (!rows_apart(d.T, d.N, 3LL * d.H, d.gi_t, d.gi_n) || !rows_apart(d.T, d.N, d.H, d.y_t, d.y_n)) return NSK_ERR_BAD_DESC;
    if ((long long)d.N * ((d.H + 63) / 64) > 0x7fffffff) return NSK_ERR_UNSUPPORTED;
    return NSK_OK;
}

// Tiles, wavefronts of a block and segments of a call.
struct Plan {
    Sizes z;
    int waves;
};
Plan plan_of(const nsk_glr_desc_t &d)
{
    Plan p{};
    const long long es = d.dtype == NSK_BF16 ? 2 : 4;
    p.z = {d.T, d.N, d.H, ceil_div(d.T, kStretch), 0, 1, 0, 0, 0, d.gi_t, d.gi_n, d.y_t, d.y_n};
    p.z.together = d.H * es % 128 != 0 || (d.gi_t | d.gi_n) * es % 128 != 0;
    // a tile reaches over 63 / H + 1 further sequences, whose offsets have to fit 30 bits (those of a single sequence do)
    const long long over = d.H < 64 ? 63 / d.H + 1 : 1, stride = d.gi_n > d.y_n ? d.gi_n : d.y_n;
    p.z.flat = stride < (1LL << 30) && (over * stride + d.H) * es < (1LL << 30);
    const long long tiles = p.z.flat ? ((long long)d.N * d.H + 63) / 64 : (long long)d.N * ((d.H + 63) / 64);
    p.z.tiles = (unsigned)tiles;
    // One round of 16 wavefronts takes a compute unit about 5 us, 0.31 a stretch.  With a block for every unit or more, blocks go through all steps of their tile;
    // with fewer, the launch before the main one costs about 6 us and 0.6 of the main one's work, but all units share the work: 6 + 1.6 * 0.31 / 256 * tiles * stretches
    // against 0.31 * stretches.  (us forward / backward, whole / shared out: T=65536, N=1, bf16 512 channels 1514 / 2126 and 92 / 147; T=4096, N=4, fp32 256 channels
    // 80 / 119 and 21 / 30; T=200, N=50, fp32 256 channels 9.2 / 14.6 and 12.6 / 18.8.)
    const bool share = tiles < 160 && (long long)p.z.stretches * (160 - tiles) > 3072;
    // Wavefronts: as many as there are stretches for a block that has a unit to itself (T=200, N=50, fp32 256 channels, 13 / 8 of them: 9.2 and 10.2 us forward); fewer
    // where several blocks share a unit, whose barriers then come at different times (T=200, N=512, bf16 768 channels, 4 / 8 / 13 of them: 77, 77, 100 us forward, 129, 133,
    // 150 backward; T=2048, N=32, bf16 768 channels, 4 / 8 / 16: 122, 111, 117 and 194, 187, 183).
    const int most = share ? 8 : tiles <= 256 ? kMostWaves : tiles < 1024 ? 8 : 4;
    p.waves = p.z.stretches < most ? p.z.stretches : most;
    const int rounds = ceil_div(p.z.stretches, p.waves);
    long long want = share ? (512 + tiles - 1) / tiles : 1;
    if (want > rounds) want = rounds;
    // (two blocks a compute unit, what the backward pass has room for: more come in a second turn)
    p.z.per = ceil_div(rounds, (int)want) * p.waves;
    p.z.segments = ceil_div(p.z.stretches, p.z.per);
    return p;
}
size_t workspace_of(const Plan &p) { return p.z.segments > 1 ? (size_t)p.z.segments * 2 * p.z.N * p.z.H * sizeof(float) : 0; }

}  // namespace
}  // namespace nsk

using namespace nsk;

extern "C" {

size_t nsk_glr_saved_bytes(const nsk_glr_desc_t *desc)
{
    nsk_glr_desc_t d;
    return check(desc, d) == NSK_OK ? (size_t)ceil_div(d.T, kStretch) * d.N * d.H * sizeof(float) : 0;
}

size_t nsk_glr_workspace_bytes(const nsk_glr_desc_t *desc, int pass)
{
    nsk_glr_desc_t d;
    return (pass == NSK_PASS_FWD || pass == NSK_PASS_DGRAD) && check(desc, d) == NSK_OK ? workspace_of(plan_of(d)) : 0;
}

int nsk_glr_fwd(const nsk_glr_desc_t *desc, const void *gi, const float *bias, const int *lengths, const float *h0, void *y, float *h_last, float *saved,
                void *workspace, size_t workspace_bytes, void *stream)
{
    nsk_glr_desc_t d;
    const int status = check(desc, d);
    if (status != NSK_OK) return status;
    if (!gi || (!y && !h_last)) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(lengths) || unaligned16(h0) || unaligned16(y) || unaligned16(h_last) || unaligned16(saved) || unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    const Plan p = plan_of(d);
    if (p.z.segments > 1 && (!workspace || workspace_bytes < workspace_of(p))) return NSK_ERR_WORKSPACE;
    const dim3 grid(p.z.tiles * (unsigned)p.z.segments), block((unsigned)p.waves * 64);
    hipStream_t st = (hipStream_t)stream;
    float *ab = (float *)workspace;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (p.z.segments > 1) hipLaunchKernelGGL(glr_fwd_fold_kernel<T>, dim3(p.z.tiles * (unsigned)(p.z.segments - 1)), block, 0, st, p.z, (const T *)gi, bias, lengths, ab);
        hipLaunchKernelGGL(glr_fwd_kernel<T>, grid, block, 0, st, p.z, (const T *)gi, bias, lengths, h0, ab, (T *)y, h_last, saved);
    };
    if (d.dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    return check_launch();
}

int nsk_glr_bwd(const nsk_glr_desc_t *desc, const void *gi, const float *bias, const int *lengths, const float *saved, const void *dy, const float *dh_last,
                void *dgi, float *dh0, void *workspace, size_t workspace_bytes, void *stream)
{
    nsk_glr_desc_t d;
    const int status = check(desc, d);
    if (status != NSK_OK) return status;
    if (!gi || !saved || (!dy && !dh_last) || !dgi) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(lengths) || unaligned16(saved) || unaligned16(dy) || unaligned16(dh_last) || unaligned16(dgi) || unaligned16(dh0) || unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    const Plan p = plan_of(d);
    if (p.z.segments > 1 && (!workspace || workspace_bytes < workspace_of(p))) return NSK_ERR_WORKSPACE;
    const dim3 grid(p.z.tiles * (unsigned)p.z.segments), block((unsigned)p.waves * 64);
    hipStream_t st = (hipStream_t)stream;
    float *ab = (float *)workspace;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (p.z.segments > 1) hipLaunchKernelGGL(glr_bwd_fold_kernel<T>, dim3(p.z.tiles * (unsigned)(p.z.segments - 1)), block, 0, st, p.z, (const T *)gi, bias, lengths, (const T *)dy, ab);
        hipLaunchKernelGGL(glr_bwd_kernel<T>, grid, block, 0, st, p.z, (const T *)gi, bias, lengths, saved, (const T *)dy, dh_last, ab, (T *)dgi, dh0);
    };
    if (d.dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    return check_launch();
}

int nsk_glr_step(int dtype, int N, int H, int S, const void *gi, const float *bias, const int *slots, float *state, void *y, void *stream)
{
    if (N <= 0 || H <= 0 || H > (1 << 28) || S <= 0 || (dtype != NSK_F32 && dtype != NSK_BF16)) return NSK_ERR_BAD_DESC;
    if (!gi || !state) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(slots) || unaligned16(state) || unaligned16(y)) return NSK_ERR_ALIGNMENT;
    const unsigned tiles = (unsigned)ceil_div(H, 64);
    if ((long long)tiles * N > 0x7fffffff) return NSK_ERR_UNSUPPORTED;
    const dim3 grid(tiles * (unsigned)N);
    if (dtype == NSK_BF16)
        hipLaunchKernelGGL(glr_step_kernel<bf16_t>, grid, dim3(64), 0, (hipStream_t)stream, H, S, (const bf16_t *)gi, bias, slots, state, (bf16_t *)y, tiles);
    else
        hipLaunchKernelGGL(glr_step_kernel<float>, grid, dim3(64), 0, (hipStream_t)stream, H, S, (const float *)gi, bias, slots, state, (float *)y, tiles);
    return check_launch();
}

}  // extern "C"
