// Gated linear recurrence: for every sequence and channel
//   f = sigmoid(gi_f + b_f), c = gi_c + b_c, o = sigmoid(gi_o + b_o),  h_t = f h_{t-1} + (1 - f) c,  y_t = o h_t,
// all steps in one call in both directions, and one token for each of many sequences.  Backwards, with G_t the gradient of h_t:
//   G_t = dy_t o_t + f_{t+1} G_{t+1},  dc = G (1 - f),  d gi_f = G (h_{t-1} - c) f (1 - f),  d gi_o = dy h o (1 - o),  dh0 = f_1 G_1.
#include <math.h>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

// sigmoid(a) and 1 - sigmoid(a), both to the last places: near 1 the difference from it would keep none of the small one's.  The hardware's exponential and
// reciprocal: 1 ulp each, and the argument's rounding, |a| of 2^-24.
constexpr float kLog2e = 1.44269504f;
__device__ inline float sigmoid(float a) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * a)); }
__device__ inline void sigmoid2(float a, float &s, float &rest)
{
    const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(a)), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
    s = a >= 0.f ? big : small;
    rest = a >= 0.f ? small : big;
}

// How the work is laid out.  A lane has one channel of one sequence, a wavefront 64 of them (a tile) and a stretch of 16 steps, whose values it keeps in registers:
// they are read once.  A stretch by itself takes a state h to A h + B; the wavefronts of a block take consecutive stretches, exchange (A, B) through LDS,
// and each then goes through its steps again from the state that enters them.  A block goes on like this to the end of its segment.  Where tiles are few
// and steps many, the steps are shared out to several segments; a launch before the main one finds (A, B) of each.
constexpr int kStretch = NSK_GLR_STRETCH;
constexpr int kMostWaves = 8;
struct Sizes {
    int T, N, H;
    int stretches;          // of the whole sequence
    int per;                // of a segment
    int flat;               // tiles go on across sequences (1), or each sequence has tiles of its own (0)
    long long gi_t, gi_n, y_t, y_n;
};
// The channel of this lane.  Offsets within a tile fit 32 bits, so that an address is a base in scalar registers and one offset a lane.
struct Lane {
    long long q;            // n * H + c; that of the last channel in lanes beyond it
    bool there;
    int n0;                 // first sequence of the tile
    int n, c;
    unsigned gi, y;         // elements from (t, n0, 0) on
};
__device__ inline Lane lane_of(const Sizes &z, unsigned tile)
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
    l.n0 = __builtin_amdgcn_readfirstlane(l.n);
    l.gi = (unsigned)((l.n - l.n0) * z.gi_n) + (unsigned)l.c;
    l.y = (unsigned)((l.n - l.n0) * z.y_n) + (unsigned)l.c;
    return l;
}
template <typename T> __device__ inline T &element(T *base, unsigned i)
{
    return *(T *)((char *)base + i * (unsigned)sizeof(T));
}
template <typename T> __device__ inline const T &element(const T *base, unsigned i)
{
    return *(const T *)((const char *)base + i * (unsigned)sizeof(T));
}
__device__ inline int steps_of(const int *lengths, const Lane &l, int T)
{
    if (!lengths) return T;
    const int len = lengths[l.n];
    return len < 0 ? 0 : len > T ? T : len;
}
__device__ inline int wave_of_block() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// The values that step i of a stretch reads, the last step's again behind the end of the sequence.
template <typename T, int GATE>
__device__ inline void load_gate(const T *__restrict__ gi, const Sizes &z, const Lane &l, int t0, T (&v)[kStretch])
{
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        const int t = t0 + i < z.T ? t0 + i : z.T - 1;
        v[i] = element(gi + (long long)t * z.gi_t + (long long)l.n0 * z.gi_n + (long long)GATE * z.H, l.gi);
    }
}

// (A, B) of this lane's stretch: f, x in, the step being h = f h + x.
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

// f, x = (1 - f) c and o of a stretch; steps that are not there leave the state.
template <typename T, bool WITH_O>
__device__ inline void gates_of(const T *__restrict__ gi, const float *__restrict__ bias, const Sizes &z, const Lane &l, int t0, int len, float (&f)[kStretch], float (&x)[kStretch],
                                float (&o)[kStretch])
{
    T rf[kStretch], rc[kStretch], ro[kStretch];
    load_gate<T, 0>(gi, z, l, t0, rf);
    load_gate<T, 1>(gi, z, l, t0, rc);
    if (WITH_O) load_gate<T, 2>(gi, z, l, t0, ro);
    const float bf = bias ? bias[l.c] : 0.f, bc = bias ? bias[z.H + l.c] : 0.f, bo = WITH_O && bias ? bias[2 * (long long)z.H + l.c] : 0.f;
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        float keep;
        sigmoid2((float)rf[i] + bf, f[i], keep);
        x[i] = keep * ((float)rc[i] + bc);
        if (WITH_O) o[i] = sigmoid((float)ro[i] + bo);
    }
    if (__builtin_amdgcn_ballot_w64(t0 + kStretch > len)) {
#pragma unroll
        for (int i = 0; i < kStretch; ++i) {
            const bool live = t0 + i < len;
            f[i] = live ? f[i] : 1.f;
            x[i] = live ? x[i] : 0.f;
            if (WITH_O) o[i] = live ? o[i] : 0.f;
        }
    }
}

// (A, B) of a segment into ab[segment][2][N * H].
template <typename T>
__global__ __launch_bounds__(512) void glr_fwd_fold_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths, float *__restrict__ ab)
{
    __shared__ float part[kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    const Lane l = lane_of(z, blockIdx.x);
    const int len = steps_of(lengths, l, z.T);
    const int begin = blockIdx.y * z.per;
    float A = 1.f, B = 0.f;
    // a wavefront takes a run of the segment's stretches, the runs are joined once
    const int each = (z.per + waves - 1) / waves, first = begin + wave * each, most = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    const int last = first + each < most ? first + each : most;
    for (int s = first; s < last; ++s) {
        if (!__builtin_amdgcn_ballot_w64(s * kStretch < len)) break;
        float f[kStretch], x[kStretch], a, b;
        gates_of<T, false>(gi, bias, z, l, s * kStretch, len, f, x, f);
        fold(f, x, a, b);
        A *= a;
        B = a * B + b;
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
        ab[(2LL * blockIdx.y) * all + l.q] = A;
        ab[(2LL * blockIdx.y + 1) * all + l.q] = B;
    }
}

template <typename T>
__global__ __launch_bounds__(512) void glr_fwd_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                       const float *__restrict__ h0, const float *__restrict__ ab, T *__restrict__ y, float *__restrict__ h_last,
                                                       float *__restrict__ saved)
{
    __shared__ float part[2][kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    const Lane l = lane_of(z, blockIdx.x);
    const long long all = (long long)z.N * z.H;
    const int len = steps_of(lengths, l, z.T);
    const int begin = blockIdx.y * z.per, end = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    float carry = h0 ? h0[l.q] : 0.f;
    for (int s = 0; s < (int)blockIdx.y; ++s) carry = ab[2LL * s * all + l.q] * carry + ab[(2LL * s + 1) * all + l.q];
    for (int k = begin, turn = 0; k < end; k += waves, turn ^= 1) {
        const int s = k + wave, t0 = s * kStretch;
        float f[kStretch], x[kStretch], o[kStretch];
        const bool any = s < end && __builtin_amdgcn_ballot_w64(t0 < len);
        if (any) {
            float A, B;
            gates_of<T, true>(gi, bias, z, l, t0, len, f, x, o);
            fold(f, x, A, B);
            part[turn][wave][0][lane] = A;
            part[turn][wave][1][lane] = B;
        } else {
            part[turn][wave][0][lane] = 1.f;
            part[turn][wave][1][lane] = 0.f;
        }
        // (a wavefront writes a buffer again only after the barrier of the next turn, which all pass behind their reads of this one)
        lds_barrier();
        float h = carry;
        for (int w = 0; w < waves; ++w) {
            if (w == wave) h = carry;
            carry = part[turn][w][0][lane] * carry + part[turn][w][1][lane];
        }
        if (s >= end) continue;
        if (saved && l.there) saved[s * all + l.q] = h;
        if (!any) {
            if (y && l.there)
                for (int i = 0; i < kStretch && t0 + i < z.T; ++i) element(y + (long long)(t0 + i) * z.y_t + (long long)l.n0 * z.y_n, l.y) = (T)0.f;
            continue;
        }
        if (y && l.there) {
#pragma unroll
            for (int i = 0; i < kStretch; ++i) {
                h = f[i] * h + x[i];
                if (t0 + i < z.T) element(y + (long long)(t0 + i) * z.y_t + (long long)l.n0 * z.y_n, l.y) = (T)(o[i] * h);
            }
        }
    }
    if (h_last && end == z.stretches && wave == 0 && l.there) h_last[l.q] = carry;
}

// Backwards a stretch takes E, the gradient of the state that leaves it, to A E + B.  What a step needs for that: f, u = dy o, and with the states, which
// come from the saved one, k = 1 - f and d = (h_{t-1} - c) f (1 - f).  The gradient of the gate o depends on nothing later.
template <typename T>
__global__ __launch_bounds__(512) void glr_bwd_fold_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                            const T *__restrict__ dy, float *__restrict__ ab)
{
    __shared__ float part[kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    const Lane l = lane_of(z, blockIdx.x);
    const int len = steps_of(lengths, l, z.T);
    const float bf = bias ? bias[l.c] : 0.f, bo = bias ? bias[2 * (long long)z.H + l.c] : 0.f;
    const int segment = blockIdx.y + 1, begin = segment * z.per;       // (nothing comes after the first)
    float A = 1.f, B = 0.f;
    const int each = (z.per + waves - 1) / waves, first = begin + wave * each, most = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    const int last = first + each < most ? first + each : most;
    for (int s = last - 1; s >= first; --s) {
        const int t0 = s * kStretch;
        if (!__builtin_amdgcn_ballot_w64(t0 < len)) continue;
        T rf[kStretch], ro[kStretch], rd[kStretch];
        load_gate<T, 0>(gi, z, l, t0, rf);
        if (dy) {
            load_gate<T, 2>(gi, z, l, t0, ro);
#pragma unroll
            for (int i = 0; i < kStretch; ++i) {
                const int t = t0 + i < z.T ? t0 + i : z.T - 1;
                rd[i] = element(dy + (long long)t * z.y_t + (long long)l.n0 * z.y_n, l.y);
            }
        }
#pragma unroll
        for (int i = kStretch - 1; i >= 0; --i) {
            const bool live = t0 + i < len;
            const float f = live ? sigmoid((float)rf[i] + bf) : 1.f;
            const float u = live && dy ? (float)rd[i] * sigmoid((float)ro[i] + bo) : 0.f;
            B = f * (B + u);
            A *= f;
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
__global__ __launch_bounds__(512) void glr_bwd_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                       const float *__restrict__ saved, const T *__restrict__ dy, const float *__restrict__ dh_last,
                                                       const float *__restrict__ ab, T *__restrict__ dgi, float *__restrict__ dh0)
{
    __shared__ float part[2][kMostWaves][2][64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    const Lane l = lane_of(z, blockIdx.x);
    const long long all = (long long)z.N * z.H;
    const int len = steps_of(lengths, l, z.T);
    const float bf = bias ? bias[l.c] : 0.f, bc = bias ? bias[z.H + l.c] : 0.f, bo = bias ? bias[2 * (long long)z.H + l.c] : 0.f;
    const int begin = blockIdx.y * z.per, end = begin + z.per < z.stretches ? begin + z.per : z.stretches;
    float carry = dh_last ? dh_last[l.q] : 0.f;
    for (int s = (int)gridDim.y - 1; s > (int)blockIdx.y; --s) carry = ab[2LL * s * all + l.q] * carry + ab[(2LL * s + 1) * all + l.q];
    for (int k = end, turn = 0; k > begin; k -= waves, turn ^= 1) {
        const int s = k - 1 - wave, t0 = s * kStretch;       // wavefront 0 has the last stretch
        const bool mine = s >= begin, any = mine && __builtin_amdgcn_ballot_w64(t0 < len);
        float f[kStretch], keep[kStretch], u[kStretch], d[kStretch];
        T *const out = dgi + (long long)t0 * z.gi_t + (long long)l.n0 * z.gi_n;
        if (any) {
            T rf[kStretch], rc[kStretch], ro[kStretch], rd[kStretch];
            float h = saved[s * all + l.q];
            load_gate<T, 0>(gi, z, l, t0, rf);
            load_gate<T, 1>(gi, z, l, t0, rc);
            if (dy) {
                load_gate<T, 2>(gi, z, l, t0, ro);
#pragma unroll
                for (int i = 0; i < kStretch; ++i) {
                    const int t = t0 + i < z.T ? t0 + i : z.T - 1;
                    rd[i] = element(dy + (long long)t * z.y_t + (long long)l.n0 * z.y_n, l.y);
                }
            }
            const bool ends = __builtin_amdgcn_ballot_w64(t0 + kStretch > len);
            float A = 1.f, B = 0.f;
#pragma unroll
            for (int i = 0; i < kStretch; ++i) {
                const bool live = !ends || t0 + i < len;
                const float c = (float)rc[i] + bc;
                sigmoid2((float)rf[i] + bf, f[i], keep[i]);
                d[i] = (h - c) * f[i] * keep[i];
                h = f[i] * h + keep[i] * c;
                float douto = 0.f;
                u[i] = 0.f;
                if (dy) {
                    float o, rest;
                    sigmoid2((float)ro[i] + bo, o, rest);
                    u[i] = (float)rd[i] * o;
                    douto = u[i] * rest * h;
                }
                if (!live) {
                    f[i] = 1.f;
                    keep[i] = d[i] = u[i] = douto = 0.f;
                }
                if (l.there && t0 + i < z.T) element(out + i * z.gi_t + 2LL * z.H, l.gi) = (T)douto;
            }
#pragma unroll
            for (int i = kStretch - 1; i >= 0; --i) {
                A *= f[i];
                B = f[i] * (B + u[i]);
            }
            part[turn][wave][0][lane] = A;
            part[turn][wave][1][lane] = B;
        } else {
            part[turn][wave][0][lane] = 1.f;
            part[turn][wave][1][lane] = 0.f;
        }
        lds_barrier();
        float E = carry;
        for (int w = 0; w < waves; ++w) {
            if (w == wave) E = carry;
            carry = part[turn][w][0][lane] * carry + part[turn][w][1][lane];
        }
        if (!mine || !l.there) continue;
        if (!any) {
            for (int i = 0; i < kStretch && t0 + i < z.T; ++i) {
                element(out + i * z.gi_t, l.gi) = (T)0.f;
                element(out + i * z.gi_t + z.H, l.gi) = (T)0.f;
                element(out + i * z.gi_t + 2LL * z.H, l.gi) = (T)0.f;
            }
            continue;
        }
#pragma unroll
        for (int i = kStretch - 1; i >= 0; --i) {
            const float G = E + u[i];
            if (t0 + i < z.T) {
                element(out + i * z.gi_t, l.gi) = (T)(G * d[i]);
                element(out + i * z.gi_t + z.H, l.gi) = (T)(G * keep[i]);
            }
            E = f[i] * G;
        }
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
    if (d.T <= 0 || d.N <= 0 || d.H <= 0 || d.H > (1 << 28) || (d.dtype != NSK_F32 && d.dtype != NSK_BF16)) return NSK_ERR_BAD_DESC;
    if ((long long)d.N * d.H > (1LL << 60) / d.T) return NSK_ERR_BAD_DESC;
    if (!rows_apart(d.T, d.N, 3LL * d.H, d.gi_t, d.gi_n) || !rows_apart(d.T, d.N, d.H, d.y_t, d.y_n)) return NSK_ERR_BAD_DESC;
    if ((long long)d.N * ((d.H + 63) / 64) > 0x7fffffff) return NSK_ERR_UNSUPPORTED;
    return NSK_OK;
}

// Tiles, wavefronts of a block and segments of a call.
struct Plan {
    Sizes z;
    unsigned tiles;
    int waves, segments;
};
Plan plan_of(const nsk_glr_desc_t &d)
{
    Plan p{};
    const long long es = d.dtype == NSK_BF16 ? 2 : 4;
    p.z = {d.T, d.N, d.H, ceil_div(d.T, kStretch), 0, 0, d.gi_t, d.gi_n, d.y_t, d.y_n};
    // a tile reaches over 63 / H + 1 further sequences, whose offsets have to fit
    const long long over = d.H < 64 ? 63 / d.H + 1 : 1, stride = d.gi_n > d.y_n ? d.gi_n : d.y_n;
    p.z.flat = stride < (1LL << 40) && (over * stride + 3LL * d.H) * es < (1LL << 31);
    const long long tiles = p.z.flat ? ((long long)d.N * d.H + 63) / 64 : (long long)d.N * ((d.H + 63) / 64);
    p.tiles = (unsigned)tiles;
    p.waves = p.z.stretches < kMostWaves ? p.z.stretches : kMostWaves;
    const int rounds = ceil_div(p.z.stretches, p.waves);
    long long want = 512 / (tiles > 0 ? tiles : 1);
    if (want > rounds / 2) want = rounds / 2;
    if (want < 1) want = 1;
    p.z.per = ceil_div(rounds, (int)want) * p.waves;
    p.segments = ceil_div(p.z.stretches, p.z.per);
    return p;
}
size_t workspace_of(const Plan &p) { return p.segments > 1 ? (size_t)p.segments * 2 * p.z.N * p.z.H * sizeof(float) : 0; }

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
    if (p.segments > 1 && (!workspace || workspace_bytes < workspace_of(p))) return NSK_ERR_WORKSPACE;
    const dim3 grid(p.tiles, (unsigned)p.segments), block((unsigned)p.waves * 64);
    hipStream_t st = (hipStream_t)stream;
    float *ab = (float *)workspace;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (p.segments > 1) hipLaunchKernelGGL(glr_fwd_fold_kernel<T>, dim3(p.tiles, (unsigned)p.segments - 1), block, 0, st, p.z, (const T *)gi, bias, lengths, ab);
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
    if (p.segments > 1 && (!workspace || workspace_bytes < workspace_of(p))) return NSK_ERR_WORKSPACE;
    const dim3 grid(p.tiles, (unsigned)p.segments), block((unsigned)p.waves * 64);
    hipStream_t st = (hipStream_t)stream;
    float *ab = (float *)workspace;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (p.segments > 1) hipLaunchKernelGGL(glr_bwd_fold_kernel<T>, dim3(p.tiles, (unsigned)p.segments - 1), block, 0, st, p.z, (const T *)gi, bias, lengths, (const T *)dy, ab);
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
