// Gated linear recurrence: for every sequence and channel
//   f = sigmoid(gi_f + b_f), c = gi_c + b_c, o = sigmoid(gi_o + b_o),  h_t = f h_{t-1} + (1 - f) c,  y_t = o h_t,
// all steps in one call in both directions, and one token for each of many sequences.  Backwards, with G_t the gradient of h_t:
//   G_t = dy_t o_t + f_{t+1} G_{t+1},  dc = G (1 - f),  d gi_f = G (h_{t-1} - c) f (1 - f),  d gi_o = dy h o (1 - o),  dh0 = f_1 G_1.
#include <math.h>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

// exp(-m), m >= 0, to 3 units of 2^-24 and 0.05 m.  The hardware's exponential (1 ulp) takes t = m log2(e), whose rounding alone would put m such units into the result (a memory of 3000
// steps is a gate's argument of 8).  What t lost of the argument, m - t ln(2), comes back as a factor.  log2(e) is rounded down so far that nothing is ever gained: the fused product's clamp
// to [0, 1], which takes no instruction, changes nothing but the NaN of an infinite argument.  ln(2) in one word leaves the 0.05 m, 4 units where the exponential ends.
__device__ inline float exp_of_minus(float m)
{
    const float t = 1.4426949f * m, lost = fminf(fmaxf(fmaf(t, -0.693147182f, m), 0.f), 1.f), e = __builtin_amdgcn_exp2f(-t);
    return fmaf(e, -lost, e);
}
// sigmoid(a) and 1 - sigmoid(a), each to within 10 units of itself whatever the argument: near 1 the difference from it would keep none of the small one's.
// The reciprocal takes a Newton step: a product of hundreds of gates adds up a rounding that leans to one side (2000 steps of 256 channels, dh0 against 64 bits: 3.5e-7
// without the step, 2.0e-7 with it).
__device__ inline void sigmoid2(float a, float &s, float &rest)
{
    const float e = exp_of_minus(fabsf(a)), x = 1.f + e, y = __builtin_amdgcn_rcpf(x);
    const float big = fmaf(fmaf(-x, y, 1.f), y, y), small = e * big;
    s = a >= 0.f ? big : small;
    rest = a >= 0.f ? small : big;
}
// For a gate that stands in no product of many: the reciprocal (1 ulp) as it is, within the same 10 units.  (With the step, T=2048, N=32, bf16 768 channels forward 90 us and T=20, N=512 19.5,
// without 87 and 18.2.)
__device__ inline float sigmoid(float a)
{
    const float e = exp_of_minus(fabsf(a));
    return __builtin_amdgcn_rcpf(1.f + e) * (a >= 0.f ? 1.f : e);
}

// How the work is laid out.  A lane has one channel of one sequence, a wavefront 64 of them (a tile) and a stretch of 16 steps, whose values it keeps in registers:
// they are read once.  A stretch by itself takes a state h to A h + B; the wavefronts of a block take consecutive stretches (a segment) and exchange (A, B)
// through LDS.  Where a tile has several segments, a block leaves its segment's (A, B) in memory, finds the state that enters it from what the blocks before it
// left, leaves the state that leaves it, and then goes through its steps again, which are still in its registers.
// The state behind a segment is A h + B with the h in front of it, whichever block computes that, so the results do not depend on how far the others are.
// Waiting ends: blocks take numbers from a counter as they begin, and a block waits only for smaller numbers, whose blocks have begun and leave (A, B) before
// they wait themselves.  And if it did not (a caller that lets something else write to this call's workspace): after kPolls looks, about a second, a block goes through all steps
// in front of its own by itself.
constexpr int kStretch = NSK_GLR_STRETCH;
constexpr int kMostWaves = 16;
constexpr int kPolls = 1 << 20;
struct Sizes {
    int T, N, H;
    int stretches;          // of the whole sequence
    int segments;           // of `waves` stretches
    unsigned tiles;
    int groups;             // parts of the tiles that have counters of their own
    int flat;               // tiles go on across sequences (1), or each sequence has tiles of its own (0)
    int polls;              // looks after which a block makes the state that enters its segment itself
    long long gi_t, gi_n, y_t, y_n;
};
typedef unsigned long long u64;
// What blocks leave for each other, all ones where nothing is yet: (A, B) and the state behind every segment of every tile.
struct Exchange {
    unsigned *counters;     // one in 16 words is used
    u64 *ab;                // [segment][tile][64]
    unsigned *behind;       // [segment][tile][64]
};
constexpr int kMostGroups = 32, kCounterWords = kMostGroups * 16;
size_t exchange_words(const Sizes &z) { return kCounterWords + (size_t)z.segments * z.tiles * 64 * 3; }
Exchange exchange_at(void *workspace, const Sizes &z)
{
    unsigned *const w = (unsigned *)workspace;
    return {w, (u64 *)(w + kCounterWords), w + kCounterWords + (size_t)z.segments * z.tiles * 64 * 2};
}
// (vectors of four words; the counters are whole ones)
__global__ __launch_bounds__(256) void glr_unset_kernel(unsigned *__restrict__ w, size_t vectors)
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < vectors; i += (size_t)gridDim.x * 256) ((u32x4 *)w)[i] = u32x4(i < kCounterWords / 4 ? 0u : ~0u);
}
template <typename U> __device__ inline U seen(const U *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename U> __device__ inline void leave(U *p, U v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline unsigned bits(float v) { return __builtin_bit_cast(unsigned, v); }
__device__ inline float value(unsigned v) { return __builtin_bit_cast(float, v); }
constexpr unsigned kNaN = 0x7fc00000u;      // (in place of a NaN of all ones)

// The tile of this block and which of its segments (in the order in which they wait for each other); false: there is nothing left for it.
// Blocks are handed to the eight XCDs in turn: with 8 or 32 groups, all segments of a tile are on one XCD, and so are most neighbouring tiles, which share the cache
// lines at their ends where rows are not whole ones.  (us forward / backward, 1 / 8 / 32 groups, T=2048, N=32, bf16 768 channels, 12288 blocks of 4 wavefronts: 165 / 176,
// 89 / 143, 86 / 142: a counter gives out a number in 12 ns; ragged T=777, N=33, fp32 201 channels: 25 / 43, 19 / 37, 20 / 42.)
__device__ inline bool place(const Sizes &z, const Exchange &x, unsigned &tile, int &segment)
{
    const unsigned g = z.groups, group = blockIdx.x % g;
    const unsigned each = z.tiles / g, more = z.tiles % g, count = each + (group < more), first = group * each + (group < more ? group : more);
    unsigned number = blockIdx.x / g;
    if (z.segments > 1) {
        __shared__ unsigned taken;
        if (threadIdx.x == 0) taken = __hip_atomic_fetch_add(x.counters + group * 16, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        number = __builtin_amdgcn_readfirstlane(taken);
    }
    if (count == 0 || number / count >= (unsigned)z.segments) return false;
    segment = (int)(number / count);
    tile = first + number % count;
    return true;
}

// (Room in LDS where tiles are few and looks go back far: T=65536, N=1, bf16 512 channels 86 us without, 78 with it.  Small blocks look back one segment or two, and the LDS would leave fewer of
// them on a compute unit.)
__host__ __device__ inline int passed_of(int waves) { return waves >= 8 ? 24 : 0; }
// The state that enters a segment; called by one wavefront.  v0 enters the first one; A, B: this segment's; alone() goes through the steps in front of it.
template <typename F> __device__ inline float entering(const Sizes &z, const Exchange &x, unsigned tile, int segment, float v0, float A, float B, F &&alone)
{
    // (A, B) of the segments that the look passes, nearest first: a second load of them takes as long as a look
    extern __shared__ u64 passed[];
    const int room = passed_of(blockDim.x >> 6);
    if (z.segments == 1) return v0;
    const int lane = threadIdx.x & 63;
    const size_t step = (size_t)z.tiles * 64, at = (size_t)tile * 64 + lane;
    const bool last = segment == z.segments - 1;
    if (segment > 0 && !last) {
        const u64 ab = (u64)bits(B) << 32 | bits(A);
        leave(x.ab + segment * step + at, ab == ~0ull ? (u64)kNaN << 32 | kNaN : ab);
    }
    // back to the nearest segment whose state is there, over those whose (A, B) are, four at a time
    float v = v0;
    int j = segment - 1, polls = z.polls;
    for (bool found = false; j >= 0 && !found;) {
        unsigned behind[4];
        u64 ab[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t k = (size_t)(j - i > 0 ? j - i : 0) * step + at;
            behind[i] = seen(x.behind + k);
            ab[i] = seen(x.ab + k);
        }
        bool wait = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (found || wait || j < 0) continue;
            if (!__builtin_amdgcn_ballot_w64(behind[i] == ~0u)) {
                v = value(behind[i]);
                found = true;
            } else if (j > 0 && !__builtin_amdgcn_ballot_w64(ab[i] == ~0ull)) {
                if (segment - 1 - j < room) passed[(segment - 1 - j) * 64 + lane] = ab[i];
                --j;
            } else wait = true;
        }
        if (wait && polls-- <= 0) {
            v = alone();
            j = segment;        // (nothing is left to apply)
            break;
        }
        if (wait) __builtin_amdgcn_s_sleep(2);
    }
    // and on from there: over those further back than there was room for first
    int k = j + 1;
#pragma unroll 4
    for (; k < segment - room; ++k) {
        const u64 ab = seen(x.ab + k * step + at);
        v = fmaf(value((unsigned)ab), v, value((unsigned)(ab >> 32)));
    }
    for (; k < segment; ++k) {
        const u64 ab = passed[(segment - 1 - k) * 64 + lane];
        v = fmaf(value((unsigned)ab), v, value((unsigned)(ab >> 32)));
    }
    if (!last) {
        const unsigned behind = bits(fmaf(A, v, B));
        leave(x.behind + segment * step + at, behind == ~0u ? kNaN : behind);
    }
    return v;
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

// Loads of a stretch: gates f, c and o into f, x and o, biases added.
template <typename T>
__device__ inline void load_gates(const T *gi, const Sizes &z, const Lane &l, const Bias &b, int t0, float (&f)[kStretch], float (&x)[kStretch], float (&o)[kStretch])
{
    const unsigned gate = (unsigned)z.H * (unsigned)sizeof(T);
    Rows<const T> in{gi, z.T - t0};
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        const __amdgpu_buffer_rsrc_t r = in.at();
        f[i] = load<T>(r, l.gi, 0);
        x[i] = load<T>(r, l.gi, gate);
        o[i] = load<T>(r, l.gi, 2 * gate);
        in.move(z.gi_t);
    }
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        f[i] += b.f;
        x[i] += b.c;
        o[i] += b.o;
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
__device__ inline void apply_gates(float (&f)[kStretch], float (&x)[kStretch], float (&o)[kStretch])
{
#pragma unroll
    for (int i = 0; i < kStretch; ++i) {
        float s, keep;
        sigmoid2(f[i], s, keep);
        x[i] *= keep;
        f[i] = s;
        o[i] = sigmoid(o[i]);
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

// (A, B) of a block's stretches through LDS; the value that enters this wavefront's stretch, and the one that leaves the block's last.
template <typename F> __device__ inline float join(const Sizes &z, const Exchange &x, unsigned tile, int segment, float v0, float A, float B, float &leaves, F &&alone)
{
    __shared__ float part[kMostWaves][2][64], enters[64];
    const int lane = threadIdx.x & 63, wave = wave_of_block(), waves = blockDim.x >> 6;
    part[wave][0][lane] = A;
    part[wave][1][lane] = B;
    lds_barrier();
    if (z.segments > 1) {
        if (wave == 0) {
            A = 1.f;
            B = 0.f;
            for (int w = 0; w < waves; ++w) {
                A *= part[w][0][lane];
                B = fmaf(part[w][0][lane], B, part[w][1][lane]);
            }
            v0 = entering(z, x, tile, segment, v0, A, B, alone);
            enters[lane] = v0;
            leaves = fmaf(A, v0, B);
        }
        lds_barrier();
        v0 = enters[lane];
    }
    float mine = v0;
    for (int w = 0; w < waves; ++w) {
        if (w == wave) mine = v0;
        v0 = fmaf(part[w][0][lane], v0, part[w][1][lane]);
    }
    if (z.segments == 1) leaves = v0;
    return mine;
}

// Bound by memory where tiles are many (3 + 1 elements and 1/4 byte a step and channel): bf16, T=2048, N=32, 768 channels 87 us, 4.8 TB/s of what a copy reaches 5.1 of;
// the vector unit, with four transcendental of some 25 instructions a step, is half busy.  By the hand-over where tiles are few: bf16, T=65536, N=1, 512 channels
// 77 us (3.6 TB/s; of the 13 us that a block lasts, its number takes 1, its loads 2, its steps 2, looking back 5 to 6: two or three loads one behind the other, 2 us each while the memory is
// loaded); and by one chain of loads, gates and stores where a call is short: fp32, T=200,
// N=50, 256 channels 12 us for 42 MB.  (Wider look-backs, 8 or 16 segments at a time or 4 by each wavefront, cost more in traffic than they gave: 92, 97, 118 us for the long one.)
template <typename T>
__global__ __launch_bounds__(1024) void glr_fwd_kernel(Sizes z, Exchange ex, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                       const float *__restrict__ h0, T *__restrict__ y, float *__restrict__ h_last, float *__restrict__ saved)
{
    unsigned tile;
    int segment;
    if (!place(z, ex, tile, segment)) return;
    long long gi0, y0;
    const Lane l = lane_of<T>(z, tile, gi0, y0);
    const long long all = (long long)z.N * z.H;
    const int len = steps_of(lengths, l, z.T);
    const Bias b = bias_of(bias, z, l);
    const int wave = wave_of_block(), s = segment * (int)(blockDim.x >> 6) + wave, t0 = s * kStretch;
    float f[kStretch], x[kStretch], o[kStretch], A = 1.f, B = 0.f, leaves;
    const bool mine = s < z.stretches, some = mine && any(t0 < len), ends = any(t0 + kStretch > len);
    if (some) {
        load_gates<T>(gi + gi0 + t0 * z.gi_t, z, l, b, t0, f, x, o);
        if (ends) leave_state(len - t0, f, x);
        apply_gates(f, x, o);
        fold(f, x, A, B);
    }
    const float start = h0 ? h0[l.q] : 0.f;
    float h = join(z, ex, tile, segment, start, A, B, leaves, [&] {
        float v = start;
        const int end = segment * (int)(blockDim.x >> 6) * kStretch;
#pragma unroll 1
        for (int t = 0; t < end; ++t) {
            const __amdgpu_buffer_rsrc_t r = Rows<const T>{gi + gi0 + t * z.gi_t, 1}.at();
            float s, rest;
            sigmoid2(load<T>(r, l.gi, 0) + b.f, s, rest);
            const float c = load<T>(r, l.gi, (unsigned)z.H * (unsigned)sizeof(T)) + b.c;
            v = t < len ? s * v + rest * c : v;
        }
        return v;
    });
    if (h_last && segment == z.segments - 1 && wave == 0 && l.there) h_last[l.q] = leaves;
    if (!mine) return;
    if (saved && l.there) saved[s * all + l.q] = h;
    if (!y) return;
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

// bf16, T=2048, N=32, 768 channels 144 us, 5.0 TB/s; fp32 with lengths and odd rows, T=777, N=33, 201 channels 36 us; T=200, N=50, fp32 256 channels 15.4 us.
// Backwards a stretch takes E, the gradient of the state that leaves it, to A E + B.  What a step needs for that: f, u = dy o, and with the states, which
// come from the saved one, k = 1 - f and d = (h_{t-1} - c) f (1 - f).  The gradient of the gate o depends on nothing later.
template <typename T>
__global__ __launch_bounds__(1024) void glr_bwd_kernel(Sizes z, Exchange ex, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                       const float *__restrict__ saved, const T *__restrict__ dy, const float *__restrict__ dh_last, T *__restrict__ dgi,
                                                       float *__restrict__ dh0)
{
    unsigned tile;
    int segment;
    if (!place(z, ex, tile, segment)) return;
    long long gi0, y0;
    const Lane l = lane_of<T>(z, tile, gi0, y0);
    const long long all = (long long)z.N * z.H;
    const int len = steps_of(lengths, l, z.T);
    const Bias b = bias_of(bias, z, l);
    const unsigned gate = (unsigned)z.H * (unsigned)sizeof(T);
    // segments and, in a block, wavefronts go from the end to the front
    const int wave = wave_of_block(), waves = blockDim.x >> 6, s = (z.segments - segment) * waves - 1 - wave, t0 = s * kStretch;
    const bool mine = s < z.stretches, some = mine && any(t0 < len), ends = any(t0 + kStretch > len);
    float f[kStretch], keep[kStretch], u[kStretch], d[kStretch], q[kStretch], A = 1.f, B = 0.f, leaves;
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
            q[i] = u[i] * shut * h;     // (stored at the end: the loads that look for other blocks' values would wait for it)
        }
#pragma unroll
        for (int i = kStretch - 1; i >= 0; --i) {
            A *= f[i];
            B = f[i] * (B + u[i]);
        }
    }
    const float start = dh_last ? dh_last[l.q] : 0.f;
    float E = join(z, ex, tile, segment, start, A, B, leaves, [&] {
        float v = start;
        const int end = (z.segments - segment) * waves * kStretch;
#pragma unroll 1
        for (int t = z.T - 1; t >= end; --t) {
            const __amdgpu_buffer_rsrc_t r = Rows<const T>{gi + gi0 + t * z.gi_t, 1}.at(), ry = Rows<const T>{dy + y0 + t * z.y_t, dy ? 1 : 0}.at();
            const float o = sigmoid(load<T>(r, l.gi, 2 * gate) + b.o), up = load<T>(ry, l.y, 0);
            float s, rest;
            sigmoid2(load<T>(r, l.gi, 0) + b.f, s, rest);
            v = t < len ? s * (v + up * o) : v;
        }
        return v;
    });
    if (dh0 && segment == z.segments - 1 && wave == 0 && l.there) dh0[l.q] = leaves;
    if (!mine) return;
    if (some) {
        Rows<T> out{dgi + at + (kStretch - 1) * z.gi_t, z.T - t0 - (kStretch - 1)};
#pragma unroll
        for (int i = kStretch - 1; i >= 0; --i) {
            const __amdgpu_buffer_rsrc_t r = out.at();
            const float G = E + u[i];
            store<T>(G * d[i], r, l.gi, 0);
            store<T>(G * keep[i], r, l.gi, gate);
            store<T>(q[i], r, l.gi, 2 * gate);
            E = f[i] * G;
            out.move(-z.gi_t, -1);
        }
    }
    if (ends) store_zeros(dgi + at, z.gi_t, len - t0, z.T - t0 < kStretch ? z.T - t0 : kStretch, l.gi, gate, 3);
}

// An element a lane, 64 of a sequence a block.  us on the device in bf16 / fp32 (floor): N=50, 256 channels 2.6, latency alone; N=1024, 1024 channels 6.8 / 7.1 (3.3 / 4.9), from the last-level
// cache, and less than the host takes for the call; N=4096, 2048 channels 33.6 / 41.4 (26.4 / 39.6): memory in fp32; in bf16 loads and stores of 2 bytes a lane reach 4.0 TB/s.
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
    // (a launch has fewer than 2^32 threads: one a channel and stretch at most)
    if (d.T > 1 << 30 || (long long)d.N * ((d.H + 63) / 64) > (3LL << 30) / ((d.T + kStretch - 1) / kStretch + kMostWaves) / 64) return NSK_ERR_UNSUPPORTED;
    return NSK_OK;
}

// Tiles, segments and wavefronts of a call.
struct Plan {
    Sizes z;
    int waves;
    unsigned blocks;
};
Plan plan_of(const nsk_glr_desc_t &d, int pass)
{
    Plan p{};
    const long long es = d.dtype == NSK_BF16 ? 2 : 4;
    p.z = {d.T, d.N, d.H, ceil_div(d.T, kStretch), 1, 0, 1, 0, hooks().glr_polls >= 0 ? hooks().glr_polls : kPolls, d.gi_t, d.gi_n, d.y_t, d.y_n};
    // a tile reaches over 63 / H + 1 further sequences, whose offsets have to fit 30 bits (those of a single sequence do)
    const long long over = d.H < 64 ? 63 / d.H + 1 : 1, stride = d.gi_n > d.y_n ? d.gi_n : d.y_n;
    p.z.flat = stride < (1LL << 30) && (over * stride + d.H) * es < (1LL << 30);
    const long long tiles = p.z.flat ? ((long long)d.N * d.H + 63) / 64 : (long long)d.N * ((d.H + 63) / 64);
    p.z.tiles = (unsigned)tiles;
    p.z.groups = tiles >= 256 ? kMostGroups : tiles >= 8 ? 8 : 1;
    // Small blocks where there are many: they fill the compute units evenly and wait at different times; no more places than stretches, an idle wavefront holds registers.
    // Large ones where tiles are few: fewer segments have to find each other.  us forward / backward with 2 / 4 / 8 / 16 wavefronts: T=200, N=512, bf16 768 channels (6144 tiles) 156 / 250,
    // 165 / 274, 183 / 315; T=2048, N=32, bf16 768 channels (384) 104 / 154, 86 / 142, 89 / 157, 111 / 171; T=65536, N=1, bf16 512 channels (8) 246 / 243, 122 / 154, 84 / 128, 85 / 127; the same with
    // 64 channels (one) 78 / 80 with 4, 44 / 47, 29 / 32.  T=130 (9 stretches), N=512, bf16 768 channels, 2 / 3 of them: 113 / 173, 101 / 169.
    // One segment and no exchange where a block can take all stretches: up to 8 (T=128, N=256, bf16 1280 channels, one / two segments: 79 / 137, 84 / 138), up to 16
    // while every block has a compute unit to itself (T=200, N=50, fp32 256 channels: 11.0 / 14.9, 14.0 / 17.1); the backward pass, of whose wavefronts a unit holds 16, has no room for
    // two or three whole blocks of 5 to 8 where many are waiting (N=512, bf16 768 channels, one segment / blocks of two, backward: T=80 119, 106; T=96 132, 120; T=128 162, 157; with
    // 1024 tiles, N=128 and 512 channels, T=112: 26.9, 29.1).
    const int few = p.z.stretches % 6 == 3 ? 3 : 2;
    const int most = tiles >= 1024 ? few : tiles > 256 ? 4 : tiles >= 8 ? 8 : kMostWaves;
    const int whole = pass == NSK_PASS_DGRAD && tiles >= 2048 ? 4 : 8;
    p.z.segments = p.z.stretches <= whole || (p.z.stretches <= kMostWaves && tiles <= 256) ? 1 : ceil_div(p.z.stretches, most);
    p.waves = ceil_div(p.z.stretches, p.z.segments);
    p.z.segments = ceil_div(p.z.stretches, p.waves);
    // (as many blocks for every group, so some of them may find nothing left: by what check() lets through, tiles * segments blocks are fewer than 2^32 threads, but these need not be)
    auto blocks = [&] { return (tiles + p.z.groups - 1) / p.z.groups * p.z.groups * p.z.segments; };
    if (blocks() * p.waves * 64 >= 1LL << 32) p.z.groups = 1;
    p.blocks = (unsigned)blocks();
    return p;
}
size_t workspace_of(const Plan &p) { return p.z.segments > 1 ? exchange_words(p.z) * sizeof(unsigned) : 0; }
// Puts the marks where blocks will look for each other's values.
void unset(const Plan &p, void *workspace, hipStream_t st)
{
    if (p.z.segments == 1) return;
    const size_t vectors = exchange_words(p.z) / 4, blocks = (vectors + 255) / 256;
    hipLaunchKernelGGL(glr_unset_kernel, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, st, (unsigned *)workspace, vectors);
}

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
    return (pass == NSK_PASS_FWD || pass == NSK_PASS_DGRAD) && check(desc, d) == NSK_OK ? workspace_of(plan_of(d, pass)) : 0;
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
    const Plan p = plan_of(d, NSK_PASS_FWD);
    if (p.z.segments > 1 && (!workspace || workspace_bytes < workspace_of(p))) return NSK_ERR_WORKSPACE;
    const dim3 grid(p.blocks), block((unsigned)p.waves * 64);
    hipStream_t st = (hipStream_t)stream;
    const Exchange ex = exchange_at(workspace, p.z);
    unset(p, workspace, st);
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        hipLaunchKernelGGL(glr_fwd_kernel<T>, grid, block, p.z.segments > 1 ? passed_of(p.waves) * 64 * sizeof(u64) : 0, st, p.z, ex, (const T *)gi, bias, lengths, h0, (T *)y, h_last, saved);
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
    const Plan p = plan_of(d, NSK_PASS_DGRAD);
    if (p.z.segments > 1 && (!workspace || workspace_bytes < workspace_of(p))) return NSK_ERR_WORKSPACE;
    const dim3 grid(p.blocks), block((unsigned)p.waves * 64);
    hipStream_t st = (hipStream_t)stream;
    const Exchange ex = exchange_at(workspace, p.z);
    unset(p, workspace, st);
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        hipLaunchKernelGGL(glr_bwd_kernel<T>, grid, block, p.z.segments > 1 ? passed_of(p.waves) * 64 * sizeof(u64) : 0, st, p.z, ex, (const T *)gi, bias, lengths, saved, (const T *)dy, dh_last, (T *)dgi, dh0);
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
    if ((long long)tiles * N >= 1 << 26) return NSK_ERR_UNSUPPORTED;        // (2^32 threads)
    const dim3 grid(tiles * (unsigned)N);
    if (dtype == NSK_BF16)
        hipLaunchKernelGGL(glr_step_kernel<bf16_t>, grid, dim3(64), 0, (hipStream_t)stream, H, S, (const bf16_t *)gi, bias, slots, state, (bf16_t *)y, tiles);
    else
        hipLaunchKernelGGL(glr_step_kernel<float>, grid, dim3(64), 0, (hipStream_t)stream, H, S, (const float *)gi, bias, slots, state, (float *)y, tiles);
    return check_launch();
}

}  // extern "C"
