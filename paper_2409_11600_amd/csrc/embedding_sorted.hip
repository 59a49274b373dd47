// Embedding with a scale, and its gradient by sorted tokens.
//   out_i = scale * table[token_i],   dtable_v (+)= scale * sum over the positions i with token_i = v of dout_i;  a padding token has zeros and no gradient.
// Both are bound by memory: the forward pass reads and writes a row a position; the gradient reads a row a position and writes a row a token.  Sorting the positions
// by token (stable: a token's stay in order) makes the rows of a token neighbours, so that a wavefront adds them up in registers and the time does not depend
// on how often a token occurs.
#include <math.h>

#include <type_traits>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }
bool dtype_ok(int dtype) { return dtype == NSK_F32 || dtype == NSK_BF16; }

// ----------------------------------------------------------------------------- forward
// Sixteen bytes a lane, or an element where rows do not begin on vectors.  A block takes kThreads * 4 of them in a row.
// (50 rows of 256 in bf16: 2.8 us, two loads one after the other.)
constexpr int kThreads = 256, kEach = 4;
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void embedding_scaled_fwd_kernel(const int *__restrict__ tokens, const T *__restrict__ table, T *__restrict__ out, long long n, int vectors, Div by,
                                                                        int rows, int pad, float scale)
{
    struct alignas(sizeof(T) * V) Vec {
        T v[V];
    };
    const long long first = (long long)blockIdx.x * (kThreads * kEach), total = n * vectors;
    const long long row0 = first / vectors;
    const int rest = (int)(first - row0 * vectors);
    Vec x[kEach];
    int token[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int at = e * kThreads + threadIdx.x, row = divide(rest + at, by);
        token[e] = 0;
        x[e] = {};
        if (first + at >= total) continue;
        token[e] = tokens[row0 + row];
        if (token[e] >= 0 && token[e] < rows && token[e] != pad) x[e] = ((const Vec *)table)[(long long)token[e] * vectors + (rest + at - row * vectors)];
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const long long at = first + e * kThreads + threadIdx.x;
        if (at >= total) continue;
        const bool wrong = token[e] < 0 || token[e] >= rows;
#pragma unroll
        for (int i = 0; i < V; ++i) x[e].v[i] = (T)(wrong ? NAN : token[e] == pad ? 0.f : scale * (float)x[e].v[i]);
        ((Vec *)out)[at] = x[e];
    }
}

// ----------------------------------------------------------------------------- sorting
__device__ __forceinline__ int lanes_below(unsigned long long ballot)
{
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(ballot >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)ballot, 0));
}
// Zeros, by the blocks that a launch has beyond those of its work.
__device__ __forceinline__ void fill(float *table, size_t elements, unsigned block, unsigned blocks)
{
    for (size_t i = (size_t)block * blockDim.x + threadIdx.x; i < elements / 4; i += (size_t)blocks * blockDim.x) ((f32x4 *)table)[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (block == 0 && threadIdx.x < elements % 4) table[elements / 4 * 4 + threadIdx.x] = 0.f;
}

// Keys are compared as unsigned numbers, so what is no token (negative, or V and more) comes behind all tokens.

// Passes over digits of the key, the lowest first, each stable.  A block takes kTile positions, each of its wavefronts a quarter of them in order.
constexpr int kBits = 9, kDigits = 1 << kBits, kTile = 1024, kWaves = kThreads / 64;
__device__ __forceinline__ int digit_of(unsigned key, int shift) { return (int)(key >> shift) & (kDigits - 1); }
// Where this lane's position goes, in order of the lanes of equal digits; `next`: the wavefront's next place of each digit.
__device__ __forceinline__ int place_of(int digit, bool there, int *next)
{
    unsigned long long same = __ballot(there);
#pragma unroll
    for (int b = 0; b < kBits; ++b) {
        const unsigned long long set = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? set : ~set;
    }
    const int rank = lanes_below(same);
    int at = 0;
    if (there) at = next[digit] + rank;
    __builtin_amdgcn_wave_barrier();
    if (there && rank == 0) next[digit] = at + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    return at;
}
// (What is no token is V here: as few digits as there can be.)
__device__ __forceinline__ unsigned key_at(const unsigned *from, int i, unsigned V) { return from[i] < V ? from[i] : V; }
__global__ __launch_bounds__(kThreads) void digits_kernel(const unsigned *__restrict__ from, int n, unsigned V, int shift, int tiles, int *__restrict__ counts, float *table, size_t elements,
                                                        int *__restrict__ list)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) list[0] = 0;
    if ((int)blockIdx.x >= tiles) return fill(table, elements, blockIdx.x - tiles, gridDim.x - tiles);
    __shared__ int found[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kThreads) found[d] = 0;
    __syncthreads();
    const int base = blockIdx.x * kTile;
    for (int i = threadIdx.x; i < kTile && base + i < n; i += kThreads) atomicAdd(&found[digit_of(key_at(from, base + i, V), shift)], 1);
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kThreads) counts[(size_t)d * tiles + blockIdx.x] = found[d];
}
// Exclusive sums over the tiles of a digit; the digit's total behind all of them.
__global__ __launch_bounds__(64) void places_kernel(int tiles, int *__restrict__ counts)
{
    int *c = counts + (size_t)blockIdx.x * tiles, carry = 0;
    for (int base = 0; base < tiles; base += 64) {
        const int i = base + threadIdx.x, v = i < tiles ? c[i] : 0;
        int s = v;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(s, o, 64);
            if ((int)threadIdx.x >= o) s += up;
        }
        if (i < tiles) c[i] = carry + s - v;
        carry += __shfl(s, 63, 64);
    }
    if (threadIdx.x == 0) counts[(size_t)kDigits * tiles + blockIdx.x] = carry;
}
__global__ __launch_bounds__(kThreads) void scatter_kernel(const unsigned *__restrict__ from, const int *__restrict__ from_order, int n, unsigned V, int shift, int tiles,
                                                           const int *__restrict__ counts, unsigned *__restrict__ keys, int *__restrict__ order)
{
    __shared__ int next[kWaves][kDigits];       // where a wavefront's next position of a digit goes
    __shared__ int sums[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, base = blockIdx.x * kTile + wave * (kTile / kWaves);
    for (int d = threadIdx.x; d < kWaves * kDigits; d += kThreads) (&next[0][0])[d] = 0;
    __syncthreads();
    unsigned key[kTile / kThreads];
#pragma unroll
    for (int r = 0; r < kTile / kThreads; ++r) {
        const int i = base + r * 64 + lane;
        key[r] = i < n ? key_at(from, i, V) : 0;
        if (i < n) atomicAdd(&next[wave][digit_of(key[r], shift)], 1);
    }
    __syncthreads();
    // the digits in front of this one, over all tiles; two digits a thread
    static_assert(kDigits == 2 * kThreads, "two digits a thread");
    const int d0 = 2 * threadIdx.x, *totals = counts + (size_t)kDigits * tiles, t0 = totals[d0], t1 = totals[d0 + 1];
    int s = t0 + t1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(s, o, 64);
        if (lane >= o) s += up;
    }
    if (lane == 63) sums[wave] = s;
    __syncthreads();
    s -= t0 + t1;
    for (int w = 0; w < wave; ++w) s += sums[w];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        int at = s + (e ? t0 : 0) + counts[(size_t)(d0 + e) * tiles + blockIdx.x];
        for (int w = 0; w < kWaves; ++w) {
            const int c = next[w][d0 + e];
            next[w][d0 + e] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kTile / kThreads; ++r) {
        const int i = base + r * 64 + lane;
        const bool there = i < n;
        if (!__ballot(there)) break;
        const int at = place_of(digit_of(key[r], shift), there, next[wave]);
        if (there) {
            keys[at] = key[r];
            order[at] = from_order ? from_order[i] : i;
        }
    }
}

// Few positions: the place of one is the number of those in front of it, counted by comparing it with all, in one launch (six launches of the kernels above wait for each other longer than they
// work: us of a call for 256 columns of fp32, 32768 words, this one / those, n = 2000 18 / 40, 10000 29 / 43, 16384 39 / 46, 20000 71 / 48 with stretches alike; all passes in one block of 16
// wavefronts took 29 us for 10000 positions, where this one takes 16, and 19 beside the zeros of a table of 34 MB).  A block has 64 positions; its wavefronts share the others, whose keys are the same for all
// lanes: scalar loads.  A comparison is min(a - b, 1) without wrapping, two keys at a time where they have 16 bits: three vector instructions a pair, beside four scalar
// ones that clamp and pack its keys.  At n = 10000 the 157 blocks issue 2.5 million vector and 3.5 million scalar instructions, 6.6 and 9.2 us of what a unit issues of each, and wait 0.47 of their time.
constexpr int kRankWaves = 16, kFew = 16384;
template <bool NARROW>
__global__ __launch_bounds__(kRankWaves * 64) void rank_kernel(const unsigned *__restrict__ tokens, int n, unsigned V, unsigned *__restrict__ keys, int *__restrict__ order, unsigned ranking,
                                                               float *table, size_t elements, int *__restrict__ list)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) list[0] = 0;
    if (blockIdx.x >= ranking) return fill(table, elements, blockIdx.x - ranking, gridDim.x - ranking);
    typedef unsigned u32x16 __attribute__((ext_vector_type(16), aligned(4)));
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    __shared__ int counts[kRankWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int base = blockIdx.x * 64, i = base + lane;
    const unsigned mine = i < n ? key_at(tokens, i, V) : 0;
    const int groups = n / 64, each = (groups + kRankWaves - 1) / kRankWaves, first = wave * each, last = groups - first < each ? groups : first + each;
    int count = 0;
    // whole groups of 64 keys: in front of the block's positions equal keys come first, behind them they do not.  (The subtractions are written out: of min(a - b, 1) the compiler makes a
    // comparison, a selection and a wait between them, four times as long.)
    auto below = [&](int from, int to, unsigned border) {
        unsigned pair = 0;
        const unsigned borders = border | border << 16;
        for (int g = from; g < to; ++g) {
            u32x16 k[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) k[q] = *(const u32x16 *)(tokens + 64 * g + 16 * q);
#pragma unroll
            for (int e = 0; e < 64; e += 2) {
                const unsigned x = k[e / 16][e % 16], y = k[e / 16][e % 16 + 1], a = x < V ? x : V, b = y < V ? y : V;
                if constexpr (NARROW) {
                    unsigned over;
                    asm("v_pk_sub_u16 %0, %1, %2 clamp" : "=v"(over) : "v"(borders), "s"(a | b << 16));
                    asm("v_pk_min_u16 %0, %1, %2" : "=v"(over) : "v"(over), "s"(0x00010001));
                    pair = __builtin_bit_cast(unsigned, __builtin_bit_cast(u16x2, pair) + __builtin_bit_cast(u16x2, over));
                } else {
                    unsigned over[2];
                    asm("v_sub_u32 %0, %1, %2 clamp" : "=v"(over[0]) : "v"(border), "s"(a));
                    asm("v_sub_u32 %0, %1, %2 clamp" : "=v"(over[1]) : "v"(border), "s"(b));
                    count += (over[0] < 1u ? over[0] : 1u) + (over[1] < 1u ? over[1] : 1u);
                }
            }
        }
        count += (pair & 0xffff) + (pair >> 16);
    };
    const int own = blockIdx.x;
    auto least = [](int a, int b) { return a < b ? a : b; };
    auto most = [](int a, int b) { return a > b ? a : b; };
    below(first, least(last, own), mine + 1);
    below(most(first, own + 1), last, mine);
    // the block's own positions, and those behind the last whole group: a key a lane
    if (wave < 2) {
        const int at = wave ? 64 * groups : base, there = wave ? n - at : own < groups ? 64 : 0;
        const unsigned key = lane < there ? key_at(tokens, at + lane, V) : 0;
        for (int e = 0; e < there; ++e) {
            const unsigned k = __builtin_amdgcn_readlane(key, e);
            count += k < mine || (k == mine && at + e < i);
        }
    }
    counts[wave][lane] = count;
    __syncthreads();
    if (wave || i >= n) return;
    int place = 0;
#pragma unroll
    for (int w = 0; w < kRankWaves; ++w) place += counts[w][lane];
    keys[place] = mine;
    order[place] = i;
}

// ----------------------------------------------------------------------------- sums of runs
// A wavefront takes a stretch of sorted positions and 256 columns.  A token whose positions begin in it and end in it or the next stretch it adds up as a whole.  Of a longer one, what lies in
// its stretch is left in memory (at most two rows), and the wavefront in whose stretch the token begins puts it on a list; join_kernel adds the parts up in order.  Bound by memory where the rows are
// many: 262144 rows of 768 in bf16 into 65536 rows of fp32 take 140 to 146 us, 3.6 TB/s of rows of 512 bytes from all over (the stream of the same bytes takes 100), the joins 12.
constexpr int kCols = 256;
constexpr int kMostRun = 32;
struct Runs {
    int n, E;
    unsigned V, pad;
    int run, stretches, chunks;
    float scale;
    int accumulate;
};
template <typename T, bool VEC> struct Row;
template <typename T> struct Row<T, true> {         // four columns in a row
    float v[4];
    __device__ __forceinline__ void load(const T *p, int left)
    {
        struct alignas(4 * sizeof(T)) Q {
            T q[4];
        };
        Q q{};
        if (left > 0) q = *(const Q *)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)q.q[e];
    }
    static __device__ __forceinline__ int column(int lane) { return 4 * lane; }
    static __device__ __forceinline__ void store(float *p, int left, const float (&s)[4]) { if (left > 0) *(f32x4 *)p = (f32x4){s[0], s[1], s[2], s[3]}; }
};
template <typename T> struct Row<T, false> {        // every 64th column
    float v[4];
    __device__ __forceinline__ void load(const T *p, int left)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = 64 * e < left ? (float)p[64 * e] : 0.f;
    }
    static __device__ __forceinline__ int column(int lane) { return lane; }
    static __device__ __forceinline__ void store(float *p, int left, const float (&s)[4])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (64 * e < left) p[64 * e] = s[e];
    }
};
// dtable (+)= scale * sum
template <bool VEC> __device__ __forceinline__ void finish(const Runs &z, float *p, int left, const float (&sum)[4])
{
    float s[4];
    Row<float, VEC> old;
    if (z.accumulate) old.load(p, left);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = z.accumulate ? fmaf(z.scale, sum[e], old.v[e]) : z.scale * sum[e];
    Row<float, VEC>::store(p, left, s);
}
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void runs_kernel(Runs z, const unsigned *__restrict__ keys, const int *__restrict__ order, const T *__restrict__ dout, float *__restrict__ dtable,
                                                        float *__restrict__ left_over, int *__restrict__ list)
{
    const int lane = threadIdx.x & 63;
    const long long task = (long long)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int stretch = (int)(task / z.chunks), chunk = (int)(task - (long long)stretch * z.chunks);
    if (stretch >= z.stretches) return;
    const int from = stretch * z.run, to = z.n - from < z.run ? z.n : from + z.run;
    const int col = chunk * kCols + Row<T, VEC>::column(lane), left = z.E - col;
    // the stretch's keys and positions, one a lane; the neighbours' keys behind them
    const int at = from + lane;
    const int end = z.n - from < 2 * z.run ? z.n : from + 2 * z.run;
    const unsigned my_key = at < end ? keys[at] : z.V, key_before = from ? keys[from - 1] : z.V, key_behind = end < z.n ? keys[end] : z.V;
    const int my_pos = at < end ? order[at] : 0;
    const int count = to - from, all = end - from;      // positions of the stretch, and of it and the next
    // the token that goes on from the stretch in front: taken there, as a whole, if it began in it and ends here
    const unsigned first_key = __builtin_amdgcn_readlane(my_key, 0), last_key = __builtin_amdgcn_readlane(my_key, count - 1);
    const bool goes_on = from && key_before == first_key;
    const bool began_before = goes_on && from > z.run && keys[from - z.run - 1] == first_key;           // further than one stretch in front
    auto key_of = [&](int i) { return i < all ? (unsigned)__builtin_amdgcn_readlane(my_key, i) : key_behind; };
    const bool whole_stretch = first_key == key_of(count);      // it goes on behind this stretch too
    int begin = 0;
    if (goes_on && !began_before && !whole_stretch)
        while (begin < count && key_of(begin) == first_key) ++begin;
    // the last token, if it began here: on to its end, or left as a part
    const bool last_goes_on = key_of(count) == last_key, last_whole = last_goes_on && !(goes_on && first_key == last_key) && (all < 2 * z.run || key_behind != last_key);
    int stop = count;
    if (last_whole)
        while (stop < all && key_of(stop) == last_key) ++stop;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8;
    for (int base = begin; base < stop; base += U) {
        Row<T, VEC> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u < stop ? base + u : base;
            const unsigned k = __builtin_amdgcn_readlane(my_key, i);
            const long long pos = __builtin_amdgcn_readlane(my_pos, i);
            x[u].load(dout + pos * z.E + col, base + u < stop && k < z.V && k != z.pad ? left : 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u;
            if (i >= stop) break;
            const unsigned k = __builtin_amdgcn_readlane(my_key, i);
            if (k >= z.V) return;               // only what is no token comes behind
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += x[u].v[e];
            if (i + 1 < stop && key_of(i + 1) == k) continue;
            const bool head = goes_on && k == first_key, tail = i + 1 == stop && last_goes_on && !last_whole;
            if (k != z.pad) {
                if (head || tail) Row<float, VEC>::store(left_over + ((size_t)stretch * 2 + (head ? 0 : 1)) * z.E + col, left, sum);
                else finish<VEC>(z, dtable + (size_t)k * z.E + col, left, sum);
                if (tail && !head && chunk == 0 && lane == 0) list[1 + atomicAdd(list, 1)] = stretch;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = 0.f;
        }
    }
}
// The tokens of the list (whose order says nothing: each is a row of its own): their parts, in order.  The wavefronts of a block take as many stretches each, one after the other.
constexpr int kJoinWaves = 8, kJoinBlocks = 512;
template <bool VEC>
__global__ __launch_bounds__(kJoinWaves * 64) void join_kernel(Runs z, const unsigned *__restrict__ keys, float *__restrict__ dtable, const float *__restrict__ left_over,
                                                               const int *__restrict__ list)
{
    __shared__ float part[kJoinWaves][kCols];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.y * kCols + Row<float, VEC>::column(lane), left = z.E - col;
    for (int entry = blockIdx.x; entry < list[0]; entry += gridDim.x) {
        const int stretch = list[1 + entry];
        const unsigned key = keys[(size_t)(stretch + 1) * z.run];
        // stretches behind this one whose first position is the token's
        int count = 0;
        for (int base = stretch + 1;; base += kJoinWaves * 64) {
            const int s = base + threadIdx.x;
            const int mine = __syncthreads_count(s < z.stretches && keys[(size_t)s * z.run] == key);
            count += mine;
            if (mine < kJoinWaves * 64) break;
        }
        const int each = (count + kJoinWaves - 1) / kJoinWaves, first = wave * each, last = count - first < each ? count : first + each;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        if (wave == 0) {
            Row<float, VEC> x;
            x.load(left_over + ((size_t)stretch * 2 + 1) * z.E + col, left);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = x.v[e];
        }
        constexpr int U = 8;
        for (int base = first; base < last; base += U) {
            Row<float, VEC> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u].load(left_over + (size_t)(stretch + 1 + (base + u < last ? base + u : base)) * 2 * z.E + col, base + u < last ? left : 0);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += x[u].v[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) part[wave][e * 64 + lane] = sum[e];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                for (int w = 1; w < kJoinWaves; ++w) sum[e] += part[w][e * 64 + lane];
            finish<VEC>(z, dtable + (size_t)key * z.E + col, left, sum);
        }
        __syncthreads();
    }
}

// Where things lie in the workspace.
struct Plan {
    bool few;
    int passes, tiles, run, stretches;
    size_t keys[2], order[2], counts, list, left_over, bytes;
};
// Short stretches where there are few positions, so that enough wavefronts share them (us of a call, 256 columns of fp32, words as frequent as in texts, stretches of 8 / of 32: n = 10000 29 / 38,
// 20000 39 / 48, 60000 55 / 57, 200000 104 / 86).
int run_of(int n) { return n <= 65536 ? 8 : kMostRun; }
Plan plan_of(int n, int E, int V)
{
    Plan p{};
    p.few = n <= kFew;
    p.tiles = ceil_div(n, kTile);
    while (p.passes < 4 && ((long long)V >> (kBits * p.passes)) > 0) ++p.passes;
    p.run = run_of(n);
    p.stretches = ceil_div(n, p.run);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    };
    for (int k = 0; k < (p.few ? 1 : 2); ++k) {
        p.keys[k] = take((size_t)n * 4);
        p.order[k] = take((size_t)n * 4);
    }
    p.counts = p.few ? 0 : take(((size_t)p.tiles + 1) * kDigits * 4);
    p.list = take(((size_t)p.stretches + 1) * 4);
    p.left_over = take((size_t)p.stretches * 2 * E * 4);
    p.bytes = at;
    return p;
}
int check(int n, int E, int V)
{
    if (n <= 0 || E <= 0 || V <= 0) return NSK_ERR_BAD_DESC;
    // (a launch has fewer than 2^32 threads: 64 for a stretch and 256 columns)
    const long long chunks = ((long long)E + kCols - 1) / kCols;
    if (n > 1 << 30 || chunks > 8192 || ((long long)n + run_of(n) - 1) / run_of(n) * chunks > 1LL << 25) return NSK_ERR_UNSUPPORTED;
    return NSK_OK;
}

}  // namespace
}  // namespace nsk

using namespace nsk;

extern "C" {

int nsk_embedding_scaled_fwd(int dtype, int n, int E, int V, const int *tokens, const void *table, float scale, int pad, void *out, void *stream)
{
    if (n <= 0 || E <= 0 || V <= 0 || !dtype_ok(dtype) || pad < -1 || pad >= V) return NSK_ERR_BAD_DESC;
    if (!tokens || !table || !out) return NSK_ERR_NULL;
    if (unaligned16(tokens) || unaligned16(table) || unaligned16(out)) return NSK_ERR_ALIGNMENT;
    const int V16 = dtype == NSK_BF16 ? 8 : 4, vectors = E % V16 ? E : E / V16;
    const long long blocks = ((long long)n * vectors + kThreads * kEach - 1) / (kThreads * kEach);
    if (blocks >= 1LL << 24 || vectors > 1 << 30) return NSK_ERR_UNSUPPORTED;     // (2^32 threads)
    const dim3 grid((unsigned)blocks);
    auto launch = [&](auto one, auto width) {
        typedef decltype(one) T;
        hipLaunchKernelGGL((embedding_scaled_fwd_kernel<T, decltype(width)::value>), grid, dim3(kThreads), 0, (hipStream_t)stream, tokens, (const T *)table, (T *)out, (long long)n, vectors,
                           make_div(vectors), V, pad, scale);
    };
    if (dtype == NSK_BF16) {
        if (E % 8) launch(bf16_t{}, std::integral_constant<int, 1>{});
        else launch(bf16_t{}, std::integral_constant<int, 8>{});
    } else {
        if (E % 4) launch(float{}, std::integral_constant<int, 1>{});
        else launch(float{}, std::integral_constant<int, 4>{});
    }
    return check_launch();
}

size_t nsk_embedding_scaled_bwd_workspace_bytes(int n, int E, int V) { return check(n, E, V) == NSK_OK ? plan_of(n, E, V).bytes : 0; }

int nsk_embedding_scaled_bwd(int dtype, int n, int E, int V, const int *tokens, const void *dout, float scale, int pad, float *dtable, int accumulate, void *workspace, size_t workspace_bytes,
                             void *stream)
{
    const int status = check(n, E, V);
    if (status == NSK_ERR_BAD_DESC || !dtype_ok(dtype) || pad < -1 || pad >= V || (accumulate != 0 && accumulate != 1)) return NSK_ERR_BAD_DESC;
    if (!tokens || !dout || !dtable) return NSK_ERR_NULL;
    if (unaligned16(tokens) || unaligned16(dout) || unaligned16(dtable) || unaligned16(workspace)) return NSK_ERR_ALIGNMENT;
    if (status != NSK_OK) return status;
    const Plan p = plan_of(n, E, V);
    if (!workspace || workspace_bytes < p.bytes) return NSK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    char *ws = (char *)workspace;
    // the table is filled beside the first step of the sort
    const size_t elements = accumulate ? 0 : (size_t)V * E;
    const unsigned filling = (unsigned)((elements + 16383) / 16384 < 1024 ? (elements + 16383) / 16384 : 1024);
    auto keys_at = [&](int k) { return (unsigned *)(ws + p.keys[k]); };
    auto order_at = [&](int k) { return (int *)(ws + p.order[k]); };
    int last = 0, *list = (int *)(ws + p.list);
    if (p.few) {
        const unsigned ranking = (unsigned)ceil_div(n, 64);
        auto rank = [&](auto narrow) {
            hipLaunchKernelGGL(rank_kernel<decltype(narrow)::value>, dim3(ranking + filling), dim3(kRankWaves * 64), 0, st, (const unsigned *)tokens, n, (unsigned)V, keys_at(0), order_at(0),
                               ranking, dtable, elements, list);
        };
        if (V < 65535) rank(std::true_type{});
        else rank(std::false_type{});
    } else {
        int *counts = (int *)(ws + p.counts);
        const unsigned *from = (const unsigned *)tokens;
        const int *from_order = nullptr;
        for (int k = 0; k < p.passes; ++k) {
            last = k & 1;
            hipLaunchKernelGGL(digits_kernel, dim3((unsigned)p.tiles + (k == 0 ? filling : 0)), dim3(kThreads), 0, st, from, n, (unsigned)V, kBits * k, p.tiles, counts, dtable, elements, list);
            hipLaunchKernelGGL(places_kernel, dim3(kDigits), dim3(64), 0, st, p.tiles, counts);
            hipLaunchKernelGGL(scatter_kernel, dim3((unsigned)p.tiles), dim3(kThreads), 0, st, from, from_order, n, (unsigned)V, kBits * k, p.tiles, counts, keys_at(last), order_at(last));
            from = keys_at(last);
            from_order = order_at(last);
        }
    }
    const unsigned *keys = keys_at(last);
    const int *order = order_at(last);
    const Runs z{n, E, (unsigned)V, pad < 0 ? (unsigned)V : (unsigned)pad, p.run, p.stretches, ceil_div(E, kCols), scale, accumulate};
    float *left_over = (float *)(ws + p.left_over);
    const dim3 grid((unsigned)(((long long)z.stretches * z.chunks + kWaves - 1) / kWaves)), joins((unsigned)(z.stretches < kJoinBlocks ? z.stretches : kJoinBlocks), (unsigned)z.chunks);
    auto launch = [&](auto one, auto vec) {
        typedef decltype(one) T;
        constexpr bool VEC = decltype(vec)::value;
        hipLaunchKernelGGL((runs_kernel<T, VEC>), grid, dim3(kThreads), 0, st, z, keys, order, (const T *)dout, dtable, left_over, list);
        hipLaunchKernelGGL(join_kernel<VEC>, joins, dim3(kJoinWaves * 64), 0, st, z, keys, dtable, left_over, list);
    };
    if (dtype == NSK_BF16) {
        if (E % 4) launch(bf16_t{}, std::false_type{});
        else launch(bf16_t{}, std::true_type{});
    } else {
        if (E % 4) launch(float{}, std::false_type{});
        else launch(float{}, std::true_type{});
    }
    return check_launch();
}

}  // extern "C"
