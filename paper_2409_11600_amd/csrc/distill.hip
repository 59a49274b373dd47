// Distillation: the loss of a row of logits z against the M largest logits t of a teacher, and its gradient.
//   p = softmax(t / tau) over the places that there are, q = softmax(z / tau) over all K,
//   l = tau^2 sum_m p_m (log p_m - log q[index_m]),   d l / d z_k = tau (q_k - sum of p_m over the places with index k).
// Both directions read each logit once, the gradient writes each once; the teacher's part is M values a row.
#include <math.h>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

constexpr int kThreads = 256;
constexpr int kMost = NSK_DISTILL_MOST;
constexpr float kLog2e = 1.44269504088896341f;

struct Sizes {
    int N, K, M;
    int pieces, piece;      // a row is taken by so many blocks, each with so many columns (a multiple of 16)
    int bits;               // of a table with room for twice M
    long long ld;
    float tau, inv;         // 1 / tau
};

// exp((x - top) / tau): the difference first, so that the rounding of the product counts for values far below the largest alone.
__device__ __forceinline__ float exp_under(float x, float top, float by) { return __builtin_amdgcn_exp2f((x - top) * by); }

// A maximum, and a sum of exponentials relative to it.  A maximum of -infinity (nothing yet) counts as 0, so that no difference of infinities is made.
struct Soft {
    float top, sum;
};
__device__ __forceinline__ float finite_top(float t) { return t == -INFINITY ? 0.f : t; }
__device__ __forceinline__ Soft join(Soft a, Soft b, float by)
{
    const float top = fmaxf(a.top, b.top), f = finite_top(top);
    return {top, a.sum * exp_under(a.top, f, by) + b.sum * exp_under(b.top, f, by)};
}
__device__ __forceinline__ Soft join_lanes(Soft s, float by)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s = join(s, {__shfl_xor(s.top, o, 64), __shfl_xor(s.sum, o, 64)}, by);
    return s;
}
__device__ __forceinline__ float sum_lanes(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ Soft join_block(Soft s, float by, float (&part)[2][kThreads / 64])
{
    s = join_lanes(s, by);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        part[0][threadIdx.x >> 6] = s.top;
        part[1][threadIdx.x >> 6] = s.sum;
    }
    __syncthreads();
    s = {part[0][0], part[1][0]};
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) s = join(s, {part[0][w], part[1][w]}, by);
    return s;
}

// Vectors of 16 bytes of a row that may begin anywhere: head elements in front of the first whole vector, body vectors, the rest.
template <typename T> struct Span {
    static constexpr int V = 16 / sizeof(T);
    int head, vectors, tail;        // tail: the first element behind the vectors
};
template <typename T> __device__ __forceinline__ Span<T> span_of(const T *row, int n)
{
    constexpr int V = Span<T>::V;
    int head = (int)((-(unsigned long long)(uintptr_t)row & 15) / sizeof(T));
    head = head < n ? head : n;
    const int vectors = (n - head) / V;
    return {head, vectors, head + vectors * V};
}
template <typename T> struct Vec {
    T v[Span<T>::V];
};
template <typename T> __device__ __forceinline__ Vec<T> load_vec(const T *p)
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(Vec<T>, *(const u32x4 *)p);
}
template <typename T> __device__ __forceinline__ void store_vec(T *p, const Vec<T> &v)
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4 *)p);
}

// (maximum, sum) over n logits by the whole block.  Each lane keeps its own pair; the sum is rescaled once a group of vectors.
template <typename T> __device__ Soft soft_row(const T *row, int n, float by, float (&part)[2][kThreads / 64])
{
    constexpr int V = Span<T>::V, U = 4;
    const Span<T> s = span_of(row, n);
    Soft a{-INFINITY, 0.f};
    auto one = [&](float x) {
        const float top = fmaxf(a.top, x), f = finite_top(top);
        a = {top, a.sum * exp_under(a.top, f, by) + exp_under(x, f, by)};
    };
    if ((int)threadIdx.x < s.head) one((float)row[threadIdx.x]);
    const T *body = row + s.head;
    int i = threadIdx.x;
    for (; i + (U - 1) * kThreads < s.vectors; i += U * kThreads) {
        Vec<T> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load_vec(body + (size_t)(i + u * kThreads) * V);
        float top = a.top;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) top = fmaxf(top, (float)x[u].v[e]);
        const float f = finite_top(top);
        float sum[4] = {a.sum * exp_under(a.top, f, by), 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e & 3] += exp_under((float)x[u].v[e], f, by);
        a = {top, (sum[0] + sum[1]) + (sum[2] + sum[3])};
    }
    for (; i < s.vectors; i += kThreads) {
        const Vec<T> x = load_vec(body + (size_t)i * V);
        float top = a.top;
#pragma unroll
        for (int e = 0; e < V; ++e) top = fmaxf(top, (float)x.v[e]);
        const float f = finite_top(top);
        float sum = a.sum * exp_under(a.top, f, by);
#pragma unroll
        for (int e = 0; e < V; ++e) sum += exp_under((float)x.v[e], f, by);
        a = {top, sum};
    }
    if (s.tail + (int)threadIdx.x < n) one((float)row[s.tail + threadIdx.x]);
    return join_block(a, by, part);
}

// The teacher's side of a row: (maximum, sum) of the places that there are, and whether any is, or one is out of range.
struct Teacher {
    Soft s;
    bool any, bad;
};
__device__ Teacher teacher_of(const Sizes &z, const int *index, const float *t, float by, float (&part)[2][kThreads / 64])
{
    Soft a{-INFINITY, 0.f};
    bool any = false, bad = false;
    for (int m = threadIdx.x; m < z.M; m += kThreads) {
        const int k = index[m];
        if (k < 0) continue;
        any = true;
        bad |= k >= z.K;
        a = join(a, {t[m], 1.f}, by);
    }
    any = __syncthreads_or(any);
    bad = __syncthreads_or(bad);
    return {join_block(a, by, part), any, bad};
}
// p of a place (0 for one of -infinity), and its logarithm.
__device__ __forceinline__ float p_of(float t, Soft s, float by) { return exp_under(t, s.top, by) / s.sum; }

// What a row's sums make of it: its loss, and what the backward pass reads.
template <typename T>
__device__ void finish_row(const Sizes &z, long long n, Soft q, const T *row, const int *index, const float *t, const Teacher &teacher, float by, float *per_row,
                           float (&part)[2][kThreads / 64])
{
    const float lq = logf(q.sum), lp = logf(teacher.s.sum);
    float loss = 0.f;
    if (!teacher.bad)
        for (int m = threadIdx.x; m < z.M; m += kThreads) {
            const int k = index[m];
            if (k < 0) continue;
            const float p = p_of(t[m], teacher.s, by);
            if (p != 0.f) loss += p * (((t[m] - teacher.s.top) * z.inv - lp) - (((float)row[k] - q.top) * z.inv - lq));
        }
    loss = sum_lanes(loss);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[0][threadIdx.x >> 6] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        loss = (part[0][0] + part[0][1]) + (part[0][2] + part[0][3]);
        per_row[n] = teacher.bad ? NAN : z.tau * z.tau * loss;
    }
}
// (The largest logit / tau is rounded, by far more than a difference of logits where all are large: the sum is that of what the backward pass computes, relative to the rounded value.)
__device__ void save_row(const Sizes &z, long long n, Soft q, float *saved)
{
    if (threadIdx.x == 0) {
        const float held = q.top * z.inv;
        saved[2 * n] = q.sum == q.sum ? held : NAN;
        saved[2 * n + 1] = q.top == -INFINITY ? NAN : 1.f / (q.sum * expf(fmaf(q.top, z.inv, -held)));
    }
}

// A row (or a piece of it) a block.  With several pieces a row, their sums go to `partial` and distill_join_kernel finishes the rows.  Bound by memory where rows are many: 10000 x 32768 in
// bf16 take 117 us, 5.6 TB/s (6.4 with what the last-level cache has kept), the vector unit busy three quarters of the time with an exponential an element; 50 x 1000 take 5.4, a chain of one
// load of the row, three joins over the block and the logits of the places.
template <typename T>
__global__ __launch_bounds__(kThreads) void distill_fwd_kernel(Sizes z, const T *__restrict__ logits, const int *__restrict__ index, const float *__restrict__ t,
                                                               const float *__restrict__ weights, float *__restrict__ per_row, float *__restrict__ saved, float *__restrict__ partial)
{
    __shared__ float part[2][kThreads / 64];
    const long long n = blockIdx.x;
    const int p = blockIdx.y;
    if (weights && weights[n] == 0.f) {
        if (p == 0 && threadIdx.x == 0) {
            per_row[n] = 0.f;
            saved[2 * n] = 0.f;
            saved[2 * n + 1] = 0.f;
        }
        return;
    }
    const float by = kLog2e * z.inv;
    const T *row = logits + n * z.ld;
    const int from = p * z.piece, count = z.K - from < z.piece ? z.K - from : z.piece;
    const Soft q = soft_row(row + from, count, by, part);
    if (z.pieces > 1) {
        if (threadIdx.x == 0) {
            partial[2 * (n * z.pieces + p)] = q.top;
            partial[2 * (n * z.pieces + p) + 1] = q.sum;
        }
        return;
    }
    const int *at = index + n * z.M;
    const float *tr = t + n * z.M;
    const Teacher teacher = teacher_of(z, at, tr, by, part);
    save_row(z, n, q, saved);
    finish_row(z, n, q, row, at, tr, teacher, by, per_row, part);
}
template <typename T>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(Sizes z, const T *__restrict__ logits, const int *__restrict__ index, const float *__restrict__ t,
                                                                const float *__restrict__ weights, float *__restrict__ per_row, float *__restrict__ saved, const float *__restrict__ partial)
{
    __shared__ float part[2][kThreads / 64];
    const long long n = blockIdx.x;
    if (weights && weights[n] == 0.f) return;
    const float by = kLog2e * z.inv;
    Soft q{-INFINITY, 0.f};
    for (int p = threadIdx.x; p < z.pieces; p += kThreads) q = join(q, {partial[2 * (n * z.pieces + p)], partial[2 * (n * z.pieces + p) + 1]}, by);
    q = join_block(q, by, part);
    const int *at = index + n * z.M;
    const float *tr = t + n * z.M;
    const Teacher teacher = teacher_of(z, at, tr, by, part);
    save_row(z, n, q, saved);
    finish_row(z, n, q, logits + n * z.ld, at, tr, teacher, by, per_row, part);
}

// Sums of w_n l_n and of w_n: a block for all rows, or kSums blocks and one that joins what they leave.  In 64 bits, in a fixed order.  2.5 us for 50 rows, 7.5 for 10000.
constexpr int kSums = 64, kRowsOfOne = 1 << 16;
__global__ __launch_bounds__(1024) void distill_loss_kernel(int N, const float *__restrict__ weights, const float *__restrict__ per_row, const double *__restrict__ joined, double *__restrict__ left,
                                                            float *__restrict__ loss, float *__restrict__ saved)
{
    __shared__ double part[2][16];
    double sum = 0., total = 0.;
    if (joined) {
        if (threadIdx.x < kSums) {
            sum = joined[2 * threadIdx.x];
            total = joined[2 * threadIdx.x + 1];
        }
    } else {
        const int each = (N + (int)gridDim.x - 1) / (int)gridDim.x, from = (int)blockIdx.x * each, to = N - from < each ? N : from + each;
        for (int n = from + (int)threadIdx.x; n < to; n += 1024) {
            const double w = weights ? (double)weights[n] : 1.;
            if (w != 0.) sum += w * (double)per_row[n];
            total += w;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o, 64);
        total += __shfl_xor(total, o, 64);
    }
    if ((threadIdx.x & 63) == 0) {
        part[0][threadIdx.x >> 6] = sum;
        part[1][threadIdx.x >> 6] = total;
    }
    __syncthreads();
    if (threadIdx.x) return;
    sum = total = 0.;
    for (int w = 0; w < 16; ++w) {
        sum += part[0][w];
        total += part[1][w];
    }
    if (left) {
        left[2 * blockIdx.x] = sum;
        left[2 * blockIdx.x + 1] = total;
        return;
    }
    loss[0] = total != 0. ? (float)(sum / total) : 0.f;
    saved[2 * (long long)N] = (float)total;
    saved[2 * (long long)N + 1] = total != 0. ? (float)(1. / total) : 0.f;
}

// A row (or a piece of it) a block.  Bound by memory: 5003 x 50001 in fp32, seven tenths of the rows with a weight, 395 us, 4.4 TB/s of reads and writes mixed (four vectors at a
// time and stores that are not kept in the caches: 5000 x 50000 in fp32, all rows, 438 us, 4.6 TB/s; two at a time 444, kept 470, both 482).  All columns are written as if the teacher had no places; the columns of its places are then written again, each by one lane
// with the sum of its places' p, from the logit (and the gradient that is added to) read before: so each is rounded once, and a place costs nothing on the way.  Which places share an index
// a hash table in LDS finds, the memory's passes running beside it; those that do look for each other one by one, so that the sum is in the places' order (comparing all places with all,
// as at first, took 321 us a call where M = 1024, N = 512, K = 32000, bf16, now 23; M = 64: 18 and 14).
constexpr int kShared = 1 << 30;        // with an index: another place has it too
template <typename T, bool ADD>
__global__ __launch_bounds__(kThreads) void distill_bwd_kernel(Sizes z, const T *logits, const int *__restrict__ index, const float *__restrict__ t, const float *__restrict__ weights,
                                                               const float *__restrict__ saved, float dloss, T *dlogits)
{
    constexpr int V = Span<T>::V, U = 4;
    extern __shared__ float lds[];
    __shared__ float part[2][kThreads / 64];
    float *p_at = lds, *z_at = lds + z.M, *old_at = lds + 2 * z.M;
    int *k_at = (int *)(lds + 3 * z.M), *table = k_at + z.M;
    const long long n = blockIdx.x;
    const int from = blockIdx.y * z.piece, count = z.K - from < z.piece ? z.K - from : z.piece;
    const T *row = logits + n * z.ld + from;
    T *out = dlogits + n * z.ld + from;
    const float by = kLog2e * z.inv, w = weights ? weights[n] : 1.f;
    const Span<T> s = span_of(out, count);
    bool none = w == 0.f;
    float c = 0.f;
    Teacher teacher{};
    if (!none) {
        const int *at = index + n * z.M;
        const float *tr = t + n * z.M;
        teacher = teacher_of(z, at, tr, by, part);
        none = !teacher.any;
        c = dloss * (w * saved[2 * (long long)z.N + 1]) * z.tau;         // (the row's share first: it is at most 1, where a weight and dloss may leave the range together)
        if (teacher.bad) c = NAN;
        if (!none) {
            for (int i = threadIdx.x; i < 1 << z.bits; i += kThreads) table[i] = -1;
            for (int m = threadIdx.x; m < z.M; m += kThreads) {
                const int k = at[m] < from || at[m] - from >= count ? -1 : at[m] - from;
                k_at[m] = k;
                if (k < 0) continue;
                p_at[m] = p_of(tr[m], teacher.s, by);
                z_at[m] = (float)row[k];
                if (ADD) old_at[m] = (float)out[k];
            }
        }
    }
    if (none) {
        if (ADD) return;
        if ((int)threadIdx.x < s.head) out[threadIdx.x] = (T)0.f;
        const Vec<T> zero{};
        for (int i = threadIdx.x; i < s.vectors; i += kThreads) store_vec(out + s.head + (size_t)i * V, zero);
        if (s.tail + (int)threadIdx.x < count) out[s.tail + threadIdx.x] = (T)0.f;
        return;
    }
    __syncthreads();
    for (int m = threadIdx.x; m < z.M; m += kThreads) {        // (the table has twice as many entries as there are places: one is free)
        const int k = k_at[m] & ~kShared;
        if (k_at[m] < 0) continue;
        for (unsigned e = (unsigned)k * 2654435769u >> (32 - z.bits);; e = (e + 1) & ((1u << z.bits) - 1)) {
            const int there = atomicCAS(&table[e], -1, m);
            if (there < 0) break;
            if ((k_at[there] & ~kShared) != k) continue;
            atomicOr(&k_at[there], kShared);
            atomicOr(&k_at[m], kShared);
            break;
        }
    }
    const float top = saved[2 * n], inv = saved[2 * n + 1] * c;
    auto gradient = [&](float x) { return __builtin_amdgcn_exp2f(fmaf(x, z.inv, -top) * kLog2e) * inv; };
    auto one = [&](int k) {
        const float g = gradient((float)row[k]);
        out[k] = (T)(ADD ? (float)out[k] + g : g);
    };
    if ((int)threadIdx.x < s.head) one(threadIdx.x);
    auto some = [&](const Vec<T> &x, const Vec<T> &old) {
        Vec<T> g;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float v = gradient((float)x.v[e]);
            g.v[e] = (T)(ADD ? (float)old.v[e] + v : v);
        }
        return g;
    };
    const T *in = row + s.head;         // (logits and gradient begin on 16 bytes and have rows of the same length: at the same place of a vector)
    T *body = out + s.head;
    int i = threadIdx.x;
    for (; i + (U - 1) * kThreads < s.vectors; i += U * kThreads) {
        Vec<T> x[U], old[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = load_vec(in + (size_t)(i + u * kThreads) * V);
            if (ADD) old[u] = load_vec(body + (size_t)(i + u * kThreads) * V);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) store_vec(body + (size_t)(i + u * kThreads) * V, some(x[u], old[u]));
    }
    for (; i < s.vectors; i += kThreads) {
        Vec<T> old{};
        if (ADD) old = load_vec(body + (size_t)i * V);
        store_vec(body + (size_t)i * V, some(load_vec(in + (size_t)i * V), old));
    }
    if (s.tail + (int)threadIdx.x < count) one(s.tail + threadIdx.x);
    __syncthreads();        // (what was written above is behind this barrier, also for other lanes' stores to the same columns)
    for (int m = threadIdx.x; m < z.M; m += kThreads) {
        const int own = k_at[m], k = own & ~kShared;
        if (own < 0) continue;
        float p = p_at[m];
        if (own & kShared) {
            bool first = true;
            p = 0.f;
            for (int j = 0; j < z.M; ++j) {
                const bool twin = k_at[j] == own;
                p += twin ? p_at[j] : 0.f;
                first &= !(twin && j < m);
            }
            if (!first) continue;
        }
        const float g = gradient(z_at[m]) - c * p;
        out[k] = (T)(ADD ? old_at[m] + g : g);
    }
}

int check(const nsk_distill_desc_t *desc, Sizes &z)
{
    if (!desc) return NSK_ERR_NULL;
    const nsk_distill_desc_t &d = *desc;
    if (d.N <= 0 || d.K <= 0 || d.M <= 0 || (d.dtype != NSK_F32 && d.dtype != NSK_BF16) || !(d.tau > 0.f) || isinf(d.tau) || isinf(1.f / d.tau)) return NSK_ERR_BAD_DESC;
    if (d.ld < 0 || (d.ld > 0 && d.N > 1 && d.ld < d.K) || d.ld > (1LL << 60) / d.N) return NSK_ERR_BAD_DESC;
    if (d.M > kMost || d.K > (1 << 30) || d.N > (1 << 23)) return NSK_ERR_UNSUPPORTED;
    z = {d.N, d.K, d.M, 1, 0, 1, d.ld ? d.ld : d.K, d.tau, 1.f / d.tau};
    while (1 << z.bits < 2 * d.M) ++z.bits;
    return NSK_OK;
}
// Few long rows are shared by several blocks.  Forwards that takes a launch more, which only rows of 65536 and more make up for; bf16, us of N x K, one block a row / pieces of 4096 and more:
// forwards 64 x 8192 9.3 / 12.5, 64 x 32768 10.9 / 12.0, 512 x 32768 14.4 / 18.0 (64 x 131072 13.3, 1 x 131072 11.4 with pieces, where one block alone would need 16 loads one after the other);
// backwards 8 x 32768 9.7 / 7.3, 64 x 8192 8.2 / 6.6, 256 x 32768 13.7 / 11.5, 512 x 32768 17.7 / 16.7.
constexpr int kLeast = 4096, kLongForward = 65536;
void cut(Sizes &z, bool forward)
{
    int pieces = 1;
    while ((!forward || z.K >= kLongForward) && pieces < 64 && (long long)z.N * pieces < 1024 && z.K / (2 * pieces) >= kLeast) pieces *= 2;
    z.piece = (ceil_div(z.K, pieces) + 15) / 16 * 16;
    z.pieces = ceil_div(z.K, z.piece);
}
size_t sums_at(const Sizes &z) { return z.pieces > 1 ? align_up((size_t)z.N * z.pieces * 2 * sizeof(float)) : 0; }
size_t workspace_of(const Sizes &z) { return sums_at(z) + (z.N > kRowsOfOne ? kSums * 2 * sizeof(double) : 0); }

}  // namespace
}  // namespace nsk

using namespace nsk;

extern "C" {

size_t nsk_distill_workspace_bytes(const nsk_distill_desc_t *desc)
{
    Sizes z;
    if (check(desc, z) != NSK_OK) return 0;
    cut(z, true);
    return workspace_of(z);
}

int nsk_distill_fwd(const nsk_distill_desc_t *desc, const void *logits, const int *top_index, const float *top_logits, const float *weights, float *per_row, float *loss, float *saved,
                    void *workspace, size_t workspace_bytes, void *stream)
{
    Sizes z;
    const int status = check(desc, z);
    if (status != NSK_OK) return status;
    if (!logits || !top_index || !top_logits || !per_row || !loss || !saved) return NSK_ERR_NULL;
    if (unaligned16(logits) || unaligned16(top_index) || unaligned16(top_logits) || unaligned16(weights) || unaligned16(per_row) || unaligned16(loss) || unaligned16(saved) ||
        unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    cut(z, true);
    if (workspace_of(z) && (!workspace || workspace_bytes < workspace_of(z))) return NSK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    float *partial = (float *)workspace;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        hipLaunchKernelGGL(distill_fwd_kernel<T>, dim3((unsigned)z.N, (unsigned)z.pieces), dim3(kThreads), 0, st, z, (const T *)logits, top_index, top_logits, weights, per_row, saved, partial);
        if (z.pieces > 1)
            hipLaunchKernelGGL(distill_join_kernel<T>, dim3((unsigned)z.N), dim3(kThreads), 0, st, z, (const T *)logits, top_index, top_logits, weights, per_row, saved, partial);
    };
    if (desc->dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    if (z.N > kRowsOfOne) {
        double *sums = (double *)((char *)workspace + sums_at(z));
        hipLaunchKernelGGL(distill_loss_kernel, dim3(kSums), dim3(1024), 0, st, z.N, weights, per_row, nullptr, sums, loss, saved);
        hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(1024), 0, st, z.N, weights, per_row, sums, nullptr, loss, saved);
    } else {
        hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(1024), 0, st, z.N, weights, per_row, nullptr, nullptr, loss, saved);
    }
    return check_launch();
}

int nsk_distill_bwd(const nsk_distill_desc_t *desc, const void *logits, const int *top_index, const float *top_logits, const float *weights, const float *saved, float dloss, void *dlogits,
                    int accumulate, void *stream)
{
    Sizes z;
    const int status = check(desc, z);
    if (status != NSK_OK) return status;
    if (accumulate != 0 && accumulate != 1) return NSK_ERR_BAD_DESC;
    if (!logits || !top_index || !top_logits || !saved || !dlogits) return NSK_ERR_NULL;
    if (unaligned16(logits) || unaligned16(top_index) || unaligned16(top_logits) || unaligned16(weights) || unaligned16(saved) || unaligned16(dlogits)) return NSK_ERR_ALIGNMENT;
    if (accumulate && logits == dlogits) return NSK_ERR_BAD_DESC;
    cut(z, false);
    const dim3 grid((unsigned)z.N, (unsigned)z.pieces);
    const size_t lds = ((size_t)z.M * 4 + ((size_t)1 << z.bits)) * 4;
    hipStream_t st = (hipStream_t)stream;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (accumulate)
            hipLaunchKernelGGL((distill_bwd_kernel<T, true>), grid, dim3(kThreads), lds, st, z, (const T *)logits, top_index, top_logits, weights, saved, dloss, (T *)dlogits);
        else
            hipLaunchKernelGGL((distill_bwd_kernel<T, false>), grid, dim3(kThreads), lds, st, z, (const T *)logits, top_index, top_logits, weights, saved, dloss, (T *)dlogits);
    };
    if (desc->dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    return check_launch();
}

}  // extern "C"
