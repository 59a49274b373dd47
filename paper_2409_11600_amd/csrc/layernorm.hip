// Layer norm over the last axis with the residual add in front of it, forward and backward.
//   s = x + residual,  y = (s - mean) * invstd * gamma + beta
//   gh = dy * gamma, xh = (s - mean) * invstd:  dx = invstd * (gh - mean(gh) - xh * mean(gh * xh)) + dsum,
//   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
// Bound by memory: a row is read once and stays in the registers of the lanes that share it (2 to 1024 of them), so that the variance is the mean square of
// the differences from the mean itself, and the backward pass sums dy * xh and dy for the weights on the way.  us (TB/s of what has to move): 65536 x 768 bf16 with a
// residual 71 (5.7), backward 61 (4.9); 30011 x 1001 bf16 backward 39-44 (4.1-4.6), as fast as rows of 1000 or 1008; 10000 x 256 fp32 backward 10.2 and the joining
// launch 3.4; 300000 x 64 bf16 13.8 (5.6).  The backward pass has the next row of each lane on its way while one is worked on: its registers leave room for two
// wavefronts a SIMD, and those alone had 24 KB a compute unit in flight (65536 x 768 bf16 121 us without).
#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

// 16 bytes of a row.  Rows of odd lengths begin anywhere: this chip's loads and stores need no alignment beyond the element's.
template <typename T> struct Vec {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// The value of lane ^ O.
template <int O> __device__ inline float other(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    if constexpr (O == 1) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, (int)u, 0xb1, 0xf, 0xf, true));      // quad_perm 1,0,3,2
    else if constexpr (O < 16) return lane_xor<O>(v);
    else {
        // (of the two results of a swap with itself, each lane has its own value and the other's)
        const auto r = O == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return __builtin_bit_cast(float, (unsigned)((threadIdx.x & O) ? r[0] : r[1]));
    }
}
// Sum over the lanes whose numbers differ in bits FROM .. TO / 2, in all of them.
template <int FROM, int TO> __device__ inline float lanes_sum(float v)
{
    if constexpr (FROM < TO) return lanes_sum<FROM * 2, TO>(v + other<FROM>(v));
    else return v;
}
// Sums of M values over the LANES lanes that share a row.  Rows of several wavefronts exchange them through LDS, in two buffers that take turns: a wavefront
// writes one again only after a barrier that all reach behind their reads of it.
template <int LANES, int M> __device__ inline void row_sum(float (&v)[M], float (&part)[2][M][16], int &turn)
{
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = lanes_sum<1, (LANES < 64 ? LANES : 64)>(v[m]);
    if constexpr (LANES > 64) {
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int m = 0; m < M; ++m)
            if ((threadIdx.x & 63) == 0) part[turn][m][wave] = v[m];
        lds_barrier();
#pragma unroll
        for (int m = 0; m < M; ++m) {
            v[m] = 0.f;
#pragma unroll
            for (int w = 0; w < LANES / 64; ++w) v[m] += part[turn][m][w];
        }
        turn ^= 1;
    }
}

// What a lane holds of a row: K vectors, LANES apart, and one of the elements behind the last whole vector.
template <typename T, int LANES, int K> struct Share {
    static constexpr int V = Vec<T>::N, SIZE = K * V + 1;
    typedef typename Vec<T>::type vec;
    int at, vectors, tail;      // this lane's place; whole vectors of a row, elements behind them
    __device__ Share(int place, int C) : at(place), vectors(C / V), tail(C % V) {}
    __device__ bool has(int k) const { return k * LANES + at < vectors; }
    __device__ bool has_tail() const { return at < tail; }
    __device__ bool valid(int i) const { return i < K * V ? has(i / V) : has_tail(); }
    // A lane's part as it lies in memory, zeros where it has none; a later row's is fetched while one is worked on.
    struct Raw {
        vec v[K];
        T tail;
    };
    __device__ void fetch(const T *row, Raw &r) const
    {
#pragma unroll
        for (int k = 0; k < K; ++k) r.v[k] = has(k) ? *(const vec *)(row + (k * LANES + at) * V) : vec{};
        r.tail = has_tail() ? row[vectors * V + at] : (T)0.f;
    }
    static __device__ void unpack(const Raw &r, float (&v)[SIZE])
    {
#pragma unroll
        for (int i = 0; i < K * V; ++i) v[i] = (float)r.v[i / V][i % V];
        v[K * V] = (float)r.tail;
    }
    __device__ void load(const float *row, float (&v)[SIZE]) const
    {
        typedef float fvec __attribute__((ext_vector_type(V), aligned(4)));
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const fvec u = has(k) ? *(const fvec *)(row + (k * LANES + at) * V) : fvec{};
#pragma unroll
            for (int e = 0; e < V; ++e) v[k * V + e] = u[e];
        }
        v[K * V] = has_tail() ? row[vectors * V + at] : 0.f;
    }
    template <typename U> __device__ void store(U *row, const float (&v)[SIZE]) const
    {
        typedef U uvec __attribute__((ext_vector_type(V), aligned(sizeof(U))));
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (has(k)) {
                uvec u;
#pragma unroll
                for (int e = 0; e < V; ++e) u[e] = (U)v[k * V + e];
                *(uvec *)(row + (k * LANES + at) * V) = u;
            }
        if (has_tail()) row[vectors * V + at] = (U)v[K * V];
    }
};

template <typename T, int LANES, int K>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void layernorm_fwd_kernel(const T *x, const T *residual, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                                  T *sum, T *__restrict__ y, float *__restrict__ save_mean, float *__restrict__ save_invstd,
                                                                                  long long rows, int C, float eps)
{
    constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    __shared__ float part[2][1][16];
    int turn = 0;
    typedef Share<T, LANES, K> S;
    const S s(threadIdx.x % LANES, C);
    float g[S::SIZE], b[S::SIZE];
    if (gamma) s.load(gamma, g);
    else
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) g[i] = 1.f;
    if (beta) s.load(beta, b);
    else
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) b[i] = 0.f;
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < rows; r0 += (long long)gridDim.x * ROWS) {
        const long long row = r0 + threadIdx.x / LANES;
        if (row >= rows) break;         // (rows of several wavefronts: one a block, none left for any)
        const size_t at = (size_t)row * C;
        float v[S::SIZE], t[1] = {0.f};
        typename S::Raw raw, more;
        s.fetch(x + at, raw);
        if (residual) s.fetch(residual + at, more);
        S::unpack(raw, v);
        if (residual) {
            float w[S::SIZE];
            S::unpack(more, w);
#pragma unroll
            for (int i = 0; i < S::SIZE; ++i) v[i] = (float)(T)(v[i] + w[i]);
            if (sum) s.store(sum + at, v);
        }
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) t[0] += v[i];
        row_sum<LANES>(t, part, turn);
        const float mean = t[0] / (float)C;
        t[0] = 0.f;
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) {
            v[i] -= mean;
            t[0] += s.valid(i) ? v[i] * v[i] : 0.f;
        }
        row_sum<LANES>(t, part, turn);
        const float invstd = 1.f / sqrtf(t[0] / (float)C + eps);
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) v[i] = v[i] * invstd * g[i] + b[i];
        s.store(y + at, v);
        if (s.at == 0) {
            if (save_mean) save_mean[row] = mean;
            if (save_invstd) save_invstd[row] = invstd;
        }
    }
}

// dx of the rows of a block, and its sums of dy * xh and dy into partial[0 / 1][block][C] (PARAMS).
template <typename T, int LANES, int K, bool PARAMS>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void layernorm_bwd_kernel(const T *__restrict__ sum, const T *__restrict__ dy, const T *dsum,
                                                                                  const float *__restrict__ gamma, const float *__restrict__ save_mean,
                                                                                  const float *__restrict__ save_invstd, T *dx, float *__restrict__ partial, long long rows, int C)
{
    constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    __shared__ float part[2][2][16];
    int turn = 0;
    typedef Share<T, LANES, K> S;
    const S s(threadIdx.x % LANES, C);
    float g[S::SIZE], dg[S::SIZE], db[S::SIZE];
    if (gamma) s.load(gamma, g);
    else
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) g[i] = 1.f;
#pragma unroll
    for (int i = 0; i < S::SIZE; ++i) dg[i] = db[i] = 0.f;
    const float over = 1.f / (float)C;
    const long long step = (long long)gridDim.x * ROWS;
    typename S::Raw rs{}, rd{}, ru{};
    float mean = 0.f, invstd = 0.f;
    auto fetch = [&](long long row) {
        const size_t at = (size_t)row * C;
        mean = save_mean[row];
        invstd = save_invstd[row];
        s.fetch(sum + at, rs);
        s.fetch(dy + at, rd);
        if (dsum) s.fetch(dsum + at, ru);
    };
    long long row = (long long)blockIdx.x * ROWS + threadIdx.x / LANES;
    if (row < rows) fetch(row);
    for (; row < rows; row += step) {       // (rows of several wavefronts: one a block, the same for all)
        float v[S::SIZE], d[S::SIZE], u[S::SIZE], t[2] = {0.f, 0.f};
        S::unpack(rs, v);
        S::unpack(rd, d);
        S::unpack(ru, u);
        const float m = mean, inv = invstd;
        if (row + step < rows) fetch(row + step);
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) {
            v[i] = (v[i] - m) * (s.valid(i) ? inv : 0.f);       // (where the lane has nothing: 0, as d is; the product with a large mean could be infinite)
            if (PARAMS) {
                dg[i] += d[i] * v[i];
                db[i] += d[i];
            }
            d[i] *= g[i];
            t[0] += d[i];
            t[1] += d[i] * v[i];
        }
        row_sum<LANES>(t, part, turn);
        const float a = t[0] * over, b = t[1] * over;
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) v[i] = inv * (d[i] - a - v[i] * b);
        if (dsum)
#pragma unroll
            for (int i = 0; i < S::SIZE; ++i) v[i] += u[i];
        s.store(dx + (size_t)row * C, v);
    }
    if constexpr (PARAMS) {
        float *const p = partial + (size_t)blockIdx.x * C, *const q = p + (size_t)gridDim.x * C;
        if constexpr (ROWS > 1) {
            // lanes of the block's other rows with the same columns: within a wavefront first, then wavefront by wavefront in LDS
#pragma unroll
            for (int i = 0; i < S::SIZE; ++i) {
                dg[i] = lanes_sum<LANES, 64>(dg[i]);
                db[i] = lanes_sum<LANES, 64>(db[i]);
            }
            extern __shared__ float sums[];     // [2][C]
            for (int w = 0; w < 4; ++w) {
                __syncthreads();
                if ((int)threadIdx.x >> 6 == w && (threadIdx.x & 63) < LANES) {
                    auto add = [&](int c, int i) {
                        sums[c] = w ? sums[c] + dg[i] : dg[i];
                        sums[C + c] = w ? sums[C + c] + db[i] : db[i];
                    };
#pragma unroll
                    for (int i = 0; i < K * S::V; ++i)
                        if (s.has(i / S::V)) add((i / S::V * LANES + s.at) * S::V + i % S::V, i);
                    if (s.has_tail()) add(s.vectors * S::V + s.at, K * S::V);
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < C; c += THREADS) {
                p[c] = sums[c];
                q[c] = sums[C + c];
            }
        } else {
            s.store(p, dg);
            s.store(q, db);
        }
    }
}

// Rows that no block holds in its registers: read again for every pass, by 1024 threads a row.
template <typename T>
__global__ __launch_bounds__(1024) void layernorm_fwd_wide_kernel(const T *x, const T *residual, const float *__restrict__ gamma, const float *__restrict__ beta, T *sum,
                                                                  T *__restrict__ y, float *__restrict__ save_mean, float *__restrict__ save_invstd, long long rows, int C, float eps)
{
    __shared__ float part[2][1][16];
    int turn = 0;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const size_t at = (size_t)row * C;
        // (a thread reads the sum that it wrote itself; where there is no place for it, it is made again)
        auto first = [&](int c) { return residual ? (float)(T)((float)x[at + c] + (float)residual[at + c]) : (float)x[at + c]; };
        auto again = [&](int c) { return sum ? (float)sum[at + c] : first(c); };
        float t[1] = {0.f};
        for (int c = threadIdx.x; c < C; c += 1024) {
            const float s = first(c);
            if (sum) sum[at + c] = (T)s;
            t[0] += s;
        }
        row_sum<1024>(t, part, turn);
        const float mean = t[0] / (float)C;
        t[0] = 0.f;
        for (int c = threadIdx.x; c < C; c += 1024) {
            const float d = again(c) - mean;
            t[0] += d * d;
        }
        row_sum<1024>(t, part, turn);
        const float invstd = 1.f / sqrtf(t[0] / (float)C + eps);
        for (int c = threadIdx.x; c < C; c += 1024) y[at + c] = (T)((again(c) - mean) * invstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f));
        if (threadIdx.x == 0) {
            if (save_mean) save_mean[row] = mean;
            if (save_invstd) save_invstd[row] = invstd;
        }
    }
}
template <typename T>
__global__ __launch_bounds__(1024) void layernorm_dx_wide_kernel(const T *__restrict__ s, const T *__restrict__ dy, const T *dsum, const float *__restrict__ gamma,
                                                                 const float *__restrict__ save_mean, const float *__restrict__ save_invstd, T *dx, long long rows, int C)
{
    __shared__ float part[2][2][16];
    int turn = 0;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const size_t at = (size_t)row * C;
        const float mean = save_mean[row], invstd = save_invstd[row];
        float t[2] = {0.f, 0.f};
        for (int c = threadIdx.x; c < C; c += 1024) {
            const float gh = (float)dy[at + c] * (gamma ? gamma[c] : 1.f);
            t[0] += gh;
            t[1] += gh * (((float)s[at + c] - mean) * invstd);
        }
        row_sum<1024>(t, part, turn);
        const float a = t[0] / (float)C, b = t[1] / (float)C;
        for (int c = threadIdx.x; c < C; c += 1024) {
            const float gh = (float)dy[at + c] * (gamma ? gamma[c] : 1.f), xh = ((float)s[at + c] - mean) * invstd;
            dx[at + c] = (T)(invstd * (gh - a - xh * b) + (dsum ? (float)dsum[at + c] : 0.f));
        }
    }
}
template <typename T>
__global__ __launch_bounds__(256) void layernorm_dparam_wide_kernel(const T *__restrict__ s, const T *__restrict__ dy, const float *__restrict__ save_mean,
                                                                    const float *__restrict__ save_invstd, float *__restrict__ partial, long long rows, int C)
{
    const int c = blockIdx.y * 256 + threadIdx.x;
    if (c >= C) return;
    float a = 0.f, b = 0.f;
#pragma unroll 4
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const float d = (float)dy[(size_t)r * C + c];
        a += d * (((float)s[(size_t)r * C + c] - save_mean[r]) * save_invstd[r]);
        b += d;
    }
    partial[(size_t)blockIdx.x * C + c] = a;
    partial[(size_t)(gridDim.x + blockIdx.x) * C + c] = b;
}

// The blocks' sums: 32 columns a block, 32 threads a column that take every 32nd block's, joined in a fixed order.
__global__ __launch_bounds__(1024) void layernorm_dparam_final_kernel(const float *__restrict__ partial, float *__restrict__ dgamma, float *__restrict__ dbeta, int shares, int C,
                                                                      int accumulate)
{
    __shared__ double part[32][33];
    const int column = threadIdx.x % 32, k0 = threadIdx.x / 32, c = blockIdx.x * 32 + column;
    float *out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    double t = 0.0;
    if (c < C)
#pragma unroll 8
        for (int k = k0; k < shares; k += 32) t += (double)partial[((size_t)blockIdx.y * shares + k) * C + c];
    part[k0][column] = t;
    __syncthreads();
    if (k0 == 0 && c < C) {
        for (int k = 1; k < 32; ++k) t += part[k][column];
        out[c] = (float)(accumulate ? (double)out[c] + t : t);
    }
}

// Lanes that share a row, and vectors of each: as many lanes as there are vectors up to a wavefront, then two vectors a lane, then more wavefronts, whose sums go through LDS.
// us forward with a residual / backward with dsum, otherwise in brackets: 20000 x 768 bf16 64 lanes of two vectors 26 / 33 (256 of one 33 / 43); 8000 x 1500 256 of one 20 / 25
// (64 of four 21 / 41, whose registers leave one or two wavefronts a SIMD); 4000 x 3000 256 of two 20 / 26 (1024 of one 35 / 29), 4000 x 4096 27 / 33 (36 / 30); 2000 x 6000 1024 of one 23 / 24
// (256 of four 21 / 35), 2000 x 8192 30 / 32 (28 / 41).
struct Plan {
    int lanes, k;       // lanes 0: the kernels that hold nothing
};
Plan plan_of(const nsk_layernorm_desc_t &d)
{
    const int v = d.dtype == NSK_BF16 ? 8 : 4, vectors = d.C / v;
    // (an element behind the last vector has a lane of its own: there are 7 of them at most)
    for (int lanes = d.C % v ? 8 : 2; lanes <= 64; lanes *= 2)
        if (vectors <= lanes) return {lanes, 1};
    if (vectors <= 128) return {64, 2};
    if (vectors <= 256) return {256, 1};
    if (vectors <= 512) return {256, 2};
    if (vectors <= 1024) return {1024, 1};
    if (vectors <= 2048) return {1024, 2};
    return {0, 0};
}
// The pass that makes dx also makes the sums for gamma and beta, unless their registers would not fit: two vectors of each of 1024 lanes, which in bf16 are 16 elements and spill 125
// registers, in fp32 8 and 6.  us with it / with a pass of its own for the sums: bf16, dsum, 2048 x 12000 150 / 62, 2048 x 16384 167 / 83; fp32, dsum, 4000 x 6000 79 / 113, 4000 x 8192
// 109 / 154, 2000 x 5000 36 / 48, 300 x 8192 16 / 21, 4000 x 6000 without dsum 59 / 99.
constexpr bool on_the_way(Plan p, size_t element_bytes) { return p.lanes > 0 && !(p.lanes == 1024 && p.k == 2 && element_bytes == 2); }
int rows_a_block(const Plan &p) { return p.lanes == 0 || p.lanes >= 256 ? 1 : 256 / p.lanes; }
// Blocks of the backward pass, each with sums of its own; 512, two a compute unit, are what its registers leave room for at once.  us with dsum, 256 / 512 / 1024 of them:
// 10000 x 256 fp32 13.4, 13.0, 13.6; 65536 x 768 bf16 86, 79, 87; 65536 x 768 fp32 225, 150, 157; 300000 x 64 bf16 42, 34, 37.
int shares_of(const nsk_layernorm_desc_t &d)
{
    const Plan p = plan_of(d);
    const long long blocks = (d.rows + rows_a_block(p) - 1) / rows_a_block(p), most = p.lanes == 1024 || p.lanes == 0 ? 256 : 512;
    return (int)(blocks < most ? blocks : most);
}

int check(const nsk_layernorm_desc_t *d)
{
    if (!d) return NSK_ERR_NULL;
    // (rows * C: a byte offset of it has to fit a pointer)
    if (d->rows <= 0 || d->C <= 0 || (d->dtype != NSK_F32 && d->dtype != NSK_BF16) || d->rows > (1LL << 60) / d->C) return NSK_ERR_BAD_DESC;
    if (d->C > 1 << 24) return NSK_ERR_UNSUPPORTED;         // (the launch over columns)
    return NSK_OK;
}

// f(LANES, K) of the plan, as constants.
template <typename F> void with(const Plan &p, F &&f)
{
#define NSK_CASE(L, N)                                                                   \
    if (p.lanes == L && p.k == N) f(std::integral_constant<int, L>{}, std::integral_constant<int, N>{});
    NSK_CASE(2, 1) NSK_CASE(4, 1) NSK_CASE(8, 1) NSK_CASE(16, 1) NSK_CASE(32, 1) NSK_CASE(64, 1) NSK_CASE(64, 2) NSK_CASE(256, 1) NSK_CASE(256, 2) NSK_CASE(1024, 1) NSK_CASE(1024, 2)
#undef NSK_CASE
}

}  // namespace
}  // namespace nsk

using namespace nsk;

extern "C" {

size_t nsk_layernorm_bwd_workspace_bytes(const nsk_layernorm_desc_t *desc)
{
    return check(desc) == NSK_OK ? (size_t)2 * shares_of(*desc) * desc->C * sizeof(float) : 0;
}

int nsk_layernorm_fwd(const nsk_layernorm_desc_t *desc, const void *x, const void *residual, const float *gamma, const float *beta, void *sum, void *y,
                      float *save_mean, float *save_invstd, void *stream)
{
    const int status = check(desc);
    if (status != NSK_OK) return status;
    if (!(desc->eps > 0.f) || (sum && !residual)) return NSK_ERR_BAD_DESC;
    if (!x || !y) return NSK_ERR_NULL;
    if (unaligned16(x) || unaligned16(residual) || unaligned16(gamma) || unaligned16(beta) || unaligned16(sum) || unaligned16(y) || unaligned16(save_mean) ||
        unaligned16(save_invstd))
        return NSK_ERR_ALIGNMENT;
    const Plan p = plan_of(*desc);
    // (a row or a few for every block: 65536 x 768 bf16 with a residual 70 us, 78 with 2048 blocks that go round, 74 with 512; blocks of a row of 1024 lanes, whose gamma and beta are
    // long, go round: 1000 x 16000 bf16 30 with 512 blocks, 32 with one a row)
    const long long need = (desc->rows + rows_a_block(p) - 1) / rows_a_block(p), most = p.lanes == 0 || p.lanes == 1024 ? 512 : 1 << 20;
    const dim3 grid((unsigned)(need < most ? need : most));
    hipStream_t st = (hipStream_t)stream;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (p.lanes == 0)
            hipLaunchKernelGGL(layernorm_fwd_wide_kernel<T>, grid, dim3(1024), 0, st, (const T *)x, (const T *)residual, gamma, beta, (T *)sum, (T *)y, save_mean, save_invstd,
                               desc->rows, desc->C, desc->eps);
        with(p, [&](auto lanes, auto k) {
            constexpr int L = decltype(lanes)::value, N = decltype(k)::value;
            hipLaunchKernelGGL((layernorm_fwd_kernel<T, L, N>), grid, dim3(L > 256 ? L : 256), 0, st, (const T *)x, (const T *)residual, gamma, beta, (T *)sum, (T *)y, save_mean,
                               save_invstd, desc->rows, desc->C, desc->eps);
        });
    };
    if (desc->dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    return check_launch();
}

int nsk_layernorm_bwd(const nsk_layernorm_desc_t *desc, const void *s, const void *dy, const void *dsum, const float *gamma, const float *save_mean,
                      const float *save_invstd, void *dx, float *dgamma, float *dbeta, int accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    const int status = check(desc);
    if (status != NSK_OK) return status;
    if (!s || !dy || !save_mean || !save_invstd || !dx) return NSK_ERR_NULL;
    if (unaligned16(s) || unaligned16(dy) || unaligned16(dsum) || unaligned16(gamma) || unaligned16(save_mean) || unaligned16(save_invstd) ||
        unaligned16(dx) || unaligned16(dgamma) || unaligned16(dbeta) || unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    const bool params = dgamma || dbeta;
    if (params && (!workspace || workspace_bytes < nsk_layernorm_bwd_workspace_bytes(desc))) return NSK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int C = desc->C, shares = shares_of(*desc);
    const Plan p = plan_of(*desc);
    const dim3 grid((unsigned)shares);
    float *const partial = (float *)workspace;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (params && !on_the_way(p, sizeof(T)))
            hipLaunchKernelGGL(layernorm_dparam_wide_kernel<T>, dim3((unsigned)shares, (unsigned)ceil_div(C, 256)), dim3(256), 0, st, (const T *)s, (const T *)dy, save_mean, save_invstd,
                               partial, desc->rows, C);
        if (p.lanes == 0)
            hipLaunchKernelGGL(layernorm_dx_wide_kernel<T>, dim3((unsigned)(desc->rows < 512 ? desc->rows : 512)), dim3(1024), 0, st, (const T *)s, (const T *)dy, (const T *)dsum, gamma,
                               save_mean, save_invstd, (T *)dx, desc->rows, C);
        with(p, [&](auto lanes, auto k) {
            constexpr int L = decltype(lanes)::value, N = decltype(k)::value;
            const dim3 block(L > 256 ? L : 256);
            constexpr bool ON_THE_WAY = on_the_way({L, N}, sizeof(T));
            if (params && ON_THE_WAY)
                hipLaunchKernelGGL((layernorm_bwd_kernel<T, L, N, ON_THE_WAY>), grid, block, L < 256 ? 2 * C * sizeof(float) : 0, st, (const T *)s, (const T *)dy, (const T *)dsum, gamma, save_mean,
                                   save_invstd, (T *)dx, partial, desc->rows, C);
            else
                hipLaunchKernelGGL((layernorm_bwd_kernel<T, L, N, false>), grid, block, 0, st, (const T *)s, (const T *)dy, (const T *)dsum, gamma, save_mean, save_invstd, (T *)dx, partial,
                                   desc->rows, C);
        });
    };
    if (desc->dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    if (params)
        hipLaunchKernelGGL(layernorm_dparam_final_kernel, dim3((unsigned)ceil_div(C, 32), 2), dim3(1024), 0, st, partial, dgamma, dbeta, shares, C, accumulate);
    return check_launch();
}

}  // extern "C"
