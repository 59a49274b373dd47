// Layer norm over the last axis with the residual add in front of it, forward and backward.
//   s = x + residual,  y = (s - mean) * invstd * gamma + beta
//   gh = dy * gamma, xh = (s - mean) * invstd:  dx = invstd * (gh - mean(gh) - xh * mean(gh * xh)) + dsum,
//   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
// Bound by memory: a row is read once and stays in the registers of the lanes that share it (8 to 1024 of them), so that the variance is the mean square of
// the differences from the mean itself, and the backward pass sums dy * xh and dy for the weights on the way.
#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

// 16 bytes of a row.  Rows of odd lengths begin anywhere: this chip's loads and stores need no alignment beyond the element's.
template <typename T> struct Vec {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Sum over groups of LANES neighbouring lanes, in all of them.
template <int LANES> __device__ inline float lanes_sum(float v)
{
    auto moved = [](float x, auto ctl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctl)::value, 0xf, 0xf, true));
    };
    static_assert(LANES >= 8 && LANES <= 64, "a row of the register file at most");
    v += moved(v, std::integral_constant<int, 0xb1>{});         // quad_perm 1,0,3,2
    v += moved(v, std::integral_constant<int, 0x4e>{});         // quad_perm 2,3,0,1
    v += moved(v, std::integral_constant<int, 0x141>{});        // row_half_mirror: the other four of eight
    if constexpr (LANES >= 16) v += moved(v, std::integral_constant<int, 0x140>{});      // row_mirror: the other eight
    if constexpr (LANES >= 32) {
        const unsigned u = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    if constexpr (LANES >= 64) {
        const unsigned u = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        v = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    return v;
}
// Sums of M values over the LANES lanes that share a row.  Rows of several wavefronts exchange them through LDS, in two buffers that take turns: a wavefront
// writes one again only after a barrier that all reach behind their reads of it.
template <int LANES, int M> __device__ inline void row_sum(float (&v)[M], float (&part)[2][M][16], int &turn)
{
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = lanes_sum<(LANES < 64 ? LANES : 64)>(v[m]);
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
    // Zeros (`none`) where the lane has nothing.
    template <typename U> __device__ void load(const U *row, float (&v)[SIZE], float none = 0.f) const
    {
        typedef U uvec __attribute__((ext_vector_type(V), aligned(sizeof(U))));
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (has(k)) {
                const uvec u = *(const uvec *)(row + (k * LANES + at) * V);
#pragma unroll
                for (int e = 0; e < V; ++e) v[k * V + e] = (float)u[e];
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) v[k * V + e] = none;
            }
        }
        v[K * V] = has_tail() ? (float)row[vectors * V + at] : none;
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
        s.load(x + at, v);
        if (residual) {
            float w[S::SIZE];
            s.load(residual + at, w);
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
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < rows; r0 += (long long)gridDim.x * ROWS) {
        const long long row = r0 + threadIdx.x / LANES;
        if (row >= rows) break;
        const size_t at = (size_t)row * C;
        const float mean = save_mean[row], invstd = save_invstd[row];
        float v[S::SIZE], d[S::SIZE], t[2] = {0.f, 0.f};
        s.load(sum + at, v, mean);      // (xh is 0 where the lane has nothing)
        s.load(dy + at, d);
#pragma unroll
        for (int i = 0; i < S::SIZE; ++i) {
            v[i] = (v[i] - mean) * invstd;
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
        for (int i = 0; i < S::SIZE; ++i) v[i] = invstd * (d[i] - a - v[i] * b);
        if (dsum) {
            s.load(dsum + at, d);
#pragma unroll
            for (int i = 0; i < S::SIZE; ++i) v[i] += d[i];
        }
        s.store(dx + at, v);
    }
    if constexpr (PARAMS) {
        float *const p = partial + (size_t)blockIdx.x * C, *const q = p + (size_t)gridDim.x * C;
        if constexpr (ROWS > 1) {
            // lanes of the block's other rows with the same columns: added up in LDS, row by row
            extern __shared__ float sums[];     // [2][C]
            for (int turn2 = 0; turn2 < ROWS; ++turn2) {
                __syncthreads();
                if ((int)threadIdx.x / LANES == turn2) {
                    auto add = [&](int c, int i) {
                        sums[c] = turn2 ? sums[c] + dg[i] : dg[i];
                        sums[C + c] = turn2 ? sums[C + c] + db[i] : db[i];
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
        for (int k = k0; k < shares; k += 32) t += (double)partial[((size_t)blockIdx.y * shares + k) * C + c];
    part[k0][column] = t;
    __syncthreads();
    if (k0 == 0 && c < C) {
        for (int k = 1; k < 32; ++k) t += part[k][column];
        out[c] = (float)(accumulate ? (double)out[c] + t : t);
    }
}

// Lanes that share a row, and vectors of each.
struct Plan {
    int lanes, k;       // lanes 0: the kernels that hold nothing
};
Plan plan_of(const nsk_layernorm_desc_t &d)
{
    const int v = d.dtype == NSK_BF16 ? 8 : 4, vectors = d.C / v;
    for (int lanes = 8; lanes <= 64; lanes *= 2)
        if (vectors <= lanes) return {lanes, 1};
    if (vectors <= 128) return {64, 2};
    if (vectors <= 256) return {64, 4};
    if (vectors <= 512) return {256, 2};
    if (vectors <= 1024) return {256, 4};
    if (vectors <= 2048) return {1024, 2};
    return {0, 0};
}
int rows_a_block(const Plan &p) { return p.lanes == 0 || p.lanes >= 256 ? 1 : 256 / p.lanes; }
// Blocks of the backward pass, each with sums of its own.
int shares_of(const nsk_layernorm_desc_t &d)
{
    const Plan p = plan_of(d);
    const long long blocks = (d.rows + 4 * rows_a_block(p) - 1) / (4 * rows_a_block(p)), most = p.lanes == 1024 ? 256 : 512;
    return (int)(blocks < most ? blocks : most);
}

int check(const nsk_layernorm_desc_t *d)
{
    if (!d) return NSK_ERR_NULL;
    // (rows * C: a byte offset of it has to fit a pointer)
    if (d->rows <= 0 || d->C <= 0 || (d->dtype != NSK_F32 && d->dtype != NSK_BF16) || d->rows > (1LL << 60) / d->C) return NSK_ERR_BAD_DESC;
    return NSK_OK;
}

// f(LANES, K) of the plan, as constants.
template <typename F> void with(const Plan &p, F &&f)
{
#define NSK_CASE(L, N)                                                                   \
    if (p.lanes == L && p.k == N) f(std::integral_constant<int, L>{}, std::integral_constant<int, N>{});
    NSK_CASE(8, 1) NSK_CASE(16, 1) NSK_CASE(32, 1) NSK_CASE(64, 1) NSK_CASE(64, 2) NSK_CASE(64, 4) NSK_CASE(256, 2) NSK_CASE(256, 4) NSK_CASE(1024, 2)
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
    const long long need = (desc->rows + rows_a_block(p) - 1) / rows_a_block(p), most = p.lanes == 0 || p.lanes == 1024 ? 512 : 2048;
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
        if (p.lanes == 0) {
            if (params)
                hipLaunchKernelGGL(layernorm_dparam_wide_kernel<T>, dim3((unsigned)shares, (unsigned)ceil_div(C, 256)), dim3(256), 0, st, (const T *)s, (const T *)dy, save_mean, save_invstd,
                                   partial, desc->rows, C);
            hipLaunchKernelGGL(layernorm_dx_wide_kernel<T>, dim3((unsigned)(desc->rows < 512 ? desc->rows : 512)), dim3(1024), 0, st, (const T *)s, (const T *)dy, (const T *)dsum, gamma,
                               save_mean, save_invstd, (T *)dx, desc->rows, C);
        }
        with(p, [&](auto lanes, auto k) {
            constexpr int L = decltype(lanes)::value, N = decltype(k)::value;
            const dim3 block(L > 256 ? L : 256);
            if (params)
                hipLaunchKernelGGL((layernorm_bwd_kernel<T, L, N, true>), grid, block, L < 256 ? 2 * C * sizeof(float) : 0, st, (const T *)s, (const T *)dy, (const T *)dsum, gamma, save_mean,
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
