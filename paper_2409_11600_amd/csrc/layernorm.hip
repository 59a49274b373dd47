// Layer norm over the last axis with the residual add in front of it, forward and backward.
//   s = x + residual,  y = (s - mean) * invstd * gamma + beta
//   gh = dy * gamma, xh = (s - mean) * invstd:  dx = invstd * (gh - mean(gh) - xh * mean(gh * xh)) + dsum,
//   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

__device__ inline float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <typename T>
__global__ __launch_bounds__(256) void layernorm_fwd_kernel(const T *__restrict__ x, const T *residual, const float *__restrict__ gamma,
                                                            const float *__restrict__ beta, T *sum, T *__restrict__ y,
                                                            float *__restrict__ save_mean, float *__restrict__ save_invstd, long long rows, int C, float eps)
{
    const int lane = threadIdx.x & 63;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const size_t at = (size_t)row * C;
    auto value = [&](int c) { return residual ? (float)(T)((float)x[at + c] + (float)residual[at + c]) : (float)x[at + c]; };
    float t = 0.f;
    for (int c = lane; c < C; c += 64) t += value(c);
    const float mean = wave_sum(t) / (float)C;
    t = 0.f;
    for (int c = lane; c < C; c += 64) {
        const float d = value(c) - mean;
        t += d * d;
    }
    const float invstd = 1.f / sqrtf(wave_sum(t) / (float)C + eps);
    for (int c = lane; c < C; c += 64) {
        const float s = value(c);
        if (sum) sum[at + c] = (T)s;
        y[at + c] = (T)((s - mean) * invstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f));
    }
    if (lane == 0) {
        if (save_mean) save_mean[row] = mean;
        if (save_invstd) save_invstd[row] = invstd;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void layernorm_dx_kernel(const T *__restrict__ s, const T *__restrict__ dy, const T *dsum, const float *__restrict__ gamma,
                                                           const float *__restrict__ save_mean, const float *__restrict__ save_invstd, T *dx, long long rows, int C)
{
    const int lane = threadIdx.x & 63;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const size_t at = (size_t)row * C;
    const float mean = save_mean[row], invstd = save_invstd[row];
    float a = 0.f, b = 0.f;
    for (int c = lane; c < C; c += 64) {
        const float gh = (float)dy[at + c] * (gamma ? gamma[c] : 1.f);
        a += gh;
        b += gh * ((float)s[at + c] - mean) * invstd;
    }
    a = wave_sum(a) / (float)C;
    b = wave_sum(b) / (float)C;
    for (int c = lane; c < C; c += 64) {
        const float gh = (float)dy[at + c] * (gamma ? gamma[c] : 1.f), xh = ((float)s[at + c] - mean) * invstd;
        dx[at + c] = (T)(invstd * (gh - a - xh * b) + (dsum ? (float)dsum[at + c] : 0.f));
    }
}

// Rows are shared out to at most kShares blocks; each leaves its sums of dy * xh and of dy, which one thread a column adds up.
constexpr int kShares = 256, kShareRows = 16;
int shares_of(long long rows) { return (int)(rows / kShareRows < 1 ? 1 : rows / kShareRows > kShares ? kShares : rows / kShareRows); }

template <typename T>
__global__ __launch_bounds__(256) void layernorm_dparam_kernel(const T *__restrict__ s, const T *__restrict__ dy, const float *__restrict__ save_mean,
                                                               const float *__restrict__ save_invstd, float *__restrict__ partial, long long rows, int C)
{
    const int c = blockIdx.y * 256 + threadIdx.x;
    if (c >= C) return;
    const long long per = (rows + gridDim.x - 1) / gridDim.x, begin = per * blockIdx.x, end = begin + per < rows ? begin + per : rows;
    float a = 0.f, b = 0.f;
    for (long long r = begin; r < end; ++r) {
        const float d = (float)dy[(size_t)r * C + c];
        a += d * ((float)s[(size_t)r * C + c] - save_mean[r]) * save_invstd[r];
        b += d;
    }
    partial[(size_t)blockIdx.x * C + c] = a;
    partial[(size_t)(gridDim.x + blockIdx.x) * C + c] = b;
}
__global__ __launch_bounds__(256) void layernorm_dparam_final_kernel(const float *__restrict__ partial, float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                                     int shares, int C, int accumulate)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    float *out = blockIdx.y ? dbeta : dgamma;
    if (c >= C || !out) return;
    double t = 0.0;
    for (int k = 0; k < shares; ++k) t += (double)partial[(size_t)(blockIdx.y * shares + k) * C + c];
    out[c] = (float)(accumulate ? (double)out[c] + t : t);
}

int check(const nsk_layernorm_desc_t *d)
{
    if (!d) return NSK_ERR_NULL;
    // (rows * C: a byte offset of it has to fit a pointer)
    if (d->rows <= 0 || d->C <= 0 || (d->dtype != NSK_F32 && d->dtype != NSK_BF16) || d->rows > (1LL << 60) / d->C) return NSK_ERR_BAD_DESC;
    if (d->rows > 4LL * 0x7fffffff) return NSK_ERR_UNSUPPORTED;
    return NSK_OK;
}

}  // namespace
}  // namespace nsk

using namespace nsk;

extern "C" {

size_t nsk_layernorm_bwd_workspace_bytes(const nsk_layernorm_desc_t *desc)
{
    return check(desc) == NSK_OK ? (size_t)2 * shares_of(desc->rows) * desc->C * sizeof(float) : 0;
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
    const dim3 grid((unsigned)((desc->rows + 3) / 4));
    if (desc->dtype == NSK_BF16)
        hipLaunchKernelGGL(layernorm_fwd_kernel<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, (const bf16_t *)x, (const bf16_t *)residual, gamma, beta,
                           (bf16_t *)sum, (bf16_t *)y, save_mean, save_invstd, desc->rows, desc->C, desc->eps);
    else
        hipLaunchKernelGGL(layernorm_fwd_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, (const float *)x, (const float *)residual, gamma, beta,
                           (float *)sum, (float *)y, save_mean, save_invstd, desc->rows, desc->C, desc->eps);
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
    const int C = desc->C, shares = shares_of(desc->rows);
    const dim3 grid((unsigned)((desc->rows + 3) / 4)), pgrid((unsigned)shares, (unsigned)ceil_div(C, 256));
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (params) hipLaunchKernelGGL(layernorm_dparam_kernel<T>, pgrid, dim3(256), 0, st, (const T *)s, (const T *)dy, save_mean, save_invstd, (float *)workspace, desc->rows, C);
        hipLaunchKernelGGL(layernorm_dx_kernel<T>, grid, dim3(256), 0, st, (const T *)s, (const T *)dy, (const T *)dsum, gamma, save_mean, save_invstd, (T *)dx, desc->rows, C);
    };
    if (desc->dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    if (params)
        hipLaunchKernelGGL(layernorm_dparam_final_kernel, dim3((unsigned)ceil_div(C, 256), 2), dim3(256), 0, st, (const float *)workspace, dgamma, dbeta, shares, C, accumulate);
    return check_launch();
}

}  // extern "C"
