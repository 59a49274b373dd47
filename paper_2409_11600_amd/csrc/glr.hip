// Gated linear recurrence: for every sequence and channel
//   f = sigmoid(gi_f + b_f), c = gi_c + b_c, o = sigmoid(gi_o + b_o),  h_t = f h_{t-1} + (1 - f) c,  y_t = o h_t,
// all steps in one call in both directions, and one token for each of many sequences.  Backwards, with G_t the gradient of h_t:
//   G_t = dy_t o_t + f_{t+1} G_{t+1},  dc = G (1 - f),  d gi_f = G (h_{t-1} - c) f (1 - f),  d gi_o = dy h o (1 - o),  dh0 = f_1 G_1.
#include <math.h>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

// sigmoid(a) and 1 - sigmoid(a), both to the last places: near 1 the difference from it would keep none of the small one's.
__device__ inline void sigmoid2(float a, float &s, float &rest)
{
    const float e = expf(-fabsf(a)), big = 1.f / (1.f + e), small = e * big;
    s = a >= 0.f ? big : small;
    rest = a >= 0.f ? small : big;
}

constexpr int kStretch = NSK_GLR_STRETCH;

// A thread a channel, step by step.
template <typename T>
__global__ __launch_bounds__(64) void glr_fwd_kernel(nsk_glr_desc_t d, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                     const float *__restrict__ h0, T *__restrict__ y, float *__restrict__ h_last, float *__restrict__ saved)
{
    const int c = blockIdx.x * 64 + threadIdx.x, n = blockIdx.y, H = d.H;
    if (c >= H) return;
    const float bf = bias ? bias[c] : 0.f, bc = bias ? bias[H + c] : 0.f, bo = bias ? bias[2 * H + c] : 0.f;
    const int len = lengths ? lengths[n] : d.T;
    float h = h0 ? h0[(size_t)n * H + c] : 0.f;
    for (int t = 0; t < d.T; ++t) {
        if (saved && t % kStretch == 0) saved[((size_t)(t / kStretch) * d.N + n) * H + c] = h;
        float out = 0.f;
        if (t < len) {
            const T *g = gi + (size_t)t * d.gi_t + (size_t)n * d.gi_n + c;
            float f, keep, o, rest;
            sigmoid2((float)g[0] + bf, f, keep);
            sigmoid2((float)g[2 * (size_t)H] + bo, o, rest);
            h = f * h + keep * ((float)g[H] + bc);
            out = o * h;
        }
        if (y) y[(size_t)t * d.y_t + (size_t)n * d.y_n + c] = (T)out;
    }
    if (h_last) h_last[(size_t)n * H + c] = h;
}

template <typename T>
__global__ __launch_bounds__(64) void glr_bwd_kernel(nsk_glr_desc_t d, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                     const float *__restrict__ saved, const T *__restrict__ dy, const float *__restrict__ dh_last, T *__restrict__ dgi,
                                                     float *__restrict__ dh0)
{
    const int c = blockIdx.x * 64 + threadIdx.x, n = blockIdx.y, H = d.H;
    if (c >= H) return;
    const float bf = bias ? bias[c] : 0.f, bc = bias ? bias[H + c] : 0.f, bo = bias ? bias[2 * H + c] : 0.f;
    const int len = lengths ? lengths[n] : d.T;
    float G = dh_last ? dh_last[(size_t)n * H + c] : 0.f;
    for (int k = (d.T - 1) / kStretch; k >= 0; --k) {
        const int t0 = k * kStretch, count = d.T - t0 < kStretch ? d.T - t0 : kStretch;
        float before[kStretch];                 // the states that enter the steps of this stretch
        float h = saved[((size_t)k * d.N + n) * H + c];
#pragma unroll
        for (int i = 0; i < kStretch; ++i) {
            before[i] = h;
            if (i < count && t0 + i < len) {
                const T *g = gi + (size_t)(t0 + i) * d.gi_t + (size_t)n * d.gi_n + c;
                float f, keep;
                sigmoid2((float)g[0] + bf, f, keep);
                h = f * h + keep * ((float)g[H] + bc);
            }
        }
#pragma unroll
        for (int i = kStretch - 1; i >= 0; --i) {
            const int t = t0 + i;
            if (i >= count) continue;
            float df = 0.f, dc = 0.f, dout = 0.f;
            if (t < len) {
                const T *g = gi + (size_t)t * d.gi_t + (size_t)n * d.gi_n + c;
                float f, keep, o, rest;
                sigmoid2((float)g[0] + bf, f, keep);
                sigmoid2((float)g[2 * (size_t)H] + bo, o, rest);
                const float cand = (float)g[H] + bc, up = dy ? (float)dy[(size_t)t * d.y_t + (size_t)n * d.y_n + c] : 0.f;
                G += up * o;
                dc = G * keep;
                df = dc * f * (before[i] - cand);
                dout = up * o * rest * (f * before[i] + keep * cand);
                G *= f;
            }
            T *q = dgi + (size_t)t * d.gi_t + (size_t)n * d.gi_n + c;
            q[0] = (T)df;
            q[H] = (T)dc;
            q[2 * (size_t)H] = (T)dout;
        }
    }
    if (dh0) dh0[(size_t)n * H + c] = G;
}

template <typename T>
__global__ __launch_bounds__(64) void glr_step_kernel(int H, int S, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ slots,
                                                      float *__restrict__ state, T *__restrict__ y)
{
    const int c = blockIdx.x * 64 + threadIdx.x, n = blockIdx.y;
    if (c >= H) return;
    const int slot = slots ? slots[n] : n;
    float out = 0.f;
    if (slot >= 0 && slot < S) {
        const T *g = gi + (size_t)n * 3 * H + c;
        float f, keep, o, rest;
        sigmoid2((float)g[0] + (bias ? bias[c] : 0.f), f, keep);
        sigmoid2((float)g[2 * (size_t)H] + (bias ? bias[2 * H + c] : 0.f), o, rest);
        float *h = state + (size_t)slot * H + c;
        *h = f * *h + keep * ((float)g[H] + (bias ? bias[H + c] : 0.f));
        out = o * *h;
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
    if (d.N > 65535) return NSK_ERR_UNSUPPORTED;
    return NSK_OK;
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

size_t nsk_glr_workspace_bytes(const nsk_glr_desc_t *, int) { return 0; }

int nsk_glr_fwd(const nsk_glr_desc_t *desc, const void *gi, const float *bias, const int *lengths, const float *h0, void *y, float *h_last, float *saved,
                void *workspace, size_t, void *stream)
{
    nsk_glr_desc_t d;
    const int status = check(desc, d);
    if (status != NSK_OK) return status;
    if (!gi || (!y && !h_last)) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(lengths) || unaligned16(h0) || unaligned16(y) || unaligned16(h_last) || unaligned16(saved) || unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    const dim3 grid((unsigned)ceil_div(d.H, 64), (unsigned)d.N);
    if (d.dtype == NSK_BF16)
        hipLaunchKernelGGL(glr_fwd_kernel<bf16_t>, grid, dim3(64), 0, (hipStream_t)stream, d, (const bf16_t *)gi, bias, lengths, h0, (bf16_t *)y, h_last, saved);
    else
        hipLaunchKernelGGL(glr_fwd_kernel<float>, grid, dim3(64), 0, (hipStream_t)stream, d, (const float *)gi, bias, lengths, h0, (float *)y, h_last, saved);
    return check_launch();
}

int nsk_glr_bwd(const nsk_glr_desc_t *desc, const void *gi, const float *bias, const int *lengths, const float *saved, const void *dy, const float *dh_last,
                void *dgi, float *dh0, void *workspace, size_t, void *stream)
{
    nsk_glr_desc_t d;
    const int status = check(desc, d);
    if (status != NSK_OK) return status;
    if (!gi || !saved || (!dy && !dh_last) || !dgi) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(lengths) || unaligned16(saved) || unaligned16(dy) || unaligned16(dh_last) || unaligned16(dgi) || unaligned16(dh0) || unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    const dim3 grid((unsigned)ceil_div(d.H, 64), (unsigned)d.N);
    if (d.dtype == NSK_BF16)
        hipLaunchKernelGGL(glr_bwd_kernel<bf16_t>, grid, dim3(64), 0, (hipStream_t)stream, d, (const bf16_t *)gi, bias, lengths, saved, (const bf16_t *)dy, dh_last, (bf16_t *)dgi, dh0);
    else
        hipLaunchKernelGGL(glr_bwd_kernel<float>, grid, dim3(64), 0, (hipStream_t)stream, d, (const float *)gi, bias, lengths, saved, (const float *)dy, dh_last, (float *)dgi, dh0);
    return check_launch();
}

int nsk_glr_step(int dtype, int N, int H, int S, const void *gi, const float *bias, const int *slots, float *state, void *y, void *stream)
{
    if (N <= 0 || H <= 0 || H > (1 << 28) || S <= 0 || (dtype != NSK_F32 && dtype != NSK_BF16)) return NSK_ERR_BAD_DESC;
    if (N > 65535) return NSK_ERR_UNSUPPORTED;
    if (!gi || !state) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(slots) || unaligned16(state) || unaligned16(y)) return NSK_ERR_ALIGNMENT;
    const dim3 grid((unsigned)ceil_div(H, 64), (unsigned)N);
    if (dtype == NSK_BF16)
        hipLaunchKernelGGL(glr_step_kernel<bf16_t>, grid, dim3(64), 0, (hipStream_t)stream, H, S, (const bf16_t *)gi, bias, slots, state, (bf16_t *)y);
    else
        hipLaunchKernelGGL(glr_step_kernel<float>, grid, dim3(64), 0, (hipStream_t)stream, H, S, (const float *)gi, bias, slots, state, (float *)y);
    return check_launch();
}

}  // extern "C"
