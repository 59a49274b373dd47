// AdamW whose moments are held in 8 bits: m and r = sqrt(v) as e4m3 values times a power of two for each 256 elements.
#include <math.h>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

constexpr int kBlock = NSK_ADAMW8_BLOCK;
static_assert(kBlock == 256, "four elements a lane of a wavefront");

// A launch takes up to kTensors tensors as one row of blocks of 256 elements: tensor k has the blocks first[k] .. first[k + 1] - 1.
constexpr int kTensors = 52;
struct Entry {
    float *w, *g;
    unsigned char *m, *r;
    float *scale_m, *scale_r;
    bf16_t *w_lp;
    unsigned long long n;
    float decay;        // 1 - lr * weight_decay
    unsigned key;       // of its random bits
};
struct Table {
    Entry e[kTensors];
    unsigned first[kTensors + 1];
    int count;
};
static_assert(sizeof(Table) + 64 <= 4096 && kTensors < 64, "kernel arguments; a lane a tensor");

struct Coef {
    float lr, beta1, rest1, beta2, rest2, eps, c1, c2;     // c1 = 1/(1-beta1^t), c2 = 1/sqrt(1-beta2^t)
};

__host__ __device__ inline unsigned mix(unsigned x)
{
    x ^= x >> 16;
    x *= 0x243F6A89u;
    x ^= x >> 15;
    x *= 0xB7E15163u;
    return x ^ (x >> 16);
}

// The exponent field of the power of two for which amax / scale lies in (224, 448].
__device__ inline int scale_exponent(float amax)
{
    const int e = (int)((__builtin_bit_cast(unsigned, amax) + 0x1fffffu) >> 23) - 8;
    return e < 1 ? 1 : e;
}
__device__ inline float power(int field) { return __builtin_bit_cast(float, (unsigned)field << 23); }

// A magnitude y <= 448 to one of its two neighbours among the e4m3 values, the upper one with the probability that makes y the mean
// (`bits`: 20 random ones).  Below 2^-6 the values are 2^-9 apart, as they are from 2^-6 to 2^-5.
__device__ inline float round_e4m3(float y, unsigned bits)
{
    const bool small = y < 0x1p-6f;
    const float z = small ? y + 0x1p-6f : y;
    const float q = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, z) + bits) & ~0xfffffu);
    return small ? q - 0x1p-6f : q;
}
__device__ inline bool finite(float x) { return (__builtin_bit_cast(unsigned, x) & 0x7fffffffu) < 0x7f800000u; }

// The largest of all lanes' values, in all of them: within rows of 16 lanes on the vector unit, then by swaps of rows and halves.
__device__ inline unsigned wave_max(unsigned v)
{
    auto higher = [](unsigned a, unsigned b) { return a > b ? a : b; };
    auto moved = [](unsigned x, auto ctl) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctl)::value, 0xf, 0xf, true); };
    v = higher(v, moved(v, std::integral_constant<int, 0xb1>{}));       // quad_perm 1,0,3,2
    v = higher(v, moved(v, std::integral_constant<int, 0x4e>{}));       // quad_perm 2,3,0,1
    v = higher(v, moved(v, std::integral_constant<int, 0x141>{}));      // row_half_mirror
    v = higher(v, moved(v, std::integral_constant<int, 0x140>{}));      // row_mirror
    auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = higher(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return higher(r[0], r[1]);
}

// A wavefront takes a block of 256 elements, four a lane: 16 bytes of w and g, 4 of m and r, and the largest magnitudes by exchange among its lanes, no LDS.
// Bound by memory, 20 or 22 bytes a weight: 64 million weights in 82 tensors with copies 258 us (5.5 TB/s), 8.8 million in 7 without 34 us (5.2 TB/s; 30 where
// they are still in the last-level cache), 95 small tensors 10 us for two launches.  Of 450 vector instructions a block 4 in 10 are the correctly rounded square root, the random
// bits and the rounding; the update's quotient takes the hardware's reciprocal (1 ulp), which no held value depends on.
__global__ __launch_bounds__(256) void adamw8_kernel(const Table tab, Coef ac, const float *__restrict__ grad_scale)
{
// (sums and products as the header writes them: the value that is rounded is then the same on every machine)
#pragma clang fp contract(off)
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x & 63;
    const float gs = grad_scale ? grad_scale[0] : 1.f;
    const unsigned units = tab.first[tab.count];
    // (the tensor of a block: as many as begin at or before it; a lane looks at one)
    const unsigned next = lane < tab.count ? tab.first[lane + 1] : ~0u;
    for (unsigned u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); u < units; u += gridDim.x * 4) {
        const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(u >= next));
        const Entry &p = tab.e[k];
        const unsigned b = u - tab.first[k];
        const unsigned long long i0 = (unsigned long long)b * kBlock + lane * 4;
        const int left = i0 >= p.n ? 0 : p.n - i0 < 4 ? (int)(p.n - i0) : 4;
        f32x4 w = {0.f, 0.f, 0.f, 0.f}, g = w;
        unsigned cm = 0, cr = 0;
        if (left == 4) {
            w = *(const f32x4 *)(p.w + i0);
            g = *(const f32x4 *)(p.g + i0);
            cm = *(const unsigned *)(p.m + i0);
            cr = *(const unsigned *)(p.r + i0);
        } else {
            for (int j = 0; j < left; ++j) {
                w[j] = p.w[i0 + j];
                g[j] = p.g[i0 + j];
                cm |= (unsigned)p.m[i0 + j] << (8 * j);
                cr |= (unsigned)p.r[i0 + j] << (8 * j);
            }
        }
        const float sm = p.scale_m[b], sr = p.scale_r[b];
        const f32x2 m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm, true);
        const f32x2 r01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cr, false), r23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cr, true);
        float m[4] = {m01[0], m01[1], m23[0], m23[1]}, r[4] = {r01[0], r01[1], r23[0], r23[1]};
        unsigned top_m = 0, top_r = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gj = g[j] * gs, mo = m[j] * sm, ro = r[j] * sr;
            m[j] = mo * ac.beta1 + gj * ac.rest1;
            r[j] = sqrtf(ro * ro * ac.beta2 + gj * gj * ac.rest2);
            w[j] = w[j] * p.decay - ac.lr * (m[j] * ac.c1 * __builtin_amdgcn_rcpf(r[j] * ac.c2 + ac.eps));
            const unsigned am = __builtin_bit_cast(unsigned, m[j]) & 0x7fffffffu, ar = __builtin_bit_cast(unsigned, r[j]);
            if (finite(m[j]) && am > top_m) top_m = am;
            if (finite(r[j]) && ar > top_r) top_r = ar;
        }
        const int em = scale_exponent(__builtin_bit_cast(float, wave_max(top_m))), er = scale_exponent(__builtin_bit_cast(float, wave_max(top_r)));
        const float im = power(254 - em), ir = power(254 - er);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned long long i = i0 + j;
            const unsigned h = mix((unsigned)i * 0x9E3779B9u + (unsigned)(i >> 32) * 0x85A308D3u + p.key);
            const float qm = round_e4m3(fabsf(m[j]) * im, (h & 0xffffu) << 4);
            float qr = round_e4m3(r[j] * ir, h >> 16 << 4);
            if (r[j] > 0.f && qr < 0x1p-9f) qr = 0x1p-9f;
            m[j] = finite(m[j]) ? copysignf(qm, m[j]) : NAN;
            r[j] = finite(r[j]) ? qr : NAN;
        }
        cm = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(m[2], m[3], __builtin_amdgcn_cvt_pk_fp8_f32(m[0], m[1], 0, false), true);
        cr = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false), true);
        if (left == 4) {
            *(f32x4 *)(p.w + i0) = w;
            *(f32x4 *)(p.g + i0) = f32x4{0.f, 0.f, 0.f, 0.f};
            *(unsigned *)(p.m + i0) = cm;
            *(unsigned *)(p.r + i0) = cr;
            if (p.w_lp) *(bf16x4 *)(p.w_lp + i0) = bf16x4{(bf16_t)w[0], (bf16_t)w[1], (bf16_t)w[2], (bf16_t)w[3]};
        } else {
            for (int j = 0; j < left; ++j) {
                p.w[i0 + j] = w[j];
                p.g[i0 + j] = 0.f;
                p.m[i0 + j] = (unsigned char)(cm >> (8 * j));
                p.r[i0 + j] = (unsigned char)(cr >> (8 * j));
                if (p.w_lp) p.w_lp[i0 + j] = (bf16_t)w[j];
            }
        }
        if (lane == 0) {
            p.scale_m[b] = power(em);
            p.scale_r[b] = power(er);
        }
    }
}

int check(const nsk_param8_t &q)
{
    if (q.n == 0 || q.n > (1ull << 39)) return NSK_ERR_BAD_DESC;
    if (!q.w || !q.grad || !q.m || !q.r || !q.scale_m || !q.scale_r) return NSK_ERR_NULL;
    if (unaligned16(q.w) || unaligned16(q.grad) || unaligned16(q.m) || unaligned16(q.r) || unaligned16(q.w_lp) || ((uintptr_t)q.scale_m & 3) || ((uintptr_t)q.scale_r & 3))
        return NSK_ERR_ALIGNMENT;
    return NSK_OK;
}

}  // namespace
}  // namespace nsk

using namespace nsk;

extern "C" {

int nsk_adamw8_step_multi(int count, const nsk_param8_t *params, int step, unsigned seed, float lr, float beta1, float beta2, float eps,
                          const float *grad_scale, void *stream)
{
    if (count <= 0 || step < 1 || !(beta1 >= 0.f && beta1 < 1.f) || !(beta2 >= 0.f && beta2 < 1.f)) return NSK_ERR_BAD_DESC;
    if (!params) return NSK_ERR_NULL;
    if ((uintptr_t)grad_scale & 3) return NSK_ERR_ALIGNMENT;
    for (int i = 0; i < count; ++i) {
        const int status = check(params[i]);
        if (status != NSK_OK) return status;
    }
    Coef ac;
    ac.lr = lr;
    ac.beta1 = beta1;
    ac.rest1 = 1.f - beta1;
    ac.beta2 = beta2;
    ac.rest2 = 1.f - beta2;
    ac.eps = eps;
    ac.c1 = (float)(1.0 / (1.0 - pow((double)beta1, (double)step)));
    ac.c2 = (float)sqrt(1.0 / (1.0 - pow((double)beta2, (double)step)));
    for (int base = 0; base < count;) {
        Table tab{};
        unsigned long long units = 0;
        // (a launch counts its blocks in 32 bits)
        while (base < count && tab.count < kTensors) {
            const nsk_param8_t &q = params[base];
            const unsigned long long more = (q.n + kBlock - 1) / kBlock;
            if (units + more > 0xf0000000ull) break;
            tab.e[tab.count] = {q.w, q.grad, (unsigned char *)q.m, (unsigned char *)q.r, q.scale_m, q.scale_r, (bf16_t *)q.w_lp, q.n,
                                1.f - lr * q.weight_decay, mix(seed + (unsigned)base * 0x9E3779B9u)};
            tab.first[tab.count++] = (unsigned)units;
            tab.first[tab.count] = (unsigned)(units += more);
            ++base;
        }
        unsigned long long blocks = (units + 3) / 4;
        // (a wavefront a block of elements: the memory then sees them in order.  64 million weights with copies: 258 us, 4096 workgroups that go round 292, 1024 272)
        if (blocks > 1 << 22) blocks = 1 << 22;
        hipLaunchKernelGGL(adamw8_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, tab, ac, grad_scale);
    }
    return check_launch();
}

}  // extern "C"
