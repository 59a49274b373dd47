// Gated delta rule: for every sequence and head a state S [D,Dv], with k^ and q^ the normalised key and query, alpha = sigmoid(a + bias), beta = sigmoid(b + bias),
//   S' = alpha S_{t-1},  S_t = S' + k^ (beta (v - S'^T k^))^T,  o_t = S_t^T q^.
// Steps go in chunks of 64.  With c_i the sum of log alpha up to step i of the chunk, C the whole chunk's, S the state that enters it and (K, Q, V) its rows:
//   A_ij = beta_i exp(c_i - c_j) k_i.k_j (j < i),  P_ij = exp(c_i - c_j) q_i.k_j (j <= i),
//   (1 + A) U = beta (V - exp(c) K S),  O = exp(c) Q S + P U,  S <- exp(C) S + (exp(C - c) K)^T U.
// Backwards, with G the gradient of the state that leaves the chunk and R = V - exp(c) K S:
//   dU = P^T dO + exp(C - c) K G,  (1 + A)^T X = dU,  G <- exp(C) G + (exp(c) Q)^T dO - (beta exp(c) K)^T X,
//   dV = beta X,  dA = -X U^T,  dP = dO U^T  (where A and P are not zero),  and with E1 = X S^T, E2 = dO S^T, E3 = U G^T:
//   dQ = exp(c) E2 + (dP L) K,  dK = -beta exp(c) E1 + exp(C - c) E3 + (dA beta L) K + (dA beta L)^T K + (dP L)^T Q,  L_ij = exp(c_i - c_j),
//   and the gradients of beta and of the lengths of q and k from the row sums of the same products.  That of log alpha_t is the sum of what the gate t lies in: of row i's products with exp(c_i)
//   from i = t on, of row j's with exp(C - c_j) in front of t, of dA_ij A_ij + dP_ij P_ij over the pairs j < t <= i, and of exp(C) S G.  Only such terms are added up: they all hold alpha_t, so
//   that the sum keeps its bits where the gate is nearly closed (heads of 32 x 24 in fp32, T=200, relative 2-norms: 3e-7 at alpha = 1e-4, 7e-7 at 1e-7; as the sum from t on of the gradients of c,
//   most of which cancels there, 4e-4 and 0.3).
// Products keep 32 bits: states, gates' gradients and the results of a chunk of 64 dependent steps.  Those of two float operands are on the fp32 matrix unit.  Keys and queries in bf16 stay what they
// are (their lengths are factors of rows and columns, applied to the products), and what they are multiplied with goes in three bf16 pieces that hold all of its bits: three products of 16
// clocks for 32 indices, where the fp32 unit takes eight of 32.
//
// Where a product's result is the next one's right operand (S, U, X, G), it stays in its registers: v_mfma_f32_16x16x4_f32 leaves lane l rows 4 (l / 16) + r, r < 4, of column l % 16,
// and a right operand of 16 rows is read in four steps of which step s takes from lane l one value of column l % 16; which row that is is free as long as the left operand's lane takes the same:
// row 4 (l / 16) + s.  So a wavefront takes 16 columns of the state through all products by itself; A, P, K and Q, the left operands, lie in LDS.
#include <math.h>

#include <type_traits>

#include "nsk_internal.h"

namespace nsk {
namespace {

bool unaligned16(const void *p) { return ((uintptr_t)p & 15) != 0; }

constexpr int kC = NSK_DELTA_CHUNK;
constexpr int kLA = kC + 4;             // a row of A or P in LDS: neighbouring rows four banks apart
constexpr float kEps = NSK_DELTA_EPS;
constexpr int kMostWidth = 128;

struct Sizes {
    int T, N, H, Hk, D, Dv, chunks;
    int vec;                            // rows of q and k are whole vectors of 16 bytes
    long long gi_t, gi_n, o_t, o_n;
};
__device__ __forceinline__ int q_at(const Sizes &z, int hk) { return hk * z.D; }
__device__ __forceinline__ int k_at(const Sizes &z, int hk) { return (z.Hk + hk) * z.D; }
__device__ __forceinline__ int v_at(const Sizes &z, int h) { return 2 * z.Hk * z.D + h * z.Dv; }
__device__ __forceinline__ int a_at(const Sizes &z, int h) { return 2 * z.Hk * z.D + z.H * z.Dv + h; }
__device__ __forceinline__ int b_at(const Sizes &z, int h) { return a_at(z, h) + z.H; }
__device__ __forceinline__ int steps_of(const Sizes &z, const int *lengths, int n)
{
    const int l = lengths ? lengths[n] : z.T;
    return l < 0 ? 0 : l < z.T ? l : z.T;
}
__host__ __device__ __forceinline__ size_t state_at(const Sizes &z, int chunk, int n, int h) { return (((size_t)chunk * z.N + n) * z.H + h) * z.D * z.Dv; }

__device__ __forceinline__ float sigmoid(float a)
{
    const float e = expf(-fabsf(a));
    return (a >= 0.f ? 1.f : e) / (1.f + e);
}

// ----------------------------------------------------------------------------- products
// This thread's lane, as a number that is made anew: what is computed from it is not kept in registers from one round of a loop to the next (LDS addresses alone would fill them).
__device__ __forceinline__ int fresh_lane()
{
    int l = threadIdx.x & 63;
    asm volatile("" : "+v"(l));
    return l;
}
__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
// A left operand's rows row0..row0+15, columns k0..k0+15 of m, or of m transposed; also a right operand's columns and rows, of m transposed or of m.
__device__ __forceinline__ f32x4 frag(int l, const float *m, int ld, int row0, int k0)
{
    return *(const f32x4 *)(m + (row0 + (l & 15)) * ld + k0 + 4 * (l >> 4));
}
__device__ __forceinline__ f32x4 frag_t(int l, const float *m, int ld, int row0, int k0)
{
    const float *p = m + (k0 + 4 * (l >> 4)) * ld + row0 + (l & 15);
    return (f32x4){p[0], p[ld], p[2 * ld], p[3 * ld]};
}
__device__ __forceinline__ f32x4 multiply(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int s = 0; s < 4; ++s) c = mfma(a[s], b[s], c);
    return c;
}
// Nothing is moved across: the fragments of one row of tiles are in flight at a time, not those of a whole product, for which there are not enough registers.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }
// Sums that are read behind a branch or in a loop's next round.  A result of v_mfma_f32_16x16x4_f32 may be read ten wait states after it at the earliest, one of v_mfma_f32_16x16x32_bf16 eight;
// within a block of instructions the compiler sees to that, but where a branch ended with one and a block of a jump alone lay between, it left no wait, and what was read was the sum before the last products.
template <int N> __device__ __forceinline__ void settle(f32x4 (&x)[N])
{
    fence();
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("s_nop 15" : "+v"(x[i]));
    fence();
}
__device__ __forceinline__ f32x4 rows_of(int l, const float *v, int row0) { return *(const f32x4 *)(v + row0 + 4 * (l >> 4)); }
// Sums over the 16 columns of a tile; all lanes have them: rows of 16 lanes turned by 8, 4, 2 and 1.
template <int BY> __device__ __forceinline__ float add_turned(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + BY, 0xf, 0xf, true));
}
__device__ __forceinline__ f32x4 sum_columns(f32x4 v)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = add_turned<1>(add_turned<2>(add_turned<4>(add_turned<8>(v[r]))));
    return v;
}

// The sum of a tile's columns up to this lane's: rows of 16 lanes moved by 1, 2, 4 and 8.
template <int BY> __device__ __forceinline__ float add_moved(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x110 + BY, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_up_to_column(float v) { return add_moved<8>(add_moved<4>(add_moved<2>(add_moved<1>(v)))); }

// ----------------------------------------------------------------------------- memory
// Rows are reached through buffer descriptors: what lies at or behind `bytes` reads as zero and is not written, and so is a lane's offset of kNowhere plus anything below 2^31.  An access is
// a lane's offset plus a uniform one: one instruction, where 64-bit addresses and conditions took six.
constexpr unsigned kNowhere = 0x80000000u;
constexpr long long kMostStride = 1LL << 25;       // elements from a step to the next: 16 steps within 2^31 bytes
template <typename T> __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const T *p, long long bytes) { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)bytes, 0x00020000); }
template <typename T> __device__ __forceinline__ unsigned load_raw(__amdgpu_buffer_rsrc_t b, unsigned at)
{
    if constexpr (sizeof(T) == 2) return (unsigned)__builtin_amdgcn_raw_buffer_load_b16(b, at, 0, 0);
    else return (unsigned)__builtin_amdgcn_raw_buffer_load_b32(b, at, 0, 0);
}
template <typename T> __device__ __forceinline__ float value_of(unsigned raw) { return __builtin_bit_cast(float, sizeof(T) == 2 ? raw << 16 : raw); }
template <typename T> __device__ __forceinline__ void store(float v, __amdgpu_buffer_rsrc_t b, unsigned at)
{
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (T)v), b, at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), b, at, 0, 0);
}

// ----------------------------------------------------------------------------- what a chunk starts with
struct alignas(16) Gates {
    double c[kC];               // sums of log alpha to the base of two: differences of far ones keep what matters
    float beta[kC], in[kC], out[kC];        // beta, exp(c), exp(C - c)
    float rest_a[kC], rest_b[kC];           // 1 - alpha, 1 - beta
    float all;                  // exp(C)
};
// By one wavefront, a step a lane.  Steps from `live` on leave the state as it is.
__device__ __forceinline__ float exp_of(double c) { return __builtin_amdgcn_exp2f((float)c); }
// c plus the sums of the lanes in front: within 16 lanes, then over the rows of 16.
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ double moved(double c)
{
    const unsigned long long u = __builtin_bit_cast(unsigned long long, c);
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, ROWS, 0xf, true), hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, ROWS, 0xf, true);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double sums_in_row(double c)
{
    c += moved<0x111>(c);       // a row moved by 1, 2, 4 and 8 lanes
    c += moved<0x112>(c);
    c += moved<0x114>(c);
    return c + moved<0x118>(c);
}
__device__ __forceinline__ double sums_up_to(double c)
{
    c = sums_in_row(c);
    c += moved<0x142, 0xa>(c);       // the last lane of a row to the next one (rows 1 and 3), then of the second to the last two
    return c + moved<0x143, 0xc>(c);
}
template <typename T> struct GateParts {
    unsigned a, b;
    __device__ __forceinline__ void load(int i, const Sizes &z, const T *row, int h, int live)
    {
        const T *p = row + (i < live ? i : 0) * z.gi_t;
        a = raw_of(p + a_at(z, h));
        b = raw_of(p + b_at(z, h));
    }
    static __device__ __forceinline__ unsigned raw_of(const T *p)
    {
        if constexpr (sizeof(T) == 2) return *(const unsigned short *)p;
        else return *(const unsigned *)p;
    }
    __device__ __forceinline__ void finish(int i, const Sizes &z, const float *bias, int h, int live, Gates &g) const
    {
        double la = 0.;
        float beta = 0.f, rest_a = 0.f, rest_b = 0.f;
        if (i < live) {
            const float x = value_of<T>(a) + (bias ? bias[h] : 0.f), y = value_of<T>(b) + (bias ? bias[z.H + h] : 0.f);
            // log sigmoid(x); below -1000 alpha is 0 in any type, and a sum of infinities would have no differences.  Its rounding, 2^-24 of it, is the more the less the product
            // of gates counts: t exp(-t) is at most 0.37.  (NaN stays NaN: fminf of it and 0 would be 0, but not the sum's other part.)
            la = x < -1000.f ? -1000.f : fminf(x, 0.f) - log1pf(expf(-fabsf(x)));
            beta = sigmoid(y);
            rest_a = sigmoid(-x);
            rest_b = sigmoid(-y);
        }
        const double c = sums_up_to(la * 1.4426950408889634);
        const unsigned long long last = __builtin_bit_cast(unsigned long long, c);
        const double C = __builtin_bit_cast(double, (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(last >> 32), 63) << 32 |
                                                        (unsigned)__builtin_amdgcn_readlane((int)(unsigned)last, 63));
        g.c[i] = c;
        g.beta[i] = beta;
        g.in[i] = exp_of(c);
        g.out[i] = exp_of(C - c);
        g.rest_a[i] = rest_a;
        g.rest_b[i] = rest_b;
        if (i == 0) g.all = exp_of(C);
    }
};
template <typename T> __device__ __forceinline__ void load_gates(int l, const Sizes &z, const T *row, const float *bias, int h, int live, Gates &g)
{
    GateParts<T> p;
    p.load(l, z, row, h, live);
    p.finish(l, z, bias, h, live, g);
}

// A row of K or Q in LDS: neighbouring rows four banks apart.
template <typename T> constexpr int row_of(int DP) { return sizeof(T) == 2 ? DP + 8 : DP + 4; }
// Lengths of the chunk's rows.  Where T is float, K and Q hold normalised rows, and in_products below leaves the products as they are.
struct Lengths {
    float k[kC], q[kC], unit_q[kC];         // 1 / |k|, 1 / |q|, 1 / (sqrt(D) |q|)
};
template <typename T> __device__ __forceinline__ f32x4 in_products(int l, f32x4 x, const float *lengths, int row0)
{
    if constexpr (sizeof(T) == 2) return x * rows_of(l, lengths, row0);
    else return x;
}
// A row of q or k: THREADS / 64 neighbouring lanes take vectors of 16 bytes in turn.  They stay as they were loaded until they are used, so that nothing waits for them before.
template <typename T, int DP, int THREADS> struct RowPart {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    static constexpr int LANES = THREADS / 64, V = 16 / sizeof(T), VECTORS = DP / V, EACH = (VECTORS + LANES - 1) / LANES, ROWS = 64 / LANES;     // ROWS: of a wavefront
    u32x4 x[EACH];
    // p: the chunk's first row
    __device__ __forceinline__ void load(int l, int wave, const T *p, long long stride, int D, int live, bool vec)
    {
        int left = live - wave * ROWS;
        left = left < ROWS ? left : ROWS;
        const __amdgpu_buffer_rsrc_t b = buffer(p + wave * ROWS * stride, left <= 0 ? 0 : ((left - 1) * stride + D) * (long long)sizeof(T));
        const unsigned at = (unsigned)(l / LANES) * (unsigned)stride * (unsigned)sizeof(T);
        const int first = l % LANES * V;
        if (vec) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int e = first + i * LANES * V;
                x[i] = (u32x4)__builtin_amdgcn_raw_buffer_load_b128(b, e < D ? at + e * (unsigned)sizeof(T) : kNowhere, 0, 0);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            unsigned raw[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int e = first + i * LANES * V + k;
                raw[k] = load_raw<T>(b, e < D ? at + e * (unsigned)sizeof(T) : kNowhere);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (V == 8) x[i][k] = raw[2 * k] | raw[2 * k + 1] << 16;
                else x[i][k] = raw[k];
            }
        }
    }
    __device__ __forceinline__ float value(int i, int e) const
    {
        const unsigned u = V == 4 ? x[i][e] : e & 1 ? x[i][e / 2] & 0xffff0000u : x[i][e / 2] << 16;
        return __builtin_bit_cast(float, u);
    }
    // 1 / sqrt(|row|^2 + eps)
    __device__ __forceinline__ float inverse_length() const
    {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < EACH; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) s = fmaf(value(i, e), value(i, e), s);
        s += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, s), 0xb1, 0xf, 0xf, true));      // of lane ^ 1
        s += lane_xor<2>(s);
        if (LANES == 8) s += lane_xor<4>(s);
        return 1.f / sqrtf(s + kEps);
    }
    __device__ __forceinline__ void store(int l, T *row, float by) const
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int v = l % LANES + i * LANES;
            if (VECTORS % LANES && v >= VECTORS) continue;
            if constexpr (sizeof(T) == 2) *(u32x4 *)(row + v * V) = x[i];
            else
#pragma unroll
            for (int e = 0; e < V; e += 4) *(f32x4 *)(row + v * V + e) = (f32x4){value(i, e) * by, value(i, e + 1) * by, value(i, e + 2) * by, value(i, e + 3) * by};
        }
    }
};
// Keys and queries of a chunk into LDS, and their lengths.
template <typename T, int DP, int THREADS> struct KeyParts {
    typedef RowPart<T, DP, THREADS> Part;
    Part k, q;
    __device__ __forceinline__ void load(int l, int wave, const Sizes &z, const T *row0, int hk, int live)
    {
        k.load(l, wave, row0 + k_at(z, hk), z.gi_t, z.D, live, z.vec);
        q.load(l, wave, row0 + q_at(z, hk), z.gi_t, z.D, live, z.vec);
    }
    __device__ __forceinline__ void finish(int l, int wave, const Sizes &z, T *K, T *Q, Lengths &lengths) const
    {
        const int r = wave * Part::ROWS + l / Part::LANES;
        const float ik = k.inverse_length(), iq = q.inverse_length(), unit = iq / sqrtf((float)z.D);
        k.store(l, K + r * row_of<T>(DP), ik);
        q.store(l, Q + r * row_of<T>(DP), unit);
        if (l % Part::LANES == 0) {
            lengths.k[r] = ik;
            lengths.q[r] = iq;
            lengths.unit_q[r] = unit;
        }
    }
};

// Right operands of products with K and Q: the state's DT tiles of 16 rows, or the chunk's four, as they are in registers or in pieces.  A lane's eight values of 32 rows are those of two tiles
// one after the other; the left operands below are read in the same order.
template <typename T, int TILES> struct Operand {
    f32x4 x[TILES];
    __device__ __forceinline__ void set(const f32x4 (&v)[TILES])
    {
#pragma unroll
        for (int i = 0; i < TILES; ++i) x[i] = v[i];
    }
};
template <int TILES> struct Operand<bf16_t, TILES> {
    Pieces x[TILES / 2];
    __device__ __forceinline__ void set(const f32x4 (&v)[TILES])
    {
#pragma unroll
        for (int i = 0; i < TILES / 2; ++i) {
            const float y[8] = {v[2 * i][0], v[2 * i][1], v[2 * i][2], v[2 * i][3], v[2 * i + 1][0], v[2 * i + 1][1], v[2 * i + 1][2], v[2 * i + 1][3]};
            x[i] = split3<false>(y);
        }
    }
};
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(bf16x8 a, const Pieces &b, f32x4 c) { return mfma(a, b.h, mfma(a, b.m, mfma(a, b.l, c))); }
__device__ __forceinline__ bf16x8 both(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
// Four rows of m from k0 + 4 (l / 16) on, of column row0 + l % 16: a read that turns 4 x 16 elements (each lane gives the address of four of a row).
__device__ __forceinline__ bf16x4 turned(int l, const bf16_t *m, int ld, int row0, int k0)
{
    typedef __attribute__((address_space(3))) bf16x4 *Lds;
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((Lds)(m + (k0 + 4 * (l >> 4) + ((l & 15) >> 2)) * ld + row0 + 4 * (l & 3)));
}
// 16 rows of m from row0 on, times the operand.
template <int TILES> __device__ __forceinline__ f32x4 times(int l, const float *m, int ld, int row0, const Operand<float, TILES> &o, f32x4 c)
{
#pragma unroll
    for (int k = 0; k < TILES; ++k) c = multiply(frag(l, m, ld, row0, 16 * k), o.x[k], c);
    return c;
}
template <int TILES> __device__ __forceinline__ f32x4 times(int l, const bf16_t *m, int ld, int row0, const Operand<bf16_t, TILES> &o, f32x4 c)
{
    const bf16_t *p = m + (row0 + (l & 15)) * ld + 4 * (l >> 4);
#pragma unroll
    for (int k = 0; k < TILES / 2; ++k) c = multiply(both(*(const bf16x4 *)(p + 32 * k), *(const bf16x4 *)(p + 32 * k + 16)), o.x[k], c);
    return c;
}
// The same of m transposed: its columns row0.., over the chunk's rows.
__device__ __forceinline__ f32x4 times_t(int l, const float *m, int ld, int row0, const Operand<float, 4> &o, f32x4 c)
{
#pragma unroll
    for (int b = 0; b < 4; ++b) c = multiply(frag_t(l, m, ld, row0, 16 * b), o.x[b], c);
    return c;
}
__device__ __forceinline__ f32x4 times_t(int l, const bf16_t *m, int ld, int row0, const Operand<bf16_t, 4> &o, f32x4 c)
{
#pragma unroll
    for (int b = 0; b < 2; ++b) c = multiply(both(turned(l, m, ld, row0, 32 * b), turned(l, m, ld, row0, 32 * b + 16)), o.x[b], c);
    return c;
}
// A right operand of 16 of the chunk's rows on the fp32 unit: normalised keys or queries.
__device__ __forceinline__ f32x4 rows_t(int l, const float *m, int ld, int row0, int k0, const float *) { return frag_t(l, m, ld, row0, k0); }
__device__ __forceinline__ f32x4 rows_t(int l, const bf16_t *m, int ld, int row0, int k0, const float *lengths)
{
    const bf16x4 x = turned(l, m, ld, row0, k0);
    return (f32x4){(float)x[0], (float)x[1], (float)x[2], (float)x[3]} * rows_of(l, lengths, k0);
}

// The tiles of 16 x 16 of A and P that are not zero: 10 each.
constexpr int kTiles = 10;
__device__ __forceinline__ void tile_at(int t, int &bi, int &bj)
{
    bi = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3;
    bj = t - bi * (bi + 1) / 2;
}
// exp(c_i - c_j) for this lane's elements of a tile; 0 where j > i, or j = i in a strict one.
__device__ __forceinline__ f32x4 decays(int l, const Gates &g, int bi, int bj, bool strict)
{
    const int i0 = 16 * bi + 4 * (l >> 4), j = 16 * bj + (l & 15);
    const double cj = g.c[j];
    f32x4 d;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float e = exp_of(g.c[i0 + r] - cj);       // (taken everywhere, without a branch)
        d[r] = i0 + r > j - !strict ? e : 0.f;
    }
    return d;
}
__device__ __forceinline__ void store_tile(int l, float *m, int bi, int bj, f32x4 v)
{
    float *p = m + (16 * bi + 4 * (l >> 4)) * kLA + 16 * bj + (l & 15);
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r * kLA] = v[r];
}
// -A and P by NW wavefronts, the first TILES tiles of 20, of which the first ten are A's: every NW-th tile from this wavefront's number on.  All of a wavefront's tiles go through the products
// together: one after the other they would wait for LDS four times each.  Returns the tiles without beta (A) or as they are (P), zeros where a wavefront has one less.
template <typename T, int DP, int NW, int TILES, int EACH = (TILES + NW - 1) / NW>
__device__ __forceinline__ void make_tiles(int l, int wave, const Gates &g, const Lengths &lengths, const T *K, const T *Q, float *A, float *P, f32x4 (&x)[EACH])
{
    constexpr int LD = row_of<T>(DP), STEP = sizeof(T) == 2 ? 32 : 16;
    typedef std::conditional_t<sizeof(T) == 2, bf16x8, f32x4> Frag;
    int bi[EACH], bj[EACH];
    const T *left[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int t = wave + i * NW < TILES ? wave + i * NW : TILES - 1;
        tile_at(t < kTiles ? t : t - kTiles, bi[i], bj[i]);
        left[i] = t < kTiles ? K : Q;
        x[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int k0 = 0; k0 < DP; k0 += STEP) {
        const int at = (l & 15) * LD + k0 + STEP / 4 * (l >> 4);
        Frag a[EACH], b[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            a[i] = *(const Frag *)(left[i] + 16 * bi[i] * LD + at);
            b[i] = *(const Frag *)(K + 16 * bj[i] * LD + at);
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) x[i] = mfma(a[i], b[i], x[i]);
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int i = 0; i < EACH; ++i) x[i] = mfma(a[i][s], b[i][s], x[i]);
        }
    }
    settle(x);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int t = wave + i * NW;
        const bool is_a = t < kTiles;
        x[i] *= decays(l, g, bi[i], bj[i], is_a);
        if constexpr (sizeof(T) == 2) x[i] *= rows_of(l, is_a ? lengths.k : lengths.unit_q, 16 * bi[i]) * lengths.k[16 * bj[i] + (l & 15)];
        const f32x4 by = -rows_of(l, g.beta, 16 * bi[i]);
        if (t >= TILES) x[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        else store_tile(l, is_a ? A : P, bi[i], bj[i], is_a ? by * x[i] : x[i]);
    }
}
// The inverse of a diagonal block of 1 + A, in its place: wavefront w takes block w, each lane a column (the four groups of 16 lanes the same).
__device__ __forceinline__ void invert_block(int l, float *A, int w)
{
    const int c = l & 15;
    float *m = A + 16 * w * kLA + 16 * w;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float sum[2] = {i == c ? 1.f : 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < i; j += 4) {
            const f32x4 a = *(const f32x4 *)(m + i * kLA + j);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < i) sum[e & 1] = fmaf(a[e], x[j + e], sum[e & 1]);
        }
        x[i] = sum[0] + sum[1];
    }
    if (l < 16)
#pragma unroll
        for (int i = 0; i < 16; ++i) m[i * kLA + c] = x[i];
}
// (1 + A) U = X, and (1 + A)^T U = X, in place for 16 columns.
__device__ __forceinline__ void solve(int l, const float *A, f32x4 (&X)[4])
{
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int j = 0; j < b; ++j) X[b] = multiply(frag(l, A, kLA, 16 * b, 16 * j), X[j], X[b]);
        X[b] = multiply(frag(l, A, kLA, 16 * b, 16 * b), X[b], (f32x4){0.f, 0.f, 0.f, 0.f});
    }
}
__device__ __forceinline__ void solve_t(int l, const float *A, f32x4 (&X)[4])
{
#pragma unroll
    for (int b = 3; b >= 0; --b) {
#pragma unroll
        for (int j = 3; j > b; --j) X[b] = multiply(frag_t(l, A, kLA, 16 * b, 16 * j), X[j], X[b]);
        X[b] = multiply(frag_t(l, A, kLA, 16 * b, 16 * b), X[b], (f32x4){0.f, 0.f, 0.f, 0.f});
    }
}

// 16 columns of a state [D,Dv] in registers.
template <int DT> __device__ __forceinline__ void load_state(int l, const Sizes &z, const float *s, int col, f32x4 (&S)[DT])
{
    const __amdgpu_buffer_rsrc_t b = buffer(s, s ? z.D * z.Dv * 4 : 0);
    const unsigned at = col < z.Dv ? (unsigned)(4 * (l >> 4) * z.Dv + col) * 4 : kNowhere;
#pragma unroll
    for (int k = 0; k < DT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[k][r] = value_of<float>(load_raw<float>(b, at + (16 * k + r) * z.Dv * 4));
}
template <int DT> __device__ __forceinline__ void store_state(int l, const Sizes &z, float *s, int col, const f32x4 (&S)[DT])
{
    const __amdgpu_buffer_rsrc_t b = buffer(s, z.D * z.Dv * 4);
    const unsigned at = col < z.Dv ? (unsigned)(4 * (l >> 4) * z.Dv + col) * 4 : kNowhere;
#pragma unroll
    for (int k = 0; k < DT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) store<float>(S[k][r], b, at + (16 * k + r) * z.Dv * 4);
}
// 16 columns of the chunk's rows of v, o or their gradients, [.., Dv] from p on; rows from `live` on are not read, and written as zeros.
struct Raw {
    unsigned x[4][4];
};
template <typename T> __device__ __forceinline__ unsigned row_bytes(const Sizes &z, long long stride, int rows)
{
    return rows <= 0 ? 0 : (unsigned)(((rows < 16 ? rows : 16) - 1) * stride + z.Dv) * (unsigned)sizeof(T);
}
template <typename T> __device__ __forceinline__ void load_rows(int l, const Sizes &z, const T *p, long long stride, int live, int col, Raw &X)
{
    const unsigned by = (unsigned)stride * (unsigned)sizeof(T), at = col < z.Dv ? 4 * (l >> 4) * by + col * (unsigned)sizeof(T) : kNowhere;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const __amdgpu_buffer_rsrc_t m = buffer(p + 16 * b * stride, p ? row_bytes<T>(z, stride, live - 16 * b) : 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) X.x[b][r] = load_raw<T>(m, at + r * by);
    }
}
template <typename T> __device__ __forceinline__ void values_of(const Raw &raw, f32x4 (&X)[4])
{
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) X[b][r] = value_of<T>(raw.x[b][r]);
}
template <typename T> __device__ __forceinline__ void store_rows(int l, const Sizes &z, T *p, long long stride, int live, int rows, int col, const f32x4 (&X)[4])
{
    const unsigned by = (unsigned)stride * (unsigned)sizeof(T), at = col < z.Dv ? 4 * (l >> 4) * by + col * (unsigned)sizeof(T) : kNowhere;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const __amdgpu_buffer_rsrc_t m = buffer(p + 16 * b * stride, row_bytes<T>(z, stride, rows - 16 * b));
#pragma unroll
        for (int r = 0; r < 4; ++r) store<T>(16 * b + 4 * (l >> 4) + r < live ? X[b][r] : 0.f, m, at + r * by);
    }
}
// Four columns of a row of a matrix [rows, columns] in memory, as an operand's fragment: row row0 + l % 16, columns k0 + 4 (l / 16) and the next.
__device__ __forceinline__ f32x4 frag_of(int l, const float *m, int rows, int row0, int columns, int k0, bool vec)
{
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    const __amdgpu_buffer_rsrc_t b = buffer(m, rows * columns * 4);
    const int k = k0 + 4 * (l >> 4);
    const unsigned at = (unsigned)((row0 + (l & 15)) * columns + k) * 4;
    if (vec) return __builtin_bit_cast(f32x4, (u32x4)__builtin_amdgcn_raw_buffer_load_b128(b, k < columns ? at : kNowhere, 0, 0));
    f32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = value_of<float>(load_raw<float>(b, k + e < columns ? at + 4 * e : kNowhere));
    return x;
}

template <typename T, int DT> struct Shared {
    static constexpr int DP = 16 * DT, LD = row_of<T>(DP);
    alignas(16) T K[kC * LD];
    alignas(16) T Q[kC * LD];
    alignas(16) float A[kC * kLA], P[kC * kLA];
    Gates g;
    alignas(16) Lengths lengths;
};

// beta (V - exp(c) K S), in place of V
template <typename T, int DT> __device__ __forceinline__ void below_state(int l, const Shared<T, DT> &s, const Operand<T, DT> &S, f32x4 (&X)[4])
{
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const f32x4 acc = in_products<T>(l, times(l, s.K, s.LD, 16 * b, S, (f32x4){0.f, 0.f, 0.f, 0.f}), s.lengths.k, 16 * b);
        X[b] = rows_of(l, s.g.beta, 16 * b) * (X[b] - rows_of(l, s.g.in, 16 * b) * acc);
        fence();
    }
}
// exp(c) Q S + P U
template <typename T, int DT> __device__ __forceinline__ void answers(int l, const Shared<T, DT> &s, const Operand<T, DT> &S, const f32x4 (&U)[4], f32x4 (&O)[4])
{
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        O[b] = rows_of(l, s.g.in, 16 * b) * in_products<T>(l, times(l, s.Q, s.LD, 16 * b, S, (f32x4){0.f, 0.f, 0.f, 0.f}), s.lengths.unit_q, 16 * b);
#pragma unroll
        for (int j = 0; j <= b; ++j) O[b] = multiply(frag(l, s.P, kLA, 16 * b, 16 * j), U[j], O[b]);
        fence();
    }
}

// ----------------------------------------------------------------------------- all steps
// A block takes the columns of a state that its wavefronts hold, 16 each, through all chunks.  Bound by the chain within a chunk (load, products, inverse, solution, products), 10 to 13 us of it:
// T=1024, heads of 128 x 128 in bf16, 198 us for 40 of them and 229 for 192; fp32 343 for 40.
template <typename T, int DT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void delta_fwd_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths, const float *__restrict__ h0,
                                                            T *__restrict__ o, float *__restrict__ h_last, float *__restrict__ saved)
{
    typedef Shared<T, DT> Lds;
    constexpr int DP = Lds::DP;
    constexpr int LD = Lds::LD;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Lds &s = *(Lds *)lds;
    const int n = blockIdx.x / z.H, h = blockIdx.x - n * z.H, hk = h / (z.H / z.Hk), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int l = fresh_lane();
    const int col = (blockIdx.y * NW + wave) * 16 + (l & 15);
    const int len = steps_of(z, lengths, n);
    const size_t own = state_at(z, 0, n, h);
    f32x4 S[DT];
    load_state(l, z, h0 ? h0 + own : nullptr, col, S);
    // a chunk's rows are on their way while the chunk in front of it is worked on
    KeyParts<T, DP, NW * 64> keys;
    GateParts<T> gates;
    Raw v;
    auto fetch = [&](int c) {
        const int t0 = c * kC, live = len - t0 < kC ? len - t0 : kC;
        const T *row0 = gi + t0 * z.gi_t + n * z.gi_n;
        keys.load(l, wave, z, row0, hk, live);
        if (wave == 0) gates.load(l, z, row0, h, live);
        load_rows(l, z, row0 + v_at(z, h), z.gi_t, live, col, v);
    };
    if (len > 0) fetch(0);
    for (int c = 0; c < z.chunks; ++c) {
        l = fresh_lane();
        const int t0 = c * kC, live = len - t0 < kC ? len - t0 : kC, rows = z.T - t0 < kC ? z.T - t0 : kC;
        if (saved) store_state(l, z, saved + state_at(z, c, n, h), col, S);
        T *out = o ? o + t0 * z.o_t + n * z.o_n + h * z.Dv : nullptr;
        f32x4 X[4] = {};
        if (live <= 0) {
            if (o) store_rows(l, z, out, z.o_t, 0, rows, col, X);
            continue;
        }
        lds_barrier();
        keys.finish(l, wave, z, s.K, s.Q, s.lengths);
        if (wave == 0) gates.finish(l, z, bias, h, live, s.g);
        values_of<T>(v, X);
        if (t0 + kC < len) fetch(c + 1);
        fence();
        lds_barrier();
        {
            f32x4 tiles[(2 * kTiles + NW - 1) / NW];
            make_tiles<T, DP, NW, 2 * kTiles>(l, wave, s.g, s.lengths, s.K, s.Q, s.A, s.P, tiles);
        }
        lds_barrier();
        if (wave < 4) invert_block(l, s.A, wave);
        Operand<T, DT> state;
        state.set(S);
        below_state(l, s, state, X);
        lds_barrier();
        solve(l, s.A, X);
        settle(X);
        if (o) {
            f32x4 O[4];
            answers(l, s, state, X, O);
            store_rows(l, z, out, z.o_t, live, rows, col, O);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) X[b] *= in_products<T>(l, rows_of(l, s.g.out, 16 * b), s.lengths.k, 16 * b);
        Operand<T, 4> written;
        written.set(X);
        const float all = s.g.all;
#pragma unroll
        for (int k = 0; k < DT; ++k) {
            S[k] = times_t(l, s.K, LD, 16 * k, written, S[k] * all);
            if (k & 1) fence();
        }
        settle(S);
    }
    if (h_last) store_state(l, z, h_last + own, col, S);
}

// The same where the columns of a head fit four wavefronts and LDS two chunks: four more wavefronts prepare the next chunk (K, Q, A, P, the inverses, none of which needs a state) while the
// first four go through this one.  Both meet three times a chunk, where the others' stages are about as long.  T=2048, heads of 64 x 64 in bf16, with it / without: 256 heads 199 / 302 us, 384
// (two rounds of blocks, as two chunks leave room for one block on a compute unit, where without there are two) 379 / 381; T=200 in fp32, 200 heads, 44 / 53.  What a chunk of 64 steps takes,
// 6 us, is the chain of its products: the matrix unit is busy a fifth of it, the vector unit (pieces, decays) 28 percent.
template <typename T, int DT> struct Preparing {
    static constexpr int DP = 16 * DT, WAVES = 4;
    KeyParts<T, DP, WAVES * 64> keys;
    GateParts<T> gates;
    __device__ __forceinline__ void load(int l, int wave, const Sizes &z, const T *row0, int h, int hk, int live)
    {
        keys.load(l, wave, z, row0, hk, live);
        if (wave == 0) gates.load(l, z, row0, h, live);
    }
    __device__ __forceinline__ void rows(int l, int wave, const Sizes &z, const float *bias, int h, int live, Shared<T, DT> &s) const
    {
        keys.finish(l, wave, z, s.K, s.Q, s.lengths);
        if (wave == 0) gates.finish(l, z, bias, h, live, s.g);
    }
    static __device__ __forceinline__ void tiles(int l, int wave, Shared<T, DT> &s)
    {
        f32x4 x[2 * kTiles / WAVES];
        make_tiles<T, DP, WAVES, 2 * kTiles>(l, wave, s.g, s.lengths, s.K, s.Q, s.A, s.P, x);
    }
};
template <typename T, int DT> constexpr bool kFlows = 2 * sizeof(Shared<T, DT>) <= 160 * 1024;
constexpr int kFlowThreads = 512;
// The preparing wavefronts' part, for chunk(i), i = 0, 1, .. count - 1.
template <typename T, int DT, typename F>
__device__ __forceinline__ void prepare(const Sizes &z, int wave, const T *rows, const float *bias, int h, int hk, int len, int count, Shared<T, DT> *s, F &&chunk)
{
    Preparing<T, DT> p;
    auto live = [&](int i) { return len - chunk(i) * kC < kC ? len - chunk(i) * kC : kC; };
    auto row0 = [&](int i) { return rows + chunk(i) * kC * z.gi_t; };
    if (count > 0) p.load(fresh_lane(), wave, z, row0(0), h, hk, live(0));
    for (int i = 0; i <= count; ++i) {          // (in step i chunk i is prepared, and the others go through chunk i - 1)
        const int l = fresh_lane();
        const bool there = i < count;
        Shared<T, DT> &to = s[i & 1];
        if (there) p.rows(l, wave, z, bias, h, live(i), to);
        if (i + 1 < count) p.load(l, wave, z, row0(i + 1), h, hk, live(i + 1));
        fence();
        lds_barrier();
        if (there) p.tiles(l, wave, to);
        lds_barrier();
        if (there) invert_block(l, to.A, wave);
        lds_barrier();
    }
}
template <typename T, int DT>
__global__ __launch_bounds__(kFlowThreads, 2) void delta_flow_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths, const float *__restrict__ h0,
                                                                     T *__restrict__ o, float *__restrict__ h_last, float *__restrict__ saved)
{
    typedef Shared<T, DT> Lds;
    constexpr int LD = Lds::LD;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Lds *both_s = (Lds *)lds;
    const int n = blockIdx.x / z.H, h = blockIdx.x - n * z.H, hk = h / (z.H / z.Hk), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = steps_of(z, lengths, n), used = (len + kC - 1) / kC;
    const T *rows0 = gi + n * z.gi_n;
    if (wave >= 4) return prepare<T, DT>(z, wave - 4, rows0, bias, h, hk, len, used, both_s, [](int i) { return i; });
    int l = fresh_lane();
    const int col = (blockIdx.y * 4 + wave) * 16 + (l & 15);
    const size_t own = state_at(z, 0, n, h);
    f32x4 S[DT];
    load_state(l, z, h0 ? h0 + own : nullptr, col, S);
    Raw v;
    auto fetch = [&](int c) { load_rows(l, z, rows0 + c * kC * z.gi_t + v_at(z, h), z.gi_t, len - c * kC < kC ? len - c * kC : kC, col, v); };
    if (used > 0) fetch(0);
    lds_barrier();
    lds_barrier();
    lds_barrier();
    for (int c = 0; c < used; ++c) {
        l = fresh_lane();
        const int t0 = c * kC, live = len - t0 < kC ? len - t0 : kC, rows = z.T - t0 < kC ? z.T - t0 : kC;
        const Lds &s = both_s[c & 1];
        if (saved) store_state(l, z, saved + state_at(z, c, n, h), col, S);
        f32x4 X[4];
        values_of<T>(v, X);
        if (c + 1 < used) fetch(c + 1);
        Operand<T, DT> state;
        state.set(S);
        below_state(l, s, state, X);
        settle(X);
        lds_barrier();
        solve(l, s.A, X);
        settle(X);
        if (o) {
            f32x4 O[4];
            answers(l, s, state, X, O);
            store_rows(l, z, o + t0 * z.o_t + n * z.o_n + h * z.Dv, z.o_t, live, rows, col, O);
        }
        lds_barrier();
#pragma unroll
        for (int b = 0; b < 4; ++b) X[b] *= in_products<T>(l, rows_of(l, s.g.out, 16 * b), s.lengths.k, 16 * b);
        Operand<T, 4> written;
        written.set(X);
        const float all = s.g.all;
#pragma unroll
        for (int k = 0; k < DT; ++k) {
            S[k] = times_t(l, s.K, LD, 16 * k, written, S[k] * all);
            if (k & 1) fence();
        }
        settle(S);
        lds_barrier();
    }
    for (int c = used; c < z.chunks; ++c) {
        const int t0 = c * kC;
        const f32x4 X[4] = {};
        if (saved) store_state(l, z, saved + state_at(z, c, n, h), col, S);
        if (o) store_rows(l, z, o + t0 * z.o_t + n * z.o_n + h * z.Dv, z.o_t, 0, z.T - t0 < kC ? z.T - t0 : kC, col, X);
    }
    if (h_last) store_state(l, z, h_last + own, col, S);
}

// ----------------------------------------------------------------------------- all chunks at once
// A chunk takes S to M S + B, and the gradient behind it to M^T G + B'.  Where heads are few, the chunks' M and B are made beside each other (the products above for a state of
// D + Dv columns, the unit matrix and zeros), then a small product a chunk goes through the sequence, and then everything else is done for all chunks beside each other.
// T=16384, 4 heads of 128 x 128 in bf16, us: matrices 60, of which the 134 MB that they write are 26; Compose 94, Jump 35, Fill 54; answers 41 (4 TB/s).  The products of Compose and Fill have to be
// on the fp32 unit (M and the state both have 32 bits), which is busy half of their time.
__host__ __device__ __forceinline__ size_t matrices_at(const Sizes &z, int chunk, int n, int h) { return (((size_t)chunk * z.N + n) * z.H + h) * z.D * (z.D + z.Dv); }

template <typename T, int DT, int NW, bool BACK>
__global__ __launch_bounds__(NW * 64) void delta_matrices_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths, const T *__restrict__ d_o,
                                                                 float *__restrict__ matrices)
{
    typedef Shared<T, DT> Lds;
    constexpr int DP = Lds::DP;
    constexpr int LD = Lds::LD;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Lds &s = *(Lds *)lds;
    const int c = blockIdx.x / (z.N * z.H), rest = blockIdx.x - c * (z.N * z.H), n = rest / z.H, h = rest - n * z.H, hk = h / (z.H / z.Hk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = fresh_lane(), lc = l & 15, g4 = 4 * (l >> 4);
    const int t0 = c * kC, len = steps_of(z, lengths, n), live = len - t0 < kC ? len - t0 : kC;
    if (live <= 0) return;
    // this wavefront's columns: of the unit matrix in front, or of v (or the gradient of o)
    const int units = (z.D + 15) / 16, tile = blockIdx.y * NW + wave;
    const bool unit = tile < units;
    const int col = (unit ? tile : tile - units) * 16 + lc;
    const T *row0 = gi + t0 * z.gi_t + n * z.gi_n;
    KeyParts<T, DP, NW * 64> keys;
    keys.load(l, wave, z, row0, hk, live);
    Raw raw;
    if (BACK) load_rows(l, z, d_o ? d_o + t0 * z.o_t + n * z.o_n + h * z.Dv : nullptr, z.o_t, live, unit ? z.Dv : col, raw);
    else load_rows(l, z, row0 + v_at(z, h), z.gi_t, live, unit ? z.Dv : col, raw);
    if (wave == 0) load_gates(l, z, row0, bias, h, live, s.g);
    keys.finish(l, wave, z, s.K, s.Q, s.lengths);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    lds_barrier();
    {
        constexpr int TILES = (BACK ? 2 : 1) * kTiles;
        f32x4 tiles[(TILES + NW - 1) / NW];
        make_tiles<T, DP, NW, TILES>(l, wave, s.g, s.lengths, s.K, s.Q, s.A, s.P, tiles);
    }
    lds_barrier();
    if (wave < 4) invert_block(l, s.A, wave);
    lds_barrier();
    f32x4 V[4];
    values_of<T>(raw, V);
    f32x4 X[4];
    if (unit) {                         // the product of K and the unit matrix
#pragma unroll
        for (int b = 0; b < 4; ++b) {
#pragma unroll
            for (int r = 0; r < 4; ++r) X[b][r] = (float)s.K[(16 * b + g4 + r) * LD + col];
            X[b] = in_products<T>(l, X[b], s.lengths.k, 16 * b);
            X[b] *= BACK ? rows_of(l, s.g.out, 16 * b) : -rows_of(l, s.g.in, 16 * b) * rows_of(l, s.g.beta, 16 * b);
        }
    } else if (!BACK) {
#pragma unroll
        for (int b = 0; b < 4; ++b) X[b] = rows_of(l, s.g.beta, 16 * b) * V[b];
    } else {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            X[b] = zero;
#pragma unroll
            for (int i = b; i < 4; ++i) X[b] = multiply(frag_t(l, s.P, kLA, 16 * b, 16 * i), V[i], X[b]);
        }
        settle(X);
    }
    if (BACK) solve_t(l, s.A, X);
    else solve(l, s.A, X);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const f32x4 in = rows_of(l, s.g.in, 16 * b);
        if (BACK) V[b] *= in_products<T>(l, in, s.lengths.unit_q, 16 * b);
        X[b] *= in_products<T>(l, BACK ? -in * rows_of(l, s.g.beta, 16 * b) : rows_of(l, s.g.out, 16 * b), s.lengths.k, 16 * b);
    }
    Operand<T, 4> written, asked;
    written.set(X);
    if (BACK) asked.set(V);
    const float all = s.g.all;
    const int width = unit ? z.D : z.Dv;
    float *m = matrices + matrices_at(z, c, n, h) + (unit ? 0 : (size_t)z.D * z.D) + col;
#pragma unroll
    for (int k = 0; k < DT; ++k) {
        f32x4 acc;
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = unit && 16 * k + g4 + r == col ? all : 0.f;
        if (BACK) acc = times_t(l, s.Q, LD, 16 * k, asked, acc);       // (zeros in the unit matrix's columns)
        acc = times_t(l, s.K, LD, 16 * k, written, acc);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (16 * k + g4 + r < z.D && col < width) m[(size_t)(16 * k + g4 + r) * width] = acc[r];
        fence();
    }
}

// States in front of the chunks (BACK: gradients behind them, from the last chunk on) to `states`, and the last one to `last`.  A block takes 16 columns of a state, a wavefront 16
// rows; the state goes round through LDS, a column in a row.  What the next chunk needs is on its way meanwhile.
// A chunk takes 2 us, which nothing hides where the blocks are few and the sequence long.  Then it is cut into segments (blockIdx.z): Compose makes the M and B of each, the columns of the
// unit matrix and of no state; Jump goes from segment to segment; Fill goes through each from the state that enters it.
enum class Scan { Whole, Compose, Jump, Fill };
// Where blocks are many, one takes two groups of 16 columns and reads M once for both (T=16384, N=1, 4 heads of 128 x 128, us of Compose / Fill with one group 133 / 69, with two 97 / 56).
template <Scan MODE> constexpr int kColumnTiles = MODE == Scan::Compose || MODE == Scan::Fill ? 2 : 1;
template <int DT, bool BACK, Scan MODE>
__global__ __launch_bounds__(DT * 64) void delta_scan_kernel(Sizes z, const int *__restrict__ lengths, const float *__restrict__ matrices, const float *__restrict__ first,
                                                             float *__restrict__ states, float *__restrict__ last, int segment)
{
    constexpr int DP = 16 * DT, LD = DP + 4, CT = kColumnTiles<MODE>;
    constexpr bool CUT = MODE == Scan::Compose || MODE == Scan::Fill;
    __shared__ __attribute__((aligned(16))) float lds[2][CT][16 * LD];
    const int n = blockIdx.x / z.H, h = blockIdx.x - n * z.H, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = fresh_lane(), lc = l & 15, g4 = 4 * (l >> 4);
    const int units = (z.D + 15) / 16, len = steps_of(z, lengths, n), used = (len + kC - 1) / kC, row = 16 * wave + g4;
    const bool vec = z.D % 4 == 0;
    // the items of the sequence (chunks, or segments) that this block goes through
    const int items = MODE == Scan::Jump ? (used + segment - 1) / segment : used, number = CUT ? blockIdx.z : 0, from = CUT ? number * segment : 0;
    const int to = CUT && items - from > segment ? from + segment : items;
    const bool ends = to >= items;
    if (from >= items && (MODE == Scan::Compose || from > 0)) return;
    if (MODE == Scan::Compose && ends) return;          // (nothing comes behind it)
    const size_t own = state_at(z, 0, n, h);
    f32x4 S[CT];
    struct Chunk {
        f32x4 M[DT], B[CT];
    };
    Chunk chunk[2];
    // each group's columns: of the unit matrix in front (Compose), or of the state
    bool unit[CT];
    int col[CT], width[CT];
    unsigned at[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        const int tile = blockIdx.y * CT + t;
        unit[t] = MODE == Scan::Compose && tile < units;
        col[t] = (MODE == Scan::Compose && !unit[t] ? tile - units : tile) * 16 + lc;
        width[t] = unit[t] ? z.D : z.Dv;
        at[t] = col[t] < width[t] ? (unsigned)(row * width[t] + col[t]) * 4 : kNowhere;
    }
    auto get = [&](const float *p, int t, f32x4 &x) {
        const __amdgpu_buffer_rsrc_t b = buffer(p, p ? z.D * width[t] * 4 : 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = value_of<float>(load_raw<float>(b, at[t] + r * width[t] * 4));
    };
    auto put = [&](float *p, int t) {
        const __amdgpu_buffer_rsrc_t b = buffer(p, z.D * width[t] * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) store<float>(S[t][r], b, at[t] + r * width[t] * 4);
    };
    auto put_all = [&](float *p) {
#pragma unroll
        for (int t = 0; t < CT; ++t) put(p, t);
    };
    auto item = [&](int i) { return BACK && MODE != Scan::Jump ? used - 1 - i : i; };
    auto fetch = [&](int i, Chunk &x) {
        const float *m = matrices + matrices_at(z, item(i), n, h);
#pragma unroll
        for (int k = 0; k < DT; ++k) x.M[k] = frag_of(l, m, z.D, 16 * wave, z.D, 16 * k, vec);
#pragma unroll
        for (int t = 0; t < CT; ++t) get(unit[t] ? nullptr : m + (size_t)z.D * z.D, t, x.B[t]);
    };
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        if (MODE == Scan::Compose) {
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = unit[t] && row + r == col[t] ? 1.f : 0.f;
        } else {
            get(MODE == Scan::Fill ? first + state_at(z, number, n, h) : first ? first + own : nullptr, t, S[t]);
        }
    }
    // the last product only if what it makes is wanted
    const int stop = MODE == Scan::Compose || (ends && last) ? to : to - 1;
    auto step = [&](int i, const Chunk &now, Chunk &next) {
        if (MODE != Scan::Compose) put_all(states + state_at(z, item(i), n, h));
        if (i >= stop) return;
        if (i + 1 < stop) fetch(i + 1, next);
#pragma unroll
        for (int t = 0; t < CT; ++t) *(f32x4 *)(lds[i & 1][t] + lc * LD + row) = S[t];
        lds_barrier();
        f32x4 acc[2 * CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            acc[2 * t] = now.B[t];
            acc[2 * t + 1] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int k = 0; k < DT; ++k)
#pragma unroll
            for (int t = 0; t < CT; ++t) acc[2 * t + (k & 1)] = multiply(now.M[k], *(const f32x4 *)(lds[i & 1][t] + lc * LD + 16 * k + g4), acc[2 * t + (k & 1)]);
        settle(acc);
#pragma unroll
        for (int t = 0; t < CT; ++t) S[t] = acc[2 * t] + acc[2 * t + 1];
    };
    if (stop > from) fetch(from, chunk[0]);
    for (int i = from; i < to; i += 2) {
        step(i, chunk[0], chunk[1]);
        if (i + 1 < to) step(i + 1, chunk[1], chunk[0]);
    }
    if (MODE == Scan::Compose) {
#pragma unroll
        for (int t = 0; t < CT; ++t) put(states + matrices_at(z, number, n, h) + (unit[t] ? 0 : (size_t)z.D * z.D), t);
        return;
    }
    if (MODE == Scan::Jump && items == 0) put_all(states + state_at(z, 0, n, h));        // (a sequence of no step: what enters it leaves it)
    if (MODE == Scan::Jump || !ends) return;
    if (!BACK)
        for (int c = used; c < z.chunks; ++c) put_all(states + state_at(z, c, n, h));
    if (last) put_all(last + own);
}

// What the chunks answer, given the states in front of them.
template <typename T, int DT, int NW>
__global__ __launch_bounds__(NW * 64) void delta_out_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths, const float *__restrict__ states,
                                                            T *__restrict__ o)
{
    typedef Shared<T, DT> Lds;
    constexpr int DP = Lds::DP;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Lds &s = *(Lds *)lds;
    const int c = blockIdx.x / (z.N * z.H), rest = blockIdx.x - c * (z.N * z.H), n = rest / z.H, h = rest - n * z.H, hk = h / (z.H / z.Hk);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = fresh_lane(), col = (blockIdx.y * NW + wave) * 16 + (l & 15);
    const int t0 = c * kC, len = steps_of(z, lengths, n), live = len - t0 < kC ? len - t0 : kC, rows = z.T - t0 < kC ? z.T - t0 : kC;
    T *out = o + t0 * z.o_t + n * z.o_n + h * z.Dv;
    f32x4 X[4] = {}, S[DT];
    if (live <= 0) return store_rows(l, z, out, z.o_t, 0, rows, col, X);
    const T *row0 = gi + t0 * z.gi_t + n * z.gi_n;
    KeyParts<T, DP, NW * 64> keys;
    keys.load(l, wave, z, row0, hk, live);
    Raw raw;
    load_rows(l, z, row0 + v_at(z, h), z.gi_t, live, col, raw);
    load_state(l, z, states + state_at(z, c, n, h), col, S);
    if (wave == 0) load_gates(l, z, row0, bias, h, live, s.g);
    keys.finish(l, wave, z, s.K, s.Q, s.lengths);
    lds_barrier();
    {
        f32x4 tiles[(2 * kTiles + NW - 1) / NW];
        make_tiles<T, DP, NW, 2 * kTiles>(l, wave, s.g, s.lengths, s.K, s.Q, s.A, s.P, tiles);
    }
    lds_barrier();
    if (wave < 4) invert_block(l, s.A, wave);
    values_of<T>(raw, X);
    Operand<T, DT> state;
    state.set(S);
    below_state(l, s, state, X);
    lds_barrier();
    solve(l, s.A, X);
    f32x4 O[4];
    answers(l, s, state, X, O);
    settle(O);
    store_rows(l, z, out, z.o_t, live, rows, col, O);
}

// ----------------------------------------------------------------------------- backwards
// The gradients of the states that leave the chunks, from the last to the first, and of the initial state.
template <typename T, int DT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void delta_ends_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths, const T *__restrict__ d_o,
                                                             const float *__restrict__ dh_last, float *__restrict__ dh0, float *__restrict__ ends)
{
    typedef Shared<T, DT> Lds;
    constexpr int DP = Lds::DP;
    constexpr int LD = Lds::LD;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Lds &s = *(Lds *)lds;
    const int n = blockIdx.x / z.H, h = blockIdx.x - n * z.H, hk = h / (z.H / z.Hk), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int l = fresh_lane();
    const int col = (blockIdx.y * NW + wave) * 16 + (l & 15);
    const int len = steps_of(z, lengths, n);
    const size_t own = state_at(z, 0, n, h);
    f32x4 G[DT];
    load_state(l, z, dh_last ? dh_last + own : nullptr, col, G);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    KeyParts<T, DP, NW * 64> keys;
    GateParts<T> gates;
    Raw raw;
    auto fetch = [&](int c) {
        const int t0 = c * kC, live = len - t0 < kC ? len - t0 : kC;
        const T *row0 = gi + t0 * z.gi_t + n * z.gi_n;
        keys.load(l, wave, z, row0, hk, live);
        if (wave == 0) gates.load(l, z, row0, h, live);
        load_rows(l, z, d_o ? d_o + t0 * z.o_t + n * z.o_n + h * z.Dv : nullptr, z.o_t, live, col, raw);
    };
    const int used = (len + kC - 1) / kC;
    if (used > 0) fetch(used - 1);
    for (int c = used - 1; c >= 0; --c) {
        l = fresh_lane();
        const int t0 = c * kC, live = len - t0 < kC ? len - t0 : kC;
        store_state(l, z, ends + state_at(z, c, n, h), col, G);
        if (c == 0 && !dh0) break;
        lds_barrier();
        keys.finish(l, wave, z, s.K, s.Q, s.lengths);
        if (wave == 0) gates.finish(l, z, bias, h, live, s.g);
        f32x4 dO[4];
        values_of<T>(raw, dO);
        if (c > 0) fetch(c - 1);
        fence();
        lds_barrier();
        {
            f32x4 tiles[(2 * kTiles + NW - 1) / NW];
            make_tiles<T, DP, NW, 2 * kTiles>(l, wave, s.g, s.lengths, s.K, s.Q, s.A, s.P, tiles);
        }
        lds_barrier();
        if (wave < 4) invert_block(l, s.A, wave);
        f32x4 X[4];
        Operand<T, DT> behind;
        behind.set(G);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            X[b] = rows_of(l, s.g.out, 16 * b) * in_products<T>(l, times(l, s.K, LD, 16 * b, behind, zero), s.lengths.k, 16 * b);
#pragma unroll
            for (int i = b; i < 4; ++i) X[b] = multiply(frag_t(l, s.P, kLA, 16 * b, 16 * i), dO[i], X[b]);
            fence();
        }
        lds_barrier();
        solve_t(l, s.A, X);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 in = rows_of(l, s.g.in, 16 * b);
            dO[b] *= in_products<T>(l, in, s.lengths.unit_q, 16 * b);
            X[b] *= in_products<T>(l, -in * rows_of(l, s.g.beta, 16 * b), s.lengths.k, 16 * b);
        }
        Operand<T, 4> asked, written;
        asked.set(dO);
        written.set(X);
        const float all = s.g.all;
#pragma unroll
        for (int k = 0; k < DT; ++k) {
            G[k] = times_t(l, s.K, LD, 16 * k, written, times_t(l, s.Q, LD, 16 * k, asked, G[k] * all));
            if (k & 1) fence();
        }
        settle(G);
    }
    if (dh0) store_state(l, z, dh0 + own, col, G);
}

// The same with the next chunk prepared meanwhile.
template <typename T, int DT>
__global__ __launch_bounds__(kFlowThreads, 2) void delta_ends_flow_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                                          const T *__restrict__ d_o, const float *__restrict__ dh_last, float *__restrict__ dh0, float *__restrict__ ends)
{
    typedef Shared<T, DT> Lds;
    constexpr int LD = Lds::LD;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Lds *both_s = (Lds *)lds;
    const int n = blockIdx.x / z.H, h = blockIdx.x - n * z.H, hk = h / (z.H / z.Hk), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = steps_of(z, lengths, n), used = (len + kC - 1) / kC, count = dh0 ? used : used - 1;       // the first chunk's product is that of dh0
    auto chunk = [&](int i) { return used - 1 - i; };
    if (wave >= 4) return prepare<T, DT>(z, wave - 4, gi + n * z.gi_n, bias, h, hk, len, count, both_s, chunk);
    int l = fresh_lane();
    const int col = (blockIdx.y * 4 + wave) * 16 + (l & 15);
    const size_t own = state_at(z, 0, n, h);
    f32x4 G[DT];
    load_state(l, z, dh_last ? dh_last + own : nullptr, col, G);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    Raw raw;
    auto fetch = [&](int i) {
        const int t0 = chunk(i) * kC;
        load_rows(l, z, d_o ? d_o + t0 * z.o_t + n * z.o_n + h * z.Dv : nullptr, z.o_t, len - t0 < kC ? len - t0 : kC, col, raw);
    };
    if (count > 0) fetch(0);
    if (count >= 0) {
        lds_barrier();
        lds_barrier();
        lds_barrier();
    }
    for (int i = 0; i < count; ++i) {
        l = fresh_lane();
        const Lds &s = both_s[i & 1];
        store_state(l, z, ends + state_at(z, chunk(i), n, h), col, G);
        f32x4 dO[4], X[4];
        values_of<T>(raw, dO);
        if (i + 1 < count) fetch(i + 1);
        Operand<T, DT> behind;
        behind.set(G);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            X[b] = rows_of(l, s.g.out, 16 * b) * in_products<T>(l, times(l, s.K, LD, 16 * b, behind, zero), s.lengths.k, 16 * b);
            fence();
        }
        settle(X);
        lds_barrier();
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int j = b; j < 4; ++j) X[b] = multiply(frag_t(l, s.P, kLA, 16 * b, 16 * j), dO[j], X[b]);
        solve_t(l, s.A, X);
        settle(X);
        lds_barrier();
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 in = rows_of(l, s.g.in, 16 * b);
            dO[b] *= in_products<T>(l, in, s.lengths.unit_q, 16 * b);
            X[b] *= in_products<T>(l, -in * rows_of(l, s.g.beta, 16 * b), s.lengths.k, 16 * b);
        }
        Operand<T, 4> asked, written;
        asked.set(dO);
        written.set(X);
        const float all = s.g.all;
#pragma unroll
        for (int k = 0; k < DT; ++k) {
            G[k] = times_t(l, s.K, LD, 16 * k, written, times_t(l, s.Q, LD, 16 * k, asked, G[k] * all));
            if (k & 1) fence();
        }
        settle(G);
        lds_barrier();
    }
    if (count < used) store_state(l, z, ends + own, col, G);
    if (dh0) store_state(l, z, dh0 + own, col, G);
}

// The gradients of a chunk's rows, given the states in front of and the gradients behind it.  A block takes a key head and the heads that share it, one after the other, so that
// their gradients of q and k are summed in registers.  64 columns of the state at a time: four wavefronts make U, the other four X; then all make the products that reach over
// the columns, each a tile column of dQ and dK and its tiles of dA and dP.
// 6144 chunks of 64 x 64 in bf16 take 640 us, 24 rounds of a block a compute unit (107 KB of LDS: 53 of X, U and dO), 27 us each: eight wavefronts wait for each other at five barriers, the vector
// unit is busy 36 percent, the matrix unit 29 (dA, dP and E1 to E3 are products of two operands of 32 bits).  Loads of the states' rows before the solution instead of behind it, which would hide
// them, do not fit the registers; a block a compute unit that goes from chunk to chunk and loads the next one's rows and state behind its column loop took 670 (244 registers instead of 188).
constexpr int kGradWaves = 8;
template <typename T, int DT> struct GradShared : Shared<T, DT> {
    struct Columns {
        float X[kC * kLA], U[kC * kLA], O[kC * kLA];
    };
    // (after the columns)
    struct Sums {
        float row_a[4][kC], col_a[4][kC], row_p[4][kC], col_p[4][kC];       // of the tiles, by their other index; col of a tile on the diagonal: what its steps' gates lie in
        float dots[DT][kC], ends[DT][kC];
        float states[DT];
    };
    union {
        Columns v;
        Sums t;
    };
    float xr[4][kC];
};
template <typename T, int DT>
__global__ __launch_bounds__(kGradWaves * 64) void delta_grad_kernel(Sizes z, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ lengths,
                                                                     const float *__restrict__ saved, const T *__restrict__ d_o, const float *__restrict__ ends, T *__restrict__ dgi)
{
    typedef GradShared<T, DT> Lds;
    constexpr int DP = Lds::DP, LD = Lds::LD, NW = kGradWaves, RT = 4 * DT / NW, KEEP = (2 * kTiles + NW - 1) / NW;
    static_assert(RT >= 1, "tiles of dQ for every wavefront");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Lds &s = *(Lds *)lds;
    const int c = blockIdx.x / (z.N * z.Hk), rest = blockIdx.x - c * (z.N * z.Hk), n = rest / z.Hk, hk = rest - n * z.Hk, group = z.H / z.Hk;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int l = fresh_lane(), g4 = 4 * (l >> 4), lc = l & 15;
    auto anew = [&] {
        l = fresh_lane();
        g4 = 4 * (l >> 4);
        lc = l & 15;
    };
    const int len = steps_of(z, lengths, n), t0 = c * kC, live = len - t0 < kC ? len - t0 : kC, rows = z.T - t0 < kC ? z.T - t0 : kC;
    const T *row0 = gi + t0 * z.gi_t + n * z.gi_n;
    T *out0 = dgi + t0 * z.gi_t + n * z.gi_n;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if (live <= 0) {
        const int widths[4] = {z.D, z.D, group * z.Dv, group}, at[4] = {q_at(z, hk), k_at(z, hk), v_at(z, hk * group), a_at(z, hk * group)};
        for (int i = wave; i < rows; i += NW) {
            T *p = out0 + i * z.gi_t;
            for (int k = 0; k < 4; ++k)
                for (int e = l; e < widths[k]; e += 64) p[at[k] + e] = (T)0.f;
            for (int e = l; e < group; e += 64) p[b_at(z, hk * group) + e] = (T)0.f;
        }
        return;
    }
    {
        KeyParts<T, DP, NW * 64> keys;
        keys.load(l, wave, z, row0, hk, live);
        keys.finish(l, wave, z, s.K, s.Q, s.lengths);
    }
    // this wavefront's tiles of dQ and dK
    const int dt = wave % DT, rt0 = wave / DT * RT;
    const bool vec = z.Dv % 4 == 0;
    f32x4 dQ[RT], dK[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) dQ[i] = dK[i] = zero;
    for (int h = hk * group; h < (hk + 1) * group; ++h) {
        anew();
        const float *S0 = saved + state_at(z, c, n, h), *G0 = ends + state_at(z, c, n, h);
        const T *do0 = d_o ? d_o + t0 * z.o_t + n * z.o_n + h * z.Dv : nullptr;
        // 16 columns: v and the state in front for U, the gradients of o and of the state behind for X
        Raw raw;
        f32x4 S[DT];
        auto fetch = [&](int v0) {
            const int col = v0 + 16 * (wave & 3) + lc;
            if (wave < 4) load_rows(l, z, row0 + v_at(z, h), z.gi_t, live, col, raw);
            else load_rows(l, z, do0, z.o_t, live, col, raw);
            load_state(l, z, wave < 4 ? S0 : G0, col, S);
        };
        fetch(0);
        if (wave == 0) load_gates(l, z, row0, bias, h, live, s.g);
        lds_barrier();
        f32x4 tile[KEEP], acc[KEEP];
        make_tiles<T, DP, NW, 2 * kTiles>(l, wave, s.g, s.lengths, s.K, s.Q, s.A, s.P, tile);
#pragma unroll
        for (int i = 0; i < KEEP; ++i) acc[i] = zero;
        lds_barrier();
        if (wave < 4) invert_block(l, s.A, wave);
        f32x4 E1[RT], E2[RT], E3[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) E1[i] = E2[i] = E3[i] = zero;
        float both = 0.f;               // sum of S * G
        for (int v0 = 0; v0 < z.Dv; v0 += 64) {
            anew();
            const int mine = 16 * (wave & 3) + lc, col = v0 + mine;
            f32x4 R[4], X[4];
            values_of<T>(raw, R);
            Operand<T, DT> state;
            state.set(S);
            const int blocks = z.Dv - v0 < 64 ? (z.Dv - v0 + 15) / 16 : 4;         // of 16 columns, this time
            if ((wave & 3) >= blocks) {
#pragma unroll
                for (int b = 0; b < 4; ++b) X[b] = zero;
            } else if (wave < 4) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    X[b] = in_products<T>(l, times(l, s.K, LD, 16 * b, state, zero), s.lengths.k, 16 * b);
                    R[b] -= rows_of(l, s.g.in, 16 * b) * X[b];
                    X[b] = rows_of(l, s.g.beta, 16 * b) * R[b];
                    fence();
                }
            } else {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    X[b] = rows_of(l, s.g.out, 16 * b) * in_products<T>(l, times(l, s.K, LD, 16 * b, state, zero), s.lengths.k, 16 * b);
#pragma unroll
                    for (int i = b; i < 4; ++i) X[b] = multiply(frag_t(l, s.P, kLA, 16 * b, 16 * i), R[i], X[b]);
                    fence();
                }
                settle(X);
            }
            if (v0 == 0) lds_barrier();         // (the inverses)
            anew();
            if ((wave & 3) >= blocks) {
            } else if (wave < 4) {
                solve(l, s.A, X);
                settle(X);
            } else {
                solve_t(l, s.A, X);
                settle(X);
            }
            anew();
            auto put = [&](float *to, const f32x4 (&x)[4]) {
                to += g4 * kLA + mine;
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) to[(16 * b + r) * kLA] = x[b][r];
            };
            put(wave < 4 ? s.v.U : s.v.X, X);
            if (wave >= 4) put(s.v.O, R);
            // rows of this wavefront's tile column of S and G
            f32x4 sf[4], gf[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sf[k] = frag_of(l, S0, z.D, 16 * dt, z.Dv, v0 + 16 * k, vec);
                gf[k] = frag_of(l, G0, z.D, 16 * dt, z.Dv, v0 + 16 * k, vec);
            }
            lds_barrier();
            if (wave < 4) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    f32x4 x;
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = s.v.X[(16 * b + g4 + r) * kLA + mine] * R[b][r];
                    x = sum_columns(x);
                    if (lc == 0) {
                        f32x4 *p = (f32x4 *)&s.xr[wave][16 * b + g4];
                        *p = v0 ? *p + x : x;
                    }
                }
            } else {
#pragma unroll
                for (int b = 0; b < 4; ++b) X[b] *= rows_of(l, s.g.beta, 16 * b);
                store_rows(l, z, out0 + v_at(z, h), z.gi_t, live, rows, col, X);
            }
            if (v0 + 64 < z.Dv) fetch(v0 + 64);
#pragma unroll
            for (int i = 0; i < KEEP; ++i) {
                const int t = wave + i * NW;
                int bi, bj;
                anew();
                if (t >= 2 * kTiles) break;
                tile_at(t < kTiles ? t : t - kTiles, bi, bj);
                const float *left = t < kTiles ? s.v.X : s.v.O;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < blocks) acc[i] = multiply(frag(l, left, kLA, 16 * bi, 16 * k), frag(l, s.v.U, kLA, 16 * bj, 16 * k), acc[i]);
                fence();
            }
            anew();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= blocks) break;
                if (rt0 == 0) both += (sf[k][0] * gf[k][0] + sf[k][1] * gf[k][1]) + (sf[k][2] * gf[k][2] + sf[k][3] * gf[k][3]);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const int b = rt0 + i;
                    E1[i] = multiply(frag(l, s.v.X, kLA, 16 * b, 16 * k), sf[k], E1[i]);
                    E2[i] = multiply(frag(l, s.v.O, kLA, 16 * b, 16 * k), sf[k], E2[i]);
                    E3[i] = multiply(frag(l, s.v.U, kLA, 16 * b, 16 * k), gf[k], E3[i]);
                }
                fence();
            }
            settle(acc);
            settle(E1);
            settle(E2);
            settle(E3);
            lds_barrier();
        }
        // dA and dP, times L, in the place of A and P; the sums of dA A and dP P over rows and columns, and on the diagonal, for each step t of the tile, over its pairs j < t <= i
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const int t = wave + i * NW;
            int bi, bj;
            if (t >= 2 * kTiles) break;
            const bool is_a = t < kTiles;
            anew();
            tile_at(is_a ? t : t - kTiles, bi, bj);
            const f32x4 beta = rows_of(l, s.g.beta, 16 * bi), d = is_a ? -acc[i] : acc[i], L = decays(l, s.g, bi, bj, is_a);
            const f32x4 by_row = d * tile[i], by_col = is_a ? beta * by_row : by_row;
            const bool diagonal = bi == bj;
            f32x4 part = by_col;
            if (diagonal)               // (columns up to lc = t - 1 of the rows from t on)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float up = sum_up_to_column(by_col[r]);
                    part[r] = g4 + r > lc ? up : 0.f;
                }
            float sum = (part[0] + part[1]) + (part[2] + part[3]);
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (l < 16) (is_a ? s.t.col_a : s.t.col_p)[bi][16 * bj + (diagonal ? (l + 1) & 15 : l)] = sum;       // (nothing comes in front of the tile's first step: the last lane's sum is 0)
            const f32x4 row = sum_columns(by_row);
            if (lc == 0) *(f32x4 *)&(is_a ? s.t.row_a : s.t.row_p)[bj][16 * bi + g4] = row;
            store_tile(l, is_a ? s.A : s.P, bi, bj, is_a ? beta * d * L : d * L);
            fence();
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int b = rt0 + i;
            anew();
            const f32x4 in = rows_of(l, s.g.in, 16 * b), k1 = -in * rows_of(l, s.g.beta, 16 * b) * E1[i], q1 = in * E2[i], e = rows_of(l, s.g.out, 16 * b) * E3[i];
            f32x4 k, q;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                k[r] = (float)s.K[(16 * b + g4 + r) * LD + 16 * dt + lc];
                q[r] = (float)s.Q[(16 * b + g4 + r) * LD + 16 * dt + lc];
            }
            k = in_products<T>(l, k, s.lengths.k, 16 * b);
            q = in_products<T>(l, q, s.lengths.unit_q, 16 * b);
            const f32x4 ek = sum_columns(e * k), dot = sum_columns(k1 * k + q1 * q);
            if (lc == 0) {
                *(f32x4 *)&s.t.ends[dt][16 * b + g4] = ek;
                *(f32x4 *)&s.t.dots[dt][16 * b + g4] = dot;
            }
            dQ[i] += q1;
            dK[i] += k1 + e;
            fence();
        }
        if (rt0 == 0) {
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) both += __shfl_xor(both, o, 64);
            if (l == 0) s.t.states[dt] = both;
        }
        lds_barrier();
        anew();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4 k = rows_t(l, s.K, LD, 16 * dt, 16 * j, s.lengths.k), q = rows_t(l, s.Q, LD, 16 * dt, 16 * j, s.lengths.unit_q);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int b = rt0 + i;
                if (j <= b) {
                    dK[i] = multiply(frag(l, s.A, kLA, 16 * b, 16 * j), k, dK[i]);
                    dQ[i] = multiply(frag(l, s.P, kLA, 16 * b, 16 * j), k, dQ[i]);
                }
                if (j >= b) {
                    dK[i] = multiply(frag_t(l, s.A, kLA, 16 * b, 16 * j), k, dK[i]);
                    dK[i] = multiply(frag_t(l, s.P, kLA, 16 * b, 16 * j), q, dK[i]);
                }
            }
        }
        settle(dQ);
        settle(dK);
        if (wave == NW - 1) {           // the gates, a step a lane
            const int b = l >> 4;
            double dots = 0., ends = 0., both_all = 0.;
#pragma unroll
            for (int k = 0; k < DT; ++k) {
                ends += (double)s.t.ends[k][l];
                dots += (double)s.t.dots[k][l];
                both_all += (double)s.t.states[k];
            }
            const float beta = s.g.beta[l], xr = (s.xr[0][l] + s.xr[1][l]) + (s.xr[2][l] + s.xr[3][l]);
            // the tiles beside the diagonal: this step's row of them, its column, and those with a block between, which hold all gates of that block: tiles (2, 0) and (3, 0) by
            // their columns in the first block's lanes, (3, 0) and (3, 1) by their rows in the last one's
            float ra = 0.f;
            double by_rows = 0., by_cols = 0., far = 0.;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k <= b) ra += s.t.row_a[k][l];
                if (k < b) {
                    const double x = (double)beta * s.t.row_a[k][l] + (double)s.t.row_p[k][l];
                    by_rows += x;
                    if (b == 3 && k < 2) far += x;
                }
                if (k > b) {
                    const double x = (double)s.t.col_a[k][l] + (double)s.t.col_p[k][l];
                    by_cols += x;
                    if (b == 0 && k > 1) far += x;
                }
            }
            far += moved<0x121>(far);       // (a row turned by 1, 2, 4 and 8 lanes)
            far += moved<0x122>(far);
            far += moved<0x124>(far);
            far += moved<0x128>(far);
            far = __shfl_xor(far, 16, 64);
            double up = (double)s.t.col_a[b][l] + (double)s.t.col_p[b][l] + (double)s.g.all * both_all;
            if (b == 1 || b == 2) up += far;
            // rows from this step on, in their block and (dots) behind it: sums over the lanes turned round; rows and columns in front of it
            const double from = sums_up_to(__shfl(dots, 63 - l, 64)) + sums_in_row(__shfl(by_rows, 63 - l, 64));
            const double before = __shfl_up(ends, 1, 64);
            up += __shfl(from, 63 - l, 64) + (sums_up_to(l ? before : 0.) + sums_in_row(moved<0x111>(by_cols)));
            if (l < rows) {
                T *q = out0 + l * z.gi_t;
                q[a_at(z, h)] = (T)(l < live ? (float)up * s.g.rest_a[l] : 0.f);
                q[b_at(z, h)] = (T)(l < live ? (xr + ra) * beta * s.g.rest_b[l] : 0.f);
            }
        }
        lds_barrier();
    }
    // through the lengths: k^ = k / |k|, q^ = q / (sqrt(D) |q|)
    anew();
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        f32x4 k, q;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            k[r] = (float)s.K[(16 * (rt0 + i) + g4 + r) * LD + 16 * dt + lc];
            q[r] = (float)s.Q[(16 * (rt0 + i) + g4 + r) * LD + 16 * dt + lc];
        }
        k = in_products<T>(l, k, s.lengths.k, 16 * (rt0 + i));
        q = in_products<T>(l, q, s.lengths.unit_q, 16 * (rt0 + i));
        const f32x4 kk = sum_columns(dK[i] * k), qq = sum_columns(dQ[i] * q);
        if (lc == 0) {
            *(f32x4 *)&s.t.ends[dt][16 * (rt0 + i) + g4] = kk;
            *(f32x4 *)&s.t.dots[dt][16 * (rt0 + i) + g4] = qq;
        }
    }
    lds_barrier();
    const float width = (float)z.D, unit = 1.f / sqrtf(width);
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * (rt0 + i) + g4 + r, d = 16 * dt + lc;
            float kk = 0.f, qq = 0.f;
#pragma unroll
            for (int k = 0; k < DT; ++k) {
                kk += s.t.ends[k][row];
                qq += s.t.dots[k][row];
            }
            if (row >= rows || d >= z.D) continue;
            T *p = out0 + row * z.gi_t;
            const float k = (float)s.K[row * LD + d] * (sizeof(T) == 2 ? s.lengths.k[row] : 1.f), q = (float)s.Q[row * LD + d] * (sizeof(T) == 2 ? s.lengths.unit_q[row] : 1.f);
            p[k_at(z, hk) + d] = (T)(row < live ? s.lengths.k[row] * (dK[i][r] - k * kk) : 0.f);
            p[q_at(z, hk) + d] = (T)(row < live ? s.lengths.q[row] * unit * (dQ[i][r] - width * q * qq) : 0.f);
        }
}

// ----------------------------------------------------------------------------- one token
// A block a head's state, which is read once and kept in registers: a thread has four columns of every (256 / GROUPS)th row.  200 states of 64 x 64 take 6.7 us: a chain of the slot, the row,
// the sums of lengths, two sums over the block and the stores.
constexpr int kStepThreads = 256;
template <typename T, int GROUPS>
__global__ __launch_bounds__(kStepThreads) void delta_step_kernel(Sizes z, int S, const T *__restrict__ gi, const float *__restrict__ bias, const int *__restrict__ slots,
                                                                  float *__restrict__ state, T *__restrict__ o)
{
    constexpr int ROWS = kStepThreads / GROUPS, EACH = kMostWidth / ROWS;
    __shared__ float K[kMostWidth], Q[kMostWidth];
    __shared__ f32x4 part[2][ROWS][GROUPS];
    const int n = blockIdx.x / z.H, h = blockIdx.x - n * z.H, hk = h / (z.H / z.Hk), cg = threadIdx.x % GROUPS, rg = threadIdx.x / GROUPS, col = 4 * cg;
    const int slot = slots ? slots[n] : n;
    const T *row = gi + n * z.gi_n;
    T *out = o ? o + (size_t)n * z.H * z.Dv + h * z.Dv + col : nullptr;
    if (slot < 0 || slot >= S) {
        if (o && rg == 0)
            for (int e = 0; e < 4; ++e)
                if (col + e < z.Dv) out[e] = (T)0.f;
        return;
    }
    float *own = state + ((size_t)slot * z.H + h) * z.D * z.Dv + col;
    const bool vec = z.Dv % 4 == 0;
    f32x4 s[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int d = rg + i * ROWS;
        s[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        if (d >= z.D || col >= z.Dv) continue;
        if (vec) s[i] = *(const f32x4 *)(own + (size_t)d * z.Dv);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < z.Dv) s[i][e] = own[(size_t)d * z.Dv + e];
    }
    const float alpha = sigmoid((float)row[a_at(z, h)] + (bias ? bias[h] : 0.f)), beta = sigmoid((float)row[b_at(z, h)] + (bias ? bias[z.H + h] : 0.f));
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = col + e < z.Dv ? (float)row[v_at(z, h) + col + e] : 0.f;
    if (threadIdx.x < 128) {            // the first wavefront the key, the second the query
        const int l = threadIdx.x & 63;
        const bool key = threadIdx.x < 64;
        const T *p = row + (key ? k_at(z, hk) : q_at(z, hk));
        const float x0 = l < z.D ? (float)p[l] : 0.f, x1 = l + 64 < z.D ? (float)p[l + 64] : 0.f;
        float sum = x0 * x0 + x1 * x1;
#pragma unroll
        for (int w = 32; w > 0; w >>= 1) sum += __shfl_xor(sum, w, 64);
        const float by = (key ? 1.f : 1.f / sqrtf((float)z.D)) / sqrtf(sum + kEps);
        float *to = key ? K : Q;
        to[l] = x0 * by;
        to[l + 64] = x1 * by;
    }
    __syncthreads();
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        s[i] *= alpha;
        sum += K[rg + i * ROWS] * s[i];
    }
    part[0][rg][cg] = sum;
    __syncthreads();
    sum = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sum += part[0][r][cg];
    const f32x4 u = beta * (v - sum);
    sum = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int d = rg + i * ROWS;
        s[i] += K[d] * u;
        sum += Q[d] * s[i];
        if (d >= z.D || col >= z.Dv) continue;
        if (vec) *(f32x4 *)(own + (size_t)d * z.Dv) = s[i];
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < z.Dv) own[(size_t)d * z.Dv + e] = s[i][e];
    }
    if (!o) return;
    part[1][rg][cg] = sum;
    __syncthreads();
    if (rg) return;
    sum = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sum += part[1][r][cg];
    for (int e = 0; e < 4; ++e)
        if (col + e < z.Dv) out[e] = (T)sum[e];
}

// ----------------------------------------------------------------------------- host
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
bool heads_ok(int H, int Hk, int D, int Dv) { return H > 0 && Hk > 0 && D > 0 && Dv > 0 && H <= 1 << 20 && D <= 1 << 20 && Dv <= 1 << 20 && H % Hk == 0; }
long long width_of(int H, int Hk, int D, int Dv) { return 2LL * Hk * D + (long long)H * Dv + 2LL * H; }
int check(const nsk_delta_desc_t *desc, Sizes &z)
{
    if (!desc) return NSK_ERR_NULL;
    nsk_delta_desc_t d = *desc;
    if (d.T <= 0 || d.N <= 0 || !heads_ok(d.H, d.Hk, d.D, d.Dv) || (d.dtype != NSK_F32 && d.dtype != NSK_BF16)) return NSK_ERR_BAD_DESC;
    const long long width = width_of(d.H, d.Hk, d.D, d.Dv);
    if (width > 1 << 30 || (long long)d.N * width > (1LL << 60) / d.T) return NSK_ERR_BAD_DESC;
    if (!rows_apart(d.T, d.N, width, d.gi_t, d.gi_n) || !rows_apart(d.T, d.N, (long long)d.H * d.Dv, d.o_t, d.o_n)) return NSK_ERR_BAD_DESC;
    // (a launch has fewer than 2^32 threads)
    const long long chunks = ((long long)d.T + kC - 1) / kC;
    if (d.D > kMostWidth || d.Dv > kMostWidth || d.T > 1 << 30 || (long long)d.N * d.H >= 1LL << 22 || chunks * d.N * d.H >= 1LL << 22) return NSK_ERR_UNSUPPORTED;
    // (a single step's stride says nothing)
    if (d.T == 1) {
        d.gi_t = width;
        d.o_t = (long long)d.H * d.Dv;
    }
    if (d.gi_t >= kMostStride || d.o_t >= kMostStride) return NSK_ERR_UNSUPPORTED;
    const int whole = d.dtype == NSK_BF16 ? 8 : 4;
    const bool vec = d.D % whole == 0 && (d.T == 1 || d.gi_t % whole == 0) && (d.N == 1 || d.gi_n % whole == 0);
    z = {d.T, d.N, d.H, d.Hk, d.D, d.Dv, (int)chunks, vec, d.gi_t, d.N == 1 ? 0 : d.gi_n, d.o_t, d.N == 1 ? 0 : d.o_n};
    return NSK_OK;
}
// The workspace: the states (or gradients) of all chunks; where the chunks are taken all at once their matrices; where the sequence is cut into segments theirs, and the states between them.
// Few heads: all at once, whose time grows with the heads and their tiles, rather than a block or two a head through all chunks, whose time is the same up to 256 blocks.  us of all at once / of that
// (heads of D x Dv, bf16; T=1024 if not said):
//   64 x 64: forwards 56 heads 79 / 91, 68 95 / 91; backwards 80 216 / 228, T=2048 96 488 / 500, 112 568 / 551;  fp32 forwards 68 120 / 142, 80 141 / 144, T=200 60 35 / 41, 80 47 / 41;
//   64 x 128: forwards 44 80 / 92, 56 92 / 92; backwards 56 222 / 245, 68 280 / 279;  128 x 128: forwards 28 99 / 113, 36 141 / 112; backwards 28 198 / 227, 36 285 / 277;
//   T=8192, 24 heads forwards 745 / 860, 32 936 / 866;  32 x 32, T=512: forwards 96 36 / 45, 128 48 / 46; backwards 192 144 / 151;  16 x 16: forwards 128 75 / 84, 200 101 / 84;
//   128 x 128 in fp32, where nothing is prepared meanwhile: forwards 56 271 / 343, 72 373 / 346; backwards 72 633 / 650, 100 896 / 780.
// One or two chunks are not worth the launches.
bool at_once(const Sizes &z, int dtype, bool back)
{
    const int tiles = ceil_div(z.D, 16) + ceil_div(z.Dv, 16);
    return z.chunks > 2 && (long long)z.N * z.H * (tiles < 4 ? 4 : tiles) < (z.D <= 64 ? back ? 850 : 540 : dtype == NSK_BF16 ? 540 : 1150);
}
// Heads of more than 64 columns take two blocks with preparing wavefronts each, if both fit the chip at once, rather than one of eight wavefronts without (T=1024 forwards, us of 100 heads of
// 128 x 128 in bf16 119 / 202, of 128 heads of 64 x 128 97 / 155, in fp32 152 / 235).
bool flows(const Sizes &z) { return z.Dv <= 64 || (long long)z.N * z.H <= 128; }
// What goes without them: eight wavefronts of many such heads, and heads of which LDS does not hold two chunks.
template <typename T, int DT, int NW> constexpr bool kAlone = NW == 8 || !kFlows<T, DT>;
// (Compose and Fill take a step a chunk of a segment, Jump one a segment: of 16 chunks and more, so many that the segments are twice as many at most: 48 chunks are 3 of 16, 256 16 of 16, 1024 32 of 32.)
int segment_of(const Sizes &z)
{
    if (z.chunks < 48 || (long long)z.N * z.H * ceil_div(z.Dv, 16) > 256) return 0;
    int s = 16;
    while ((long long)z.chunks > 2LL * s * s) s *= 2;
    return s;
}
size_t saved_of(const Sizes &z);
struct Plan {
    int segment, segments;
    size_t matrices, composed, between, bytes;
};
Plan plan_of(const Sizes &z, int dtype, bool back)
{
    Plan p{};
    const bool all = at_once(z, dtype, back);
    p.segment = all ? segment_of(z) : 0;
    p.segments = p.segment ? ceil_div(z.chunks, p.segment) : 0;
    p.matrices = back || all ? align_up(saved_of(z)) : 0;
    p.composed = p.matrices + (all ? align_up(matrices_at(z, z.chunks, 0, 0) * sizeof(float)) : 0);
    p.between = p.composed + align_up(matrices_at(z, p.segments, 0, 0) * sizeof(float));
    p.bytes = p.between + align_up(state_at(z, p.segments, 0, 0) * sizeof(float));
    return p;
}
template <int DT, bool BACK> void scan(const Sizes &z, const Plan &p, const int *lengths, char *workspace, const float *first, float *states, float *last, hipStream_t st)
{
    const float *matrices = (const float *)(workspace + p.matrices);
    const unsigned heads = (unsigned)(z.N * z.H), columns = (unsigned)ceil_div(z.Dv, 16), both = columns + (unsigned)ceil_div(z.D, 16);
    const dim3 block(DT * 64);
    if (!p.segment) {
        hipLaunchKernelGGL((delta_scan_kernel<DT, BACK, Scan::Whole>), dim3(heads, columns), block, 0, st, z, lengths, matrices, first, states, last, 0);
        return;
    }
    float *composed = (float *)(workspace + p.composed), *between = (float *)(workspace + p.between);
    hipLaunchKernelGGL((delta_scan_kernel<DT, BACK, Scan::Compose>), dim3(heads, (both + kColumnTiles<Scan::Compose> - 1) / kColumnTiles<Scan::Compose>, (unsigned)p.segments), block, 0, st, z, lengths, matrices, (const float *)nullptr, composed,
                       (float *)nullptr, p.segment);
    hipLaunchKernelGGL((delta_scan_kernel<DT, BACK, Scan::Jump>), dim3(heads, columns), block, 0, st, z, lengths, composed, first, between, (float *)nullptr, p.segment);
    hipLaunchKernelGGL((delta_scan_kernel<DT, BACK, Scan::Fill>), dim3(heads, (columns + kColumnTiles<Scan::Fill> - 1) / kColumnTiles<Scan::Fill>, (unsigned)p.segments), block, 0, st, z, lengths, matrices, between, states, last, p.segment);
}
size_t saved_of(const Sizes &z) { return (size_t)z.chunks * z.N * z.H * z.D * z.Dv * sizeof(float); }

// A call with the tiles of D and the wavefronts' columns as constants.
template <typename F> int with_sizes(const Sizes &z, F &&f)
{
    auto columns = [&](auto dt) { return z.Dv <= 64 ? f(dt, std::integral_constant<int, 4>{}) : f(dt, std::integral_constant<int, 8>{}); };
    if (z.D <= 32) return columns(std::integral_constant<int, 2>{});
    if (z.D <= 64) return columns(std::integral_constant<int, 4>{});
    return columns(std::integral_constant<int, 8>{});
}

}  // namespace
}  // namespace nsk

using namespace nsk;

extern "C" {

size_t nsk_delta_saved_bytes(const nsk_delta_desc_t *desc)
{
    Sizes z;
    return check(desc, z) == NSK_OK ? saved_of(z) : 0;
}

size_t nsk_delta_workspace_bytes(const nsk_delta_desc_t *desc, int pass)
{
    Sizes z;
    if ((pass != NSK_PASS_FWD && pass != NSK_PASS_DGRAD) || check(desc, z) != NSK_OK) return 0;
    return plan_of(z, desc->dtype, pass == NSK_PASS_DGRAD).bytes;
}

int nsk_delta_fwd(const nsk_delta_desc_t *desc, const void *gi, const float *bias, const int *lengths, const float *h0, void *o, float *h_last, float *saved, void *workspace,
                  size_t workspace_bytes, void *stream)
{
    Sizes z;
    const int status = check(desc, z);
    if (status != NSK_OK) return status;
    if (!gi || (!o && !h_last)) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(lengths) || unaligned16(h0) || unaligned16(o) || unaligned16(h_last) || unaligned16(saved) || unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    const Plan p = plan_of(z, desc->dtype, false);
    if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return NSK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    float *matrices = (float *)((char *)workspace + p.matrices), *states = saved ? saved : (float *)workspace;
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        return with_sizes(z, [&](auto dt, auto nw) {
            constexpr int DT = decltype(dt)::value, NW = decltype(nw)::value;
            const size_t bytes = sizeof(Shared<T, DT>);
            int allowed = NSK_OK;
            if (at_once(z, desc->dtype, false)) {
                allowed = allow_lds<delta_matrices_kernel<T, DT, NW, false>>(bytes);
                if (allowed == NSK_OK) allowed = allow_lds<delta_out_kernel<T, DT, NW>>(bytes);
                if (allowed != NSK_OK) return allowed;
                const unsigned all = (unsigned)(z.chunks * z.N * z.H);
                hipLaunchKernelGGL((delta_matrices_kernel<T, DT, NW, false>), dim3(all, (unsigned)ceil_div(ceil_div(z.D, 16) + ceil_div(z.Dv, 16), NW)), dim3(NW * 64), bytes, st, z,
                                   (const T *)gi, bias, lengths, (const T *)nullptr, matrices);
                scan<DT, false>(z, p, lengths, (char *)workspace, h0, states, h_last, st);
                if (o)
                    hipLaunchKernelGGL((delta_out_kernel<T, DT, NW>), dim3(all, (unsigned)ceil_div(z.Dv, 16 * NW)), dim3(NW * 64), bytes, st, z, (const T *)gi, bias, lengths, states, (T *)o);
                return check_launch();
            }
            if (kFlows<T, DT> && flows(z)) {
                if constexpr (kFlows<T, DT>) {
                    allowed = allow_lds<delta_flow_kernel<T, DT>>(2 * bytes);
                    if (allowed != NSK_OK) return allowed;
                    hipLaunchKernelGGL((delta_flow_kernel<T, DT>), dim3((unsigned)(z.N * z.H), (unsigned)ceil_div(z.Dv, 64)), dim3(kFlowThreads), 2 * bytes, st, z, (const T *)gi, bias, lengths,
                                       h0, (T *)o, h_last, saved);
                }
            } else if constexpr (kAlone<T, DT, NW>) {
                allowed = allow_lds<delta_fwd_kernel<T, DT, NW>>(bytes);
                if (allowed != NSK_OK) return allowed;
                hipLaunchKernelGGL((delta_fwd_kernel<T, DT, NW>), dim3((unsigned)(z.N * z.H), (unsigned)ceil_div(z.Dv, 16 * NW)), dim3(NW * 64), bytes, st, z, (const T *)gi, bias, lengths, h0,
                                   (T *)o, h_last, saved);
            }
            return check_launch();
        });
    };
    return desc->dtype == NSK_BF16 ? launch(bf16_t{}) : launch(float{});
}

int nsk_delta_bwd(const nsk_delta_desc_t *desc, const void *gi, const float *bias, const int *lengths, const float *saved, const void *d_o, const float *dh_last, void *dgi, float *dh0,
                  void *workspace, size_t workspace_bytes, void *stream)
{
    Sizes z;
    const int status = check(desc, z);
    if (status != NSK_OK) return status;
    if (!gi || !saved || (!d_o && !dh_last) || !dgi) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(lengths) || unaligned16(saved) || unaligned16(d_o) || unaligned16(dh_last) || unaligned16(dgi) || unaligned16(dh0) ||
        unaligned16(workspace))
        return NSK_ERR_ALIGNMENT;
    const Plan p = plan_of(z, desc->dtype, true);
    if (!workspace || workspace_bytes < p.bytes) return NSK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    float *ends = (float *)workspace, *matrices = (float *)((char *)workspace + p.matrices);
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        return with_sizes(z, [&](auto dt, auto nw) {
            constexpr int DT = decltype(dt)::value, NW = decltype(nw)::value;
            const size_t bytes = sizeof(Shared<T, DT>), grad_bytes = sizeof(GradShared<T, DT>);
            static_assert(sizeof(GradShared<T, DT>) <= 160 * 1024, "what a compute unit has");
            int allowed = allow_lds<delta_grad_kernel<T, DT>>(grad_bytes);
            if (allowed != NSK_OK) return allowed;
            if (at_once(z, desc->dtype, true)) {
                allowed = allow_lds<delta_matrices_kernel<T, DT, NW, true>>(bytes);
                if (allowed != NSK_OK) return allowed;
                hipLaunchKernelGGL((delta_matrices_kernel<T, DT, NW, true>), dim3((unsigned)(z.chunks * z.N * z.H), (unsigned)ceil_div(ceil_div(z.D, 16) + ceil_div(z.Dv, 16), NW)),
                                   dim3(NW * 64), bytes, st, z, (const T *)gi, bias, lengths, (const T *)d_o, matrices);
                scan<DT, true>(z, p, lengths, (char *)workspace, dh_last, ends, dh0, st);
            } else if (kFlows<T, DT> && flows(z)) {
                if constexpr (kFlows<T, DT>) {
                    allowed = allow_lds<delta_ends_flow_kernel<T, DT>>(2 * bytes);
                    if (allowed != NSK_OK) return allowed;
                    hipLaunchKernelGGL((delta_ends_flow_kernel<T, DT>), dim3((unsigned)(z.N * z.H), (unsigned)ceil_div(z.Dv, 64)), dim3(kFlowThreads), 2 * bytes, st, z, (const T *)gi, bias, lengths,
                                       (const T *)d_o, dh_last, dh0, ends);
                }
            } else if constexpr (kAlone<T, DT, NW>) {
                allowed = allow_lds<delta_ends_kernel<T, DT, NW>>(bytes);
                if (allowed != NSK_OK) return allowed;
                hipLaunchKernelGGL((delta_ends_kernel<T, DT, NW>), dim3((unsigned)(z.N * z.H), (unsigned)ceil_div(z.Dv, 16 * NW)), dim3(NW * 64), bytes, st, z, (const T *)gi, bias, lengths,
                                   (const T *)d_o, dh_last, dh0, ends);
            }
            hipLaunchKernelGGL((delta_grad_kernel<T, DT>), dim3((unsigned)(z.chunks * z.N * z.Hk)), dim3(kGradWaves * 64), grad_bytes, st, z, (const T *)gi, bias, lengths, saved,
                               (const T *)d_o, ends, (T *)dgi);
            return check_launch();
        });
    };
    return desc->dtype == NSK_BF16 ? launch(bf16_t{}) : launch(float{});
}

int nsk_delta_step(int dtype, int N, int H, int Hk, int D, int Dv, int S, const void *gi, const float *bias, const int *slots, float *state, void *o, void *stream)
{
    if (N <= 0 || S <= 0 || !heads_ok(H, Hk, D, Dv) || width_of(H, Hk, D, Dv) > 1 << 30 || (dtype != NSK_F32 && dtype != NSK_BF16)) return NSK_ERR_BAD_DESC;
    if (!gi || !state) return NSK_ERR_NULL;
    if (unaligned16(gi) || unaligned16(bias) || unaligned16(slots) || unaligned16(state) || unaligned16(o)) return NSK_ERR_ALIGNMENT;
    if (D > kMostWidth || Dv > kMostWidth || (long long)N * H >= 1LL << 24) return NSK_ERR_UNSUPPORTED;     // (2^32 threads)
    const Sizes z{1, N, H, Hk, D, Dv, 1, 0, 0, width_of(H, Hk, D, Dv), 0, 0};
    auto launch = [&](auto one) {
        typedef decltype(one) T;
        if (Dv <= 64)
            hipLaunchKernelGGL((delta_step_kernel<T, 16>), dim3((unsigned)(N * H)), dim3(kStepThreads), 0, (hipStream_t)stream, z, S, (const T *)gi, bias, slots, state, (T *)o);
        else
            hipLaunchKernelGGL((delta_step_kernel<T, 32>), dim3((unsigned)(N * H)), dim3(kStepThreads), 0, (hipStream_t)stream, z, S, (const T *)gi, bias, slots, state, (T *)o);
    };
    if (dtype == NSK_BF16) launch(bf16_t{});
    else launch(float{});
    return check_launch();
}

}  // extern "C"
