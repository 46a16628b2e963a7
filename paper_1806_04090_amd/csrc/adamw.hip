// AdamW over many tensors, the norm of their gradients, and what 8-bit states stand for.
//
// Every element is read and written once and has about fourteen operations (some fifty, and a quarter of a Philox block, with 8-bit
// states): the bound is HBM, 28 bytes per element with 32-bit states and gradients, 16 with states in 8 bits.
// The tensors of a plan are described once on the device; a step is one launch over chunks of CHUNK elements of all of
// them (two, if both kinds of states occur).
// Parameters, gradients and states go past the caches, both ways (0.27 billion parameters with bf16 gradients and copies, 28 bytes each:
// 1.31 ms, 5.7 TB/s; through the caches 1.39; with 8-bit states 0.73 and 0.79).  That takes whole cache lines per row of lanes: with eight
// neighbouring elements per lane and half a line per store, 8-bit states were slower by two fifths past the caches than through them.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <vector>

#include "element_types.h"

namespace atomo {

namespace {

// Elements of a workgroup of 256 threads, eight per thread.  (The 62 tensors of ResNet-18, most of them short, 57 us with a norm and 8-bit
// states; 62 with 4096, 64 with 8192.)
constexpr int CHUNK = 2048;
constexpr int BLOCK8 = 128;            // elements of an 8-bit state with one scale: eight of each of 16 lanes
// Up to so many chunks a norm is one launch, of a workgroup per chunk: a ticket takes 25 ns, the second launch 2.3 us (one chunk 6.4 -> 4.1
// us, 64 chunks 6.4 -> 5.4, 128 6.3 -> 7.2).
constexpr int FEW_CHUNKS = 64;
constexpr int NORM_PARTS = 2048;       // partial sums of a norm

struct Tensor {
    float* param;
    void* copy;
    const void* grad;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    long long n;
    long long first_block;             // 8-bit blocks of the tensors in front
    int grad_type, copy_type;
    float lr_mult, weight_decay;
};

struct Chunk { int tensor, chunk; };   // elements [chunk * CHUNK, + CHUNK) of it

// What a step needs besides the tensors.  Of beta^t a kernel forms what it needs itself if t lies on the device.
struct StepArgs {
    double lr, rate, beta1, beta2;     // rate = lr / (1 - beta1^t)
    const long long* step_dev;
    const float* lr_dev;
    const float* grad_norm;
    long long step;
    uint64_t seed;
    float b1, c1, b2, c2;              // beta and 1 - beta, rounded once each from double
    float eps, root;                   // root = 1 / sqrt(1 - beta2^t)
    float max_norm, grad_scale;
    bool plain_eps;
};

__device__ double power(double x, long long t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1, x *= x)
        if (t & 1) r *= x;
    return r;
}

// What is the same for all elements of a workgroup's tensor.
struct Rates {
    float gs, rate, decay, root;
    long long step;
};

// false: the step is skipped
__device__ inline bool rates_of(const StepArgs& a, const Tensor& t, Rates& r)
{
    float coefficient = 1.0f;
    if (a.grad_norm) {
        const float norm = *a.grad_norm;
        if (!(norm <= 3.4028235e38f)) return false;              // (infinite or NaN)
        if (a.max_norm > 0.0f && norm > a.max_norm) coefficient = a.max_norm / norm;
    }
    r.gs = a.grad_scale * coefficient;
    double lr = a.lr, rate = a.rate;
    r.root = a.root;
    r.step = a.step;
    if (a.lr_dev) lr = (double)*a.lr_dev;
    if (a.step_dev) {
        const long long given = *a.step_dev;
        r.step = given < 1 ? 1 : given;
        rate = lr / (1.0 - power(a.beta1, r.step));
        r.root = (float)(1.0 / sqrt(1.0 - power(a.beta2, r.step)));
    } else if (a.lr_dev) {
        rate = lr / (1.0 - power(a.beta1, r.step));
    }
    r.rate = (float)(rate * (double)t.lr_mult);
    r.decay = (float)(lr * (double)t.lr_mult * (double)t.weight_decay);
    return true;
}

// m and v of one element.  Their products and sums are rounded each by itself, without fused multiply-adds: the 8-bit codes
// depend on the last bit, and this way they are the same as those of any program that forms the two sums in fp32.
__device__ inline void average(const StepArgs& a, const Rates& r, float g, float& m, float& v)
{
#pragma clang fp contract(off)
    g = g * r.gs;
    m = a.b1 * m + a.c1 * g;
    v = a.b2 * v + a.c2 * (g * g);
}

// What `v` has to be for the instruction's square root, which takes numbers below the smallest normal one for zero.
constexpr uint32_t SMALLEST_ROOT = 0x00800000u;

// Whether denominators are numbers that the instruction's reciprocal takes and gives as they are, whatever v is: it takes those below the
// smallest normal one for zero, and gives zero for what lies below it.  (The root with its factor is below 2^91.)
inline bool plain_eps(float eps) { return eps >= 0x1p-126f && eps <= 0x1p125f; }

// The parameters of N elements.  Root and quotient are rounded once each.  FAST: where v and eps are in their range, root and reciprocal are
// those of the hardware, off by at most one unit in the last place each, some twenty instructions per element less: the update is off by 13
// half units in all instead of 12.  8-bit states take them (0.27 billion 0.73 ms, with the exact forms 0.79), whose codes are off
// by far more; 32-bit states would gain 1.5 of 61.4 us where all lies in the last cache (ResNet-18, clipped) and nothing where it does not.
template <bool FAST, int N>
__device__ inline void update(const StepArgs& a, const Rates& r, float (&p)[N], const float (&m)[N], const float (&v)[N])
{
    const auto all = [&](auto quotient) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float step = r.rate * quotient(m[e], v[e]);
            p[e] = p[e] - (step + r.decay * p[e]);
        }
    };
    if constexpr (FAST) {
        uint32_t least = ~0u;                                    // of the v that are not zero, less one
#pragma unroll
        for (int e = 0; e < N; ++e) least = min(least, __float_as_uint(v[e]) - 1);
        if (a.plain_eps && !__any(least < SMALLEST_ROOT - 1)) {
            all([&](float x, float y) { return x * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(y) * r.root + a.eps); });
            return;
        }
    }
    all([&](float x, float y) {
        const float d = sqrtf(y) * r.root + a.eps;
        return x == 0.0f && d == 0.0f ? 0.0f : x / d;            // (an element that has had no gradient yet, with an eps of zero)
    });
}

__device__ inline f32x4 load_any4(int type, const void* base, long long i)
{
    return type == ATOMO_F32 ? load4<ATOMO_F32, true>(base, i) : type == ATOMO_BF16 ? load4<ATOMO_BF16, true>(base, i) : load4<ATOMO_F16, true>(base, i);
}

__device__ inline float load_any1(int type, const void* base, long long i)
{
    return type == ATOMO_F32 ? load1<ATOMO_F32>(base, i) : type == ATOMO_BF16 ? load1<ATOMO_BF16>(base, i) : load1<ATOMO_F16>(base, i);
}

__device__ inline void store_any4(int type, void* base, long long i, f32x4 x)
{
    if (type == ATOMO_F32) store4<ATOMO_F32, true>(base, i, x);
    else if (type == ATOMO_BF16) store4<ATOMO_BF16, true>(base, i, x);
    else store4<ATOMO_F16, true>(base, i, x);
}

__device__ inline void store_any1(int type, void* base, long long i, float x)
{
    if (type == ATOMO_F32) store1<ATOMO_F32>(base, i, x);
    else if (type == ATOMO_BF16) store1<ATOMO_BF16>(base, i, x);
    else store1<ATOMO_F16>(base, i, x);
}

__global__ __launch_bounds__(256) void adamw_states32(const Tensor* tensors, const Chunk* chunks, StepArgs a)
{
    const Chunk c = chunks[blockIdx.x];
    const Tensor t = tensors[c.tensor];
    Rates r;
    if (!rates_of(a, t, r)) return;
    const long long first = (long long)c.chunk * CHUNK;
    float* const m = (float*)t.m;
    float* const v = (float*)t.v;
#pragma unroll
    for (int k = 0; k < CHUNK / 1024; ++k) {
        const long long i = first + k * 1024 + threadIdx.x * 4;
        if (i + 4 <= t.n) {
            const f32x4 g = load_any4(t.grad_type, t.grad, i);
            const f32x4 p4 = load4<ATOMO_F32, true>(t.param, i), m4 = load4<ATOMO_F32, true>(m, i), v4 = load4<ATOMO_F32, true>(v, i);
            float pe[4], me[4], ve[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pe[e] = p4[e]; me[e] = m4[e]; ve[e] = v4[e];
                average(a, r, g[e], me[e], ve[e]);
            }
            update<false>(a, r, pe, me, ve);
            const f32x4 new_p = {pe[0], pe[1], pe[2], pe[3]};
            store4<ATOMO_F32, true>(t.param, i, new_p);
            store4<ATOMO_F32, true>(m, i, f32x4{me[0], me[1], me[2], me[3]});
            store4<ATOMO_F32, true>(v, i, f32x4{ve[0], ve[1], ve[2], ve[3]});
            if (t.copy) store_any4(t.copy_type, t.copy, i, new_p);
        } else {
            for (long long j = i; j < t.n; ++j) {
                float pe[1] = {t.param[j]}, me[1] = {m[j]}, ve[1] = {v[j]};
                average(a, r, load_any1(t.grad_type, t.grad, j), me[0], ve[0]);
                update<false>(a, r, pe, me, ve);
                t.param[j] = pe[0];
                m[j] = me[0];
                v[j] = ve[0];
                if (t.copy) store_any1(t.copy_type, t.copy, j, pe[0]);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// 8-bit states
// ---------------------------------------------------------------------------------------------

// A code of three mantissa bits lies in the top of an fp32 number: shifted there, its exponent bias is fp32's, so that
// one exact scaling by a power of two gives its value (the smallest codes are fp32 denormals in between, which the instruction keeps).
constexpr int M_BIAS = 7, V_BIAS = 15;
constexpr int TO_FP32 = 127;

__device__ inline int block_exponent(int scale) { return (scale > 1 ? scale : 1) - 127; }

__device__ inline float m_value(uint32_t code, int e)
{
    const float x = ldexpf(__uint_as_float((code & 0x7f) << 20), TO_FP32 - M_BIAS + e - M_BIAS);
    const float y = (code & 0x7f) == 0x7f ? __uint_as_float(0x7fc00000u) : x;
    return code & 0x80 ? -y : y;
}

template <bool NAN_CODES = true>
__device__ inline float v_value(uint32_t code, int e)
{
    const float x = ldexpf(__uint_as_float(code << 20), TO_FP32 - V_BIAS + e - V_BIAS);
    return NAN_CODES && code == 0xff ? __uint_as_float(0x7fc00000u) : x;
}

// Whether one of four codes is 0xff.
__device__ inline bool has_ff(uint32_t q) { return ((~q - 0x01010101u) & q & 0x80808080u) != 0; }

// Four codes of m at a time: the instruction's format is that of the codes.
__device__ inline void m_values(uint32_t q, int e, float* m)
{
    const float unit = ldexpf(1.0f, e - M_BIAS);
    m[0] = __builtin_amdgcn_cvt_f32_fp8((int)q, 0) * unit;
    m[1] = __builtin_amdgcn_cvt_f32_fp8((int)q, 1) * unit;
    m[2] = __builtin_amdgcn_cvt_f32_fp8((int)q, 2) * unit;
    m[3] = __builtin_amdgcn_cvt_f32_fp8((int)q, 3) * unit;
}

__device__ inline bool finite(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u; }

// |x| scaled to where its code's exponent is fp32's; then adding r below the three mantissa bits carries into them with the
// probability of what is cut off.  (Below the smallest normal code the scaled number is a denormal, rounded to 2^-20 of a step.)
__device__ inline uint32_t code_of(float x, int exponent, uint32_t r)
{
    return (__float_as_uint(ldexpf(fabsf(x), exponent)) + (r << 4)) >> 20;
}

// Codes of four elements.  FINITE: all of them are.
template <bool FINITE>
__device__ inline uint32_t m_codes(const float* x, int e, const uint32_t* words)
{
    uint32_t q = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t c = FINITE || finite(x[k]) ? code_of(x[k], M_BIAS - e - (TO_FP32 - M_BIAS), words[k] & 0xffff) : 0x7fu;
        q |= (c | (x[k] < 0.0f ? 0x80u : 0u)) << (8 * k);
    }
    return q;
}

template <bool FINITE>
__device__ inline uint32_t v_codes(const float* x, int e, const uint32_t* words)
{
    uint32_t q = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t c = code_of(x[k], V_BIAS - e - (TO_FP32 - V_BIAS), words[k] >> 16);
        // (a v of zero under an m that is not would be a step without bound)
        q |= (FINITE || finite(x[k]) ? max(c, min(__float_as_uint(x[k]), 1u)) : 0xffu) << (8 * k);
    }
    return q;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The larger of each half of x and of another lane's x.
template <int FROM>
__device__ inline uint32_t max_u16x2(uint32_t x)
{
    const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, FROM, 0xf, 0xf, false);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, other)));
}

// The largest of each half of x over the sixteen lanes of a row: neighbours, pairs, the mirror images of eight lanes and of sixteen.
__device__ inline uint32_t row_max_u16x2(uint32_t x) { return max_u16x2<0x140>(max_u16x2<0x141>(max_u16x2<0x4e>(max_u16x2<0xb1>(x)))); }

// Eight elements per thread, four in each half of a block: a scale belongs to the sixteen lanes of a row, and what a row loads or
// stores at a time fills whole cache lines.
__global__ __launch_bounds__(256) void adamw_states8(const Tensor* tensors, const Chunk* chunks, StepArgs a)
{
    const Chunk c = chunks[blockIdx.x];
    const Tensor t = tensors[c.tensor];
    Rates r;
    if (!rates_of(a, t, r)) return;
    const long long first = (long long)c.chunk * CHUNK + threadIdx.x / 16 * BLOCK8, block = first / BLOCK8;
    const long long at[2] = {first + threadIdx.x % 16 * 4, first + threadIdx.x % 16 * 4 + BLOCK8 / 2};
    const bool live = first < t.n, whole = first + BLOCK8 <= t.n;            // (the same for the lanes of a row)
    uint8_t* const mc = (uint8_t*)t.m;
    uint8_t* const vc = (uint8_t*)t.v;
    float p[8], g[8], m[8], v[8];
    uint32_t mq[2] = {0, 0}, vq[2] = {0, 0};
    const int m_scale = live ? t.m_scale[block] : 0, v_scale = live ? t.v_scale[block] : 0;
    if (whole) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            __builtin_memcpy(&mq[h], mc + at[h], 4);
            __builtin_memcpy(&vq[h], vc + at[h], 4);
            const f32x4 p4 = load4<ATOMO_F32, true>(t.param, at[h]), g4 = load_any4(t.grad_type, t.grad, at[h]);
#pragma unroll
            for (int e = 0; e < 4; ++e) { p[4 * h + e] = p4[e]; g[4 * h + e] = g4[e]; }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const long long i = at[e / 4] + e % 4;
            p[e] = g[e] = 0.0f;
            if (i < t.n) {
                p[e] = t.param[i];
                g[e] = load_any1(t.grad_type, t.grad, i);
                mq[e / 4] |= (uint32_t)mc[i] << (8 * (e % 4));
                vq[e / 4] |= (uint32_t)vc[i] << (8 * (e % 4));
            }
        }
    }
    const int em = block_exponent(m_scale), ev = block_exponent(v_scale);
    uint32_t sm = 0, sv = 0;
    m_values(mq[0], em, m);
    m_values(mq[1], em, m + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v_value<false>(vq[e / 4] >> (8 * (e % 4)) & 0xff, ev);
    if (__any(has_ff(vq[0]) || has_ff(vq[1]))) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v_value(vq[e / 4] >> (8 * (e % 4)) & 0xff, ev);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        average(a, r, g[e], m[e], v[e]);
        sm = max(sm, __float_as_uint(m[e]) >> 23 & 0xff);
        sv = max(sv, __float_as_uint(v[e]) >> 23 & 0xff);
    }
    update<true>(a, r, p, m, v);
    const bool finite_all = !__any(sm == 0xff || sv == 0xff);
    if (!finite_all) {                                           // scales are those of the finite ones
        sm = sv = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (finite(m[e])) sm = max(sm, __float_as_uint(m[e]) >> 23 & 0xff);
            if (finite(v[e])) sv = max(sv, __float_as_uint(v[e]) >> 23);
        }
    }
    const uint32_t largest = row_max_u16x2(sm << 16 | sv);
    sm = largest >> 16;
    sv = largest & 0xffff;
    const int fm = block_exponent((int)sm), fv = block_exponent((int)sv);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32x4 w = philox4x32_10((uint64_t)(t.first_block * (BLOCK8 / 4) + at[h] / 4), (uint64_t)r.step, a.seed);
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
        if (finite_all) {
            mq[h] = m_codes<true>(m + 4 * h, fm, words);
            vq[h] = v_codes<true>(v + 4 * h, fv, words);
        } else {
            mq[h] = m_codes<false>(m + 4 * h, fm, words);
            vq[h] = v_codes<false>(v + 4 * h, fv, words);
        }
    }
    if (whole) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 p4 = {p[4 * h], p[4 * h + 1], p[4 * h + 2], p[4 * h + 3]};
            store4<ATOMO_F32, true>(t.param, at[h], p4);
            if (t.copy) store_any4(t.copy_type, t.copy, at[h], p4);
            __builtin_memcpy(mc + at[h], &mq[h], 4);
            __builtin_memcpy(vc + at[h], &vq[h], 4);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const long long i = at[e / 4] + e % 4;
            if (i < t.n) {
                t.param[i] = p[e];
                if (t.copy) store_any1(t.copy_type, t.copy, i, p[e]);
                mc[i] = (uint8_t)(mq[e / 4] >> (8 * (e % 4)));
                vc[i] = (uint8_t)(vq[e / 4] >> (8 * (e % 4)));
            }
        }
    }
    if (live && threadIdx.x % 16 == 0) {
        t.m_scale[block] = (uint8_t)sm;
        t.v_scale[block] = (uint8_t)sv;
    }
}

// One byte read and two or four written per element, sixteen bytes per store (eight codes of a thread, four where they become fp32), which
// the caches need not keep, and GROUPS of them on their way at a time.
constexpr int GROUPS = 2;

template <int TYPE, bool V>
__global__ __launch_bounds__(256) void state8_values(const uint8_t* codes, const uint8_t* scales, long long n, void* out)
{
    constexpr int VEC = TYPE == ATOMO_F32 ? 4 : 8;
    const long long first = ((long long)blockIdx.x * (256 * GROUPS) + threadIdx.x) * VEC;
    if (((long long)blockIdx.x + 1) * (256 * GROUPS * VEC) <= n) {
        uint32_t q[GROUPS][VEC / 4];
        int e[GROUPS];
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            __builtin_memcpy(q[u], codes + first + u * (256 * VEC), VEC);
            e[u] = scales[(first + u * (256 * VEC)) / BLOCK8];
        }
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const long long i = first + u * (256 * VEC);
            float x[VEC];
#pragma unroll
            for (int h = 0; h < VEC / 4; ++h) {
                if constexpr (V) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[4 * h + k] = v_value(q[u][h] >> (8 * k) & 0xff, block_exponent(e[u]));
                } else {
                    m_values(q[u][h], block_exponent(e[u]), x + 4 * h);
                }
            }
            if constexpr (TYPE == ATOMO_F32) {
                store4<TYPE, true>(out, i, f32x4{x[0], x[1], x[2], x[3]});
            } else {
                u16x8_any s;
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = Element<TYPE>::down(x[j % VEC]);
                __builtin_nontemporal_store(s, (u16x8_any*)((uint16_t*)out + i));
            }
        }
    } else {
        for (long long i = (long long)blockIdx.x * (256 * GROUPS * VEC) + threadIdx.x; i < n; i += 256) {
            const int e = block_exponent(scales[i / BLOCK8]);
            store1<TYPE>(out, i, V ? v_value(codes[i], e) : m_value(codes[i], e));
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The norm of all gradients
// ---------------------------------------------------------------------------------------------

__device__ double workgroup_sum(double x)
{
    __shared__ double part[4];
    __syncthreads();                                             // (it may still be read from a sum before)
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}

// Squares and sums in double precision: neither the square of a tiny gradient nor that of a huge one is lost.  Sixteen bytes per
// load, a chunk's all on their way at once, and the next chunk looked up meanwhile.
template <int TYPE>
__device__ inline double chunk_squares(const void* grad, long long first, long long n)
{
    constexpr int VEC = TYPE == ATOMO_F32 ? 4 : 8, LOADS = CHUNK / 256 / VEC;
    double sum = 0.0;
    if (first + CHUNK <= n) {
        float x[LOADS][VEC];
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const long long i = first + (k * 256 + (int)threadIdx.x) * VEC;
            if constexpr (TYPE == ATOMO_F32) {
                const f32x4 g = load4<TYPE>(grad, i);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[k][e] = g[e];
            } else {
                const u16x8_any g = *(const u16x8_any*)((const uint16_t*)grad + i);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k][e] = Element<TYPE>::up(g[e]);
            }
        }
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum = fma((double)x[k][e], (double)x[k][e], sum);
    } else {
        for (long long i = first + threadIdx.x; i < n; i += 256) {
            const double g = (double)load1<TYPE>(grad, i);
            sum = fma(g, g, sum);
        }
    }
    return sum;
}

// LAST: the last of few workgroups to end (by a ticket that it puts back) forms the total in the same launch.
template <bool LAST>
__global__ __launch_bounds__(256) void norm_parts(const Tensor* tensors, const Chunk* chunks, int n_chunks, double* parts, unsigned* ticket, float scale, float* norm)
{
    double sum = 0.0;
    Chunk c = chunks[blockIdx.x];
    for (int b = blockIdx.x; b < n_chunks; b += gridDim.x) {
        const Chunk next = chunks[min(b + (int)gridDim.x, n_chunks - 1)];
        const Tensor& t = tensors[c.tensor];
        const long long n = t.n, first = (long long)c.chunk * CHUNK;
        const void* const grad = t.grad;
        const int type = t.grad_type;
        sum += type == ATOMO_F32 ? chunk_squares<ATOMO_F32>(grad, first, n)
             : type == ATOMO_BF16 ? chunk_squares<ATOMO_BF16>(grad, first, n) : chunk_squares<ATOMO_F16>(grad, first, n);
        c = next;
    }
    sum = workgroup_sum(sum);
    if constexpr (LAST) {
        __shared__ bool last;
        if (threadIdx.x == 0) {
            parts[blockIdx.x] = sum;
            __threadfence();
            last = atomicInc(ticket, gridDim.x - 1) == gridDim.x - 1;           // (back at zero with the last)
            __threadfence();
        }
        __syncthreads();
        if (!last) return;
        const double part = __hip_atomic_load(&parts[min((int)threadIdx.x, (int)gridDim.x - 1)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sum = workgroup_sum(threadIdx.x < gridDim.x ? part : 0.0);
        if (threadIdx.x == 0) norm[0] = (float)((double)scale * sqrt(sum));
    } else if (threadIdx.x == 0) {
        parts[blockIdx.x] = sum;
    }
}

__global__ __launch_bounds__(256) void norm_total(const double* parts, int n, float scale, float* norm)
{
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < NORM_PARTS / 256; ++k) {
        const double part = parts[min(k * 256 + (int)threadIdx.x, n - 1)];
        sum += k * 256 + (int)threadIdx.x < n ? part : 0.0;
    }
    sum = workgroup_sum(sum);
    if (threadIdx.x == 0) norm[0] = (float)((double)scale * sqrt(sum));
}

}  // namespace

}  // namespace atomo

struct atomo_adamw {
    int device = 0;
    void* dev = nullptr;               // tables and partial sums, one block
    atomo::Tensor* tensors = nullptr;
    atomo::Chunk* chunks = nullptr;    // those of tensors with 32-bit states first
    double* parts = nullptr;
    unsigned* ticket = nullptr;        // zero between calls
    int n32 = 0, n8 = 0;               // chunks
    bool updates = false;              // has parameters
};

namespace atomo {

// Whether something that a step writes overlaps anything else of the plan.
bool adamw_overlap(const atomo_adamw_tensor* tensors, int n)
{
    struct Range { uintptr_t first, end; bool written; };
    std::vector<Range> ranges;
    const auto add = [&](const void* p, int64_t bytes, bool written) {
        if (p) ranges.push_back(Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written});
    };
    for (int j = 0; j < n; ++j) {
        const atomo_adamw_tensor& t = tensors[j];
        add(t.grad, t.n * type_bytes(t.grad_type), false);
        if (!t.param) continue;
        const int64_t state_bytes = t.n * (t.m_scale ? 1 : 4), blocks = (t.n + BLOCK8 - 1) / BLOCK8;
        add(t.param, t.n * 4, true);
        add(t.copy, t.n * type_bytes(t.copy_type), true);
        add(t.m, state_bytes, true);
        add(t.v, state_bytes, true);
        add(t.m_scale, blocks, true);
        add(t.v_scale, blocks, true);
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range& x, const Range& y) { return x.first < y.first; });
    uintptr_t end = 0, end_written = 0;                          // of the ranges in front: all, those that are written
    for (const Range& r : ranges) {
        if (r.first < (r.written ? end : end_written)) return true;
        end = std::max(end, r.end);
        if (r.written) end_written = std::max(end_written, r.end);
    }
    return false;
}

int64_t adamw_chunks(const atomo_adamw_tensor* tensors, int n)
{
    int64_t chunks = 0;
    for (int j = 0; j < n; ++j) chunks += (tensors[j].n + CHUNK - 1) / CHUNK;
    return chunks;
}

int adamw_create(atomo_ctx* ctx, const atomo_adamw_tensor* tensors, int n, atomo_adamw** out)
{
    std::vector<Tensor> table(n);
    std::vector<Chunk> chunks, chunks8;
    long long blocks = 0;
    for (int j = 0; j < n; ++j) {
        const atomo_adamw_tensor& t = tensors[j];
        table[j] = Tensor{t.param, t.copy, t.grad, t.m, t.v, t.m_scale, t.v_scale, (long long)t.n, blocks,
                          t.grad_type, t.copy_type, t.lr_mult, t.weight_decay};
        blocks += (t.n + BLOCK8 - 1) / BLOCK8;
        for (int64_t k = 0; k * CHUNK < t.n; ++k) (t.param && t.m_scale ? chunks8 : chunks).push_back(Chunk{j, (int)k});
    }
    std::unique_ptr<atomo_adamw> plan(new atomo_adamw());
    plan->device = ctx->device;
    plan->n32 = (int)chunks.size();
    plan->n8 = (int)chunks8.size();
    plan->updates = tensors[0].param != nullptr;
    chunks.insert(chunks.end(), chunks8.begin(), chunks8.end());
    const auto carve = [&](void* base) {
        Carver c(base);
        plan->tensors = c.take<Tensor>(n);
        plan->chunks = c.take<Chunk>(chunks.size());
        plan->parts = c.take<double>(NORM_PARTS);
        plan->ticket = c.take<unsigned>(1);
        return c.off;
    };
    // tables, and a ticket of zero, in one copy
    std::vector<char> image(carve(nullptr), 0);
    carve(image.data());
    memcpy(plan->tensors, table.data(), n * sizeof(Tensor));
    memcpy(plan->chunks, chunks.data(), chunks.size() * sizeof(Chunk));
    hipError_t e = hipMalloc(&plan->dev, image.size());
    if (e != hipSuccess) {
        (void)hipGetLastError();              // (reported by the status alone: a later call is not to find it)
        ctx->last_hip = (int)e;
        return e == hipErrorOutOfMemory ? ATOMO_ENOMEM : ATOMO_EHIP;
    }
    carve(plan->dev);
    e = hipMemcpy(plan->dev, image.data(), image.size(), hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
        ctx->last_hip = (int)e;
        (void)hipFree(plan->dev);
        return ATOMO_EHIP;
    }
    *out = plan.release();
    return ATOMO_OK;
}

int adamw_destroy(atomo_ctx* ctx, atomo_adamw* plan)
{
    // (hipFree waits for the device, so no kernel still reads the tables)
    const hipError_t e = plan->dev ? hipFree(plan->dev) : hipSuccess;
    delete plan;
    ATOMO_HIP(ctx, e);
    return ATOMO_OK;
}

int adamw_device(const atomo_adamw* plan) { return plan->device; }
bool adamw_updates(const atomo_adamw* plan) { return plan->updates; }

int adamw_grad_norm(atomo_ctx* ctx, const atomo_adamw* plan, float grad_scale, float* norm, hipStream_t stream)
{
    ProfScope ps(ctx, ATOMO_K_ADAMW, stream);
    const int n = plan->n32 + plan->n8;
    if (n <= FEW_CHUNKS) {
        norm_parts<true><<<n, 256, 0, stream>>>(plan->tensors, plan->chunks, n, plan->parts, plan->ticket, fabsf(grad_scale), norm);
    } else {
        const int grid = std::min(n, NORM_PARTS);
        norm_parts<false><<<grid, 256, 0, stream>>>(plan->tensors, plan->chunks, n, plan->parts, nullptr, 0.0f, nullptr);
        norm_total<<<1, 256, 0, stream>>>(plan->parts, grid, fabsf(grad_scale), norm);
    }
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

int adamw_step(atomo_ctx* ctx, const atomo_adamw* plan, const atomo_adamw_options& o, hipStream_t stream)
{
    StepArgs a = {};
    a.lr = o.lr;
    a.beta1 = o.beta1;
    a.beta2 = o.beta2;
    a.step_dev = (const long long*)o.step_dev;
    a.lr_dev = o.lr_dev;
    a.grad_norm = o.grad_norm;
    a.step = o.step_dev ? 1 : o.step;
    a.rate = o.lr / (1.0 - std::pow(o.beta1, (double)a.step));
    a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(o.beta2, (double)a.step)));
    a.seed = o.seed;
    a.b1 = (float)o.beta1;
    a.c1 = (float)(1.0 - o.beta1);
    a.b2 = (float)o.beta2;
    a.c2 = (float)(1.0 - o.beta2);
    a.eps = (float)o.eps;
    a.plain_eps = plain_eps(a.eps);
    a.max_norm = o.max_norm;
    a.grad_scale = o.grad_scale;
    ProfScope ps(ctx, ATOMO_K_ADAMW, stream);
    if (plan->n32) adamw_states32<<<plan->n32, 256, 0, stream>>>(plan->tensors, plan->chunks, a);
    if (plan->n8) adamw_states8<<<plan->n8, 256, 0, stream>>>(plan->tensors, plan->chunks + plan->n32, a);
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

int state8_unpack(atomo_ctx* ctx, int which, const uint8_t* codes, const uint8_t* scales, int64_t n, int type, void* out,
                  hipStream_t stream)
{
    ProfScope ps(ctx, ATOMO_K_ADAMW, stream);
    with_type(type, [&](auto ty) {
        constexpr int PER = 256 * GROUPS * (ty == ATOMO_F32 ? 4 : 8);
        const unsigned grid = (unsigned)((n + PER - 1) / PER);
        if (which == ATOMO_STATE_V) state8_values<ty, true><<<grid, 256, 0, stream>>>(codes, scales, n, out);
        else state8_values<ty, false><<<grid, 256, 0, stream>>>(codes, scales, n, out);
    });
    ATOMO_HIP(ctx, hipGetLastError());
    return ATOMO_OK;
}

}  // namespace atomo
