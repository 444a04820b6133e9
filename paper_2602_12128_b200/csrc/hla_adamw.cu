// One AdamW step over many tensors, with moments in fp32 or in 8 bits, and the global gradient norm it is clipped by.
//
//     m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2,   p' = p - lr wd p - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// What bounds it: with fp32 moments memory (28 bytes an element with fp32 weights, their bf16 copies and bf16 gradients: 227 M elements in
// 1018 to 1042 us, 6.1 to 6.2 TB/s, and 70 to 79 us for the norm's pass over the gradients).  With 8-bit moments and bf16 weights (10 bytes) 54 instructions an
// element, 21 of them on the integer pipe, which takes one every other cycle: 490 us, where the bytes would take 353.  No unit is at its limit there
// (issue slots 73 %, integer pipe 55 %, DRAM 55 %).
//
// Layout: a row is 128 consecutive elements of a tensor, which is also what shares a scale.  A warp takes two rows, four elements of each a lane (with
// fp32 moments, so that every load is contiguous) or eight of one (8-bit moments).  Tensors from a few weights to
// millions are cut into chunks of 16 rows; a launch knows up to kMany tensors of one type from its parameters alone (nothing to upload, a
// captured step holds it) and its blocks go through the chunks in turns.
//
// 8-bit moments: e4m3 codes of x / scale, scale = max |x| of the row / 448.  Rounded up or down at random with the probability that
// keeps the mean: a second moment changes by a thousandth of itself a step, about a hundredth of the way from one code to the
// next, and rounding to the nearest would leave it where it is for ever.  A positive second moment never becomes zero (the
// quotient would explode): its code is at least 1.  bf16 weights without an fp32 original are rounded in the same way.
#include "../../include/hla.h"

#include <math.h>

#include <algorithm>
#include <memory>
#include <new>
#include <vector>

#include <cuda_fp16.h>

#include "hla_ops_common.cuh"

namespace hla {
namespace adamw {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRow = 128;                        // elements of a row: a scale of the 8-bit states
constexpr int kRows = 2;                         // rows of a warp per chunk
constexpr int kChunk = kWarps * kRows * kRow;
constexpr int kFew = 40, kMany = 360;            // tensors per launch: 3.7 and 32 KB of parameters
// Blocks of a step on an SM, and the most chunks of a turn.  8-bit states live on their arithmetic: three blocks, with registers for the next chunk
// on its way, take 587 us (the norm included) over eight transformer blocks, four 645, two 609; without the next chunk three take 673, four 632,
// five 638.  fp32 moments live on memory, which likes few places at a time: one block 1239 us, two 1120, three 1143, four 1152, five 1166; two
// with turns of one chunk 1175, two 1127, four 1108, eight 1116, sixteen 1123.  The next chunk in registers changes nothing there (1111).
template <bool Q8> constexpr int kBlocks = Q8 ? 3 : 2;
template <bool Q8> constexpr int kSpan = Q8 ? 8 : 4;
constexpr float kDead = 7.888609052210118e-31f;  // 2^-100: a row whose largest entry is below is held as zeros (its scale could not be inverted)

struct Tensor {
    void *p, *copy;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    long long n;
    float lr_mul, decay;
    uint32_t first;      // its first unit in the launch
    uint32_t number;     // its place in the caller's list
    uint8_t p_bf16, g_bf16;      // the same in all tensors of a launch
};

template <int MANY>
struct Args {
    int n;                        // tensors of this launch
    uint32_t units;               // turns: up to `span` chunks of a tensor each
    int span;
    int norm_blocks;              // partial sums of the squared norm (0: no norm)
    double* part;
    float* norm_out;
    float max_norm, grad_scale;
    float b1, r1, b2, r2, eps;
    double beta1, beta2;
    float lr, inv1, inv2;         // 1 / (1 - b1^t) and (1 - b2^t)^(-1/2) where the step is known on the host
    long long step;
    const float* lr_device;
    const long long* step_device;
    uint32_t seed_lo, seed_hi;
    Tensor t[MANY];
};

// A mixing function of 32 bits: two rounds of xor-shift and multiplication, shifts and factors those of Wellons' "lowbias32" (Hash Prospector),
// which were searched for the least bias between input and output bits.
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}

// The tensor that unit c belongs to, from the one that an earlier unit belonged to on.
template <int MANY>
__device__ __forceinline__ int tensor_of(const Args<MANY>& a, uint32_t c, int from) {
    if (from + 1 >= a.n || c < a.t[from + 1].first) return from;
    int lo = from + 1, hi = a.n;      // first[lo] <= c < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        (c < a.t[mid].first ? hi : lo) = mid;
    }
    return lo;
}

// Four elements at `i` of a tensor with `n` elements in all, as raw words; elements behind the end are zeros.  WHOLE: none are.
template <bool WHOLE>
__device__ __forceinline__ uint4 load_f32(const void* base, int i, int n) {
    const float* p = static_cast<const float*>(base) + i;
    if (WHOLE || i + 4 <= n) return *reinterpret_cast<const uint4*>(p);
    uint4 r = make_uint4(0, 0, 0, 0);
    if (i < n) r.x = __float_as_uint(p[0]);
    if (i + 1 < n) r.y = __float_as_uint(p[1]);
    if (i + 2 < n) r.z = __float_as_uint(p[2]);
    return r;
}
template <bool WHOLE>
__device__ __forceinline__ uint2 load_bf16(const void* base, int i, int n) {
    const unsigned short* p = static_cast<const unsigned short*>(base) + i;
    if (WHOLE || i + 4 <= n) return *reinterpret_cast<const uint2*>(p);
    uint2 r = make_uint2(0, 0);
    if (i < n) r.x = p[0];
    if (i + 1 < n) r.x |= (uint32_t)p[1] << 16;
    if (i + 2 < n) r.y = p[2];
    return r;
}
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_b8(const void* base, int i, int n) {
    const unsigned char* p = static_cast<const unsigned char*>(base) + i;
    if (WHOLE || i + 4 <= n) return *reinterpret_cast<const uint32_t*>(p);
    uint32_t r = 0;
    if (i < n) r = p[0];
    if (i + 1 < n) r |= (uint32_t)p[1] << 8;
    if (i + 2 < n) r |= (uint32_t)p[2] << 16;
    return r;
}
// Four floats or bf16 values.
template <bool BF16, bool WHOLE>
__device__ __forceinline__ uint4 load_any(const void* base, int i, int n) {
    if (!BF16) return load_f32<WHOLE>(base, i, n);
    const uint2 r = load_bf16<WHOLE>(base, i, n);
    return make_uint4(r.x, r.y, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ void unpack(const uint4& r, P2 (&x)[2]) {
    if (BF16) {
        x[0] = pair(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u));
        x[1] = pair(__uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
    } else {
        x[0] = pair(__uint_as_float(r.x), __uint_as_float(r.y));
        x[1] = pair(__uint_as_float(r.z), __uint_as_float(r.w));
    }
}
__device__ __forceinline__ void four(const P2 (&x)[2], float (&y)[4]) {
    const float2 a = both(x[0]), b = both(x[1]);
    y[0] = a.x; y[1] = a.y; y[2] = b.x; y[3] = b.y;
}
template <bool WHOLE>
__device__ __forceinline__ void store_f32(void* base, int i, int n, const float (&x)[4]) {
    float* p = static_cast<float*>(base) + i;
    if (WHOLE || i + 4 <= n) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); return; }
    for (int j = 0; j < 3; ++j)
        if (i + j < n) p[j] = x[j];
}
template <bool WHOLE>
__device__ __forceinline__ void store_bf16(void* base, int i, int n, uint32_t lo, uint32_t hi) {
    unsigned short* p = static_cast<unsigned short*>(base) + i;
    if (WHOLE || i + 4 <= n) { *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi); return; }
    if (i < n) p[0] = (unsigned short)lo;
    if (i + 1 < n) p[1] = (unsigned short)(lo >> 16);
    if (i + 2 < n) p[2] = (unsigned short)hi;
}
template <bool WHOLE>
__device__ __forceinline__ void store_b8(void* base, int i, int n, uint32_t c) {
    unsigned char* p = static_cast<unsigned char*>(base) + i;
    if (WHOLE || i + 4 <= n) { *reinterpret_cast<uint32_t*>(p) = c; return; }
    if (i < n) p[0] = (unsigned char)c;
    if (i + 1 < n) p[1] = (unsigned char)(c >> 8);
    if (i + 2 < n) p[2] = (unsigned char)(c >> 16);
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Two e4m3 codes as floats (exact).
__device__ __forceinline__ P2 decode2(uint32_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)codes));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return pair(f.x, f.y);
}

__device__ __forceinline__ float max_abs(float a, float b, float c) {      // a NaN stays
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Root and reciprocal of the update are the hardware's approximations, off by a unit or two in the last place of an update that is small against its
// weight and has some ten roundings anyway.  Correctly rounded ones are sequences of instructions; the moments, which are what is kept, have
// neither.
//
// Roots of second moments.  SMALL: of those below the smallest normal number too, which a tiny eps does not cover.
template <bool SMALL>
__device__ __forceinline__ float sqrt_fast(float x) {
    float r;
    if (SMALL) asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    else asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float reciprocal(float x) {      // (what is inverted is at least eps, which is a normal number)
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The largest |x| of a lane's eight; not a number if one of them is none.
__device__ __forceinline__ float most_of(const P2 (&v)[2][2]) {
    float x[4], y[4];
    four(v[0], x);
    four(v[1], y);
    return max_abs(max_abs(max_abs(max_abs(x[0], x[1], x[2]), x[3], y[0]), y[1], y[2]), y[3], y[3]);
}

// Values as e4m3.  With x / scale times 2^-120 the smallest normal e4m3 falls on the smallest normal fp32, so that one addition of 20 random bits
// below the code's rounds normal and subnormal codes alike.  The code ends up in the top byte: integer additions and shifts are what this
// kernel has too many of, so the shift is a product with the addition.  `per` is 448 / most, rounded: x per may pass 448 by a unit in the
// last place, and what that could carry over into the code of no number is cut off.
constexpr uint32_t kTop = 0x7effffffu;
__device__ __forceinline__ uint32_t top_bytes(const uint32_t (&w)[4]) {
    return __byte_perm(__byte_perm(w[0], w[1], 0x0073), __byte_perm(w[2], w[3], 0x0073), 0x5410);
}
__device__ __forceinline__ void scaled(const P2 (&x)[2], float per, float (&y)[4]) {
    const P2 z[2] = {mul2(mul2(x[0], twice(per)), twice(0x1p-120f)), mul2(mul2(x[1], twice(per)), twice(0x1p-120f))};
    four(z, y);
}
// The codes of four entries, of a moment that may be negative (low random bits) and of one that may not (high ones, and at least 1 where
// the entry is not zero).
__device__ __forceinline__ uint32_t codes(const P2 (&x)[2], float per, const uint32_t* bits) {
    float y[4], s[4];
    scaled(x, per, y);
    four(x, s);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = min(__float_as_uint(y[j]) * 16u + (bits[j] * 4096u >> 8), kTop) | (__float_as_uint(s[j]) & 0x80000000u);      // (the sign is shifted out)
    return top_bytes(w);
}
__device__ __forceinline__ uint32_t codes_positive(const P2 (&x)[2], float per, const uint32_t* bits) {
    float y[4], s[4];
    scaled(x, per, y);
    const P2 up[2] = {mul2(x[0], twice(0x1p20f)), mul2(x[1], twice(0x1p20f))};      // (bits of at least 2^20 for whatever is not zero, 2^-149 too)
    four(up, s);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = min(max(__float_as_uint(y[j]), min(__float_as_uint(s[j]), 1u << 20)) * 16u + (bits[j] >> 8), kTop);
    return top_bytes(w);
}
__device__ __forceinline__ bool held(float most) { return most >= kDead && most <= 3.402823466e38f; }

// The sum of the partial sums of the squared norm, in a fixed order, to every thread.
__device__ __forceinline__ double block_total(const double* part, int count, double* scratch) {
    double v = 0.0;
    for (int i = threadIdx.x; i < count; i += kThreads) v += part[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kWarps; ++w) v += scratch[w];
    return v;
}

// What a block does of a tensor in one turn: `whole` chunks, then the tensor's last, incomplete one if there is a `rest`.
struct Share {
    long long begin;      // its first element
    int whole, rest;      // rest: elements of the incomplete chunk
    __device__ __forceinline__ Share(const Tensor& t, uint32_t unit, int span) {
        begin = (long long)(unit - t.first) * span * kChunk;
        const long long left = t.n - begin;
        whole = left >= (long long)span * kChunk ? span : (int)(left / kChunk);
        rest = whole < span ? (int)(left - (long long)whole * kChunk) : 0;
    }
};

// The squares of four elements, in 64 bits.  Formed in fp32 where they and their sum are normal there; huge and tiny gradients are squared
// in 64 bits.
__device__ __forceinline__ double squares(const float (&g)[4]) {
    const float q = fmaf(g[0], g[0], g[1] * g[1]) + fmaf(g[2], g[2], g[3] * g[3]);
    if (q > 1e-25f && q < 1e38f) return q;
    double v = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) v = fma((double)g[j], (double)g[j], v);
    return v;
}

// This lane's part of COUNT chunks from `base` on, of `n` elements if not WHOLE.
template <bool BF16, bool WHOLE, int COUNT>
__device__ __forceinline__ double chunk_squares(const char* base, int n) {
    uint4 raw[COUNT][kRows];
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
#pragma unroll
        for (int r = 0; r < kRows; ++r) raw[i][r] = load_any<BF16, WHOLE>(base, i * kChunk + r * kRow, n);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            P2 pairs[2];
            float g[4];
            unpack<BF16>(raw[i][r], pairs);
            four(pairs, g);
            sum += squares(g);
        }
    return sum;
}
// Of `count` chunks, four at a time: with the loads of one chunk on their way the norm of 227 M bf16 elements took 85 us.
template <bool BF16>
__device__ __forceinline__ double run_squares(const char* base, int count) {
    constexpr int kBytes = kChunk * (BF16 ? 2 : 4);
    double sum = 0.0;
    for (; count >= 4; count -= 4, base += 4 * kBytes) sum += chunk_squares<BF16, true, 4>(base, 0);
    for (; count > 0; --count, base += kBytes) sum += chunk_squares<BF16, true, 1>(base, 0);
    return sum;
}

// Sums of squares run in 64 bits: the norm does not overflow where its gradients do not, and hardly depends on how the tensors were cut.
template <int MANY, bool GB>
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ Args<MANY> a) {
    __shared__ double scratch[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double sum = 0.0;
    int at = 0;
    for (uint32_t c = blockIdx.x; c < a.units; c += gridDim.x) {
        at = tensor_of(a, c, at);
        const Tensor& t = a.t[at];
        const Share s(t, c, a.span);
        const int own = warp * (kRows * kRow) + lane * 4;
        const char* base = static_cast<const char*>(t.g) + (s.begin + own) * (GB ? 2 : 4);
        sum += run_squares<GB>(base, s.whole);
        if (s.rest) sum += chunk_squares<GB, false, 1>(base + s.whole * (kChunk * (GB ? 2 : 4)), s.rest - own);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) scratch[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < kWarps; ++w) sum += scratch[w];
        a.part[blockIdx.x] = sum;
    }
}

// A sum that is not contracted with the product before it.
__device__ __forceinline__ P2 sum2(P2 a, P2 b) {
    const float2 x = both(a), y = both(b);
    return pair(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
}

struct Coefficients {
    float gain, b1, r1, b2, r2, eps, lr, inv1, inv2;
    uint32_t key;
};

// The new moments and weights of two elements.  The moments are formed in single products and sums, each rounded: what is rounded at random
// to 8 bits is then the same in every program that follows the formula, and so are the codes.
template <bool SMALL>
__device__ __forceinline__ void advance2(const Coefficients& k, float size, float shrink, P2 g, P2& m, P2& v, P2& w) {
    g = mul2(g, twice(k.gain));
    m = sum2(mul2(twice(k.b1), m), mul2(twice(k.r1), g));
    v = sum2(mul2(twice(k.b2), v), mul2(mul2(twice(k.r2), g), g));
    const float2 square = both(v);
    const float2 below = both(fma2(pair(sqrt_fast<SMALL>(square.x), sqrt_fast<SMALL>(square.y)), twice(k.inv2), twice(k.eps)));
    w = fma2(twice(-size), mul2(m, pair(reciprocal(below.x), reciprocal(below.y))), fma2(twice(-shrink), w, w));
}

// The random words of a row's pairs `first` to `first` + PAIRS - 1, `key` being that of its tensor.
template <int PAIRS>
__device__ __forceinline__ void random_words(uint32_t key, uint32_t row, int first, uint32_t (&bits)[2 * PAIRS]) {
    const uint32_t block = mix32(key + row * 0x9E3779B9u) + (uint32_t)first * 0x9E3779B9u;
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
        uint32_t x = block + (uint32_t)j * 0x9E3779B9u;
        x ^= x >> 16;
        x *= 0x7FEB352Du;
        x = (x ^ (x >> 15)) * 0x846CA68Bu;
        const uint32_t y = x * 0xC2B2AE35u;
        bits[2 * j] = x ^ (x >> 16);
        bits[2 * j + 1] = y ^ (y >> 15);
    }
}

// Four weights to bf16, rounded by the upper halves of products of their random words.
__device__ __forceinline__ uint2 round_bf16(const float (&p)[4], const uint32_t* bits) {
    uint32_t h[4];
    const float any = (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = __float_as_uint(p[j]) + (bits[j] * 0x9E3779B9u >> 16);
    if (!(fabsf(any) <= 3.402823466e38f)) {      // an infinity has no low bits to carry from; a NaN would overflow
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (p[j] != p[j]) h[j] = __float_as_uint(p[j]);
    }
    return make_uint2(__byte_perm(h[0], h[1], 0x7632), __byte_perm(h[2], h[3], 0x7632));
}

// fp32 moments: `count` chunks of a tensor from element `begin` on, of `n` elements if not WHOLE.  Four elements of a row a lane.
template <bool PB, bool GB, bool WHOLE>
__device__ __forceinline__ void update(const Tensor& t, const Coefficients& k, long long begin, int count, int n, int warp, int lane) {
    constexpr int kP = PB ? 2 : 4, kG = GB ? 2 : 4;
    const int own = warp * (kRows * kRow) + lane * 4;
    const long long first = begin + own;
    const char* pg = static_cast<const char*>(t.g) + first * kG;
    char *pp = static_cast<char*>(t.p) + first * kP, *pm = static_cast<char*>(t.m) + first * 4, *pv = static_cast<char*>(t.v) + first * 4;
    char* pc = PB || !t.copy ? nullptr : static_cast<char*>(t.copy) + first * 2;
    uint32_t row = (uint32_t)(begin / kRow) + warp * kRows;      // (tensors have up to 2^38 elements)
    const float rate = k.lr * t.lr_mul, size = rate * k.inv1, shrink = rate * t.decay;
    const uint32_t key = PB ? mix32(k.key + t.number) : 0;
    n -= own;
    for (; count > 0; --count) {
        uint4 rg[kRows], rp[kRows], rm[kRows], rv[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int i = r * kRow;
            rg[r] = load_any<GB, WHOLE>(pg, i, n);
            rp[r] = load_any<PB, WHOLE>(pp, i, n);
            rm[r] = load_f32<WHOLE>(pm, i, n);
            rv[r] = load_f32<WHOLE>(pv, i, n);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int i = r * kRow;
            P2 g[2], m[2], v[2], w[2];
            unpack<GB>(rg[r], g);
            unpack<PB>(rp[r], w);
            unpack<false>(rm[r], m);
            unpack<false>(rv[r], v);
#pragma unroll
            for (int j = 0; j < 2; ++j) advance2<true>(k, size, shrink, g[j], m[j], v[j], w[j]);
            float x[4];
            four(w, x);
            if (PB) {
                uint32_t bits[4];
                random_words<2>(key, row + r, lane * 2, bits);
                const uint2 h = round_bf16(x, bits);
                store_bf16<WHOLE>(pp, i, n, h.x, h.y);
            } else {
                store_f32<WHOLE>(pp, i, n, x);
                if (pc) store_bf16<WHOLE>(pc, i, n, two_bf16(x[0], x[1]), two_bf16(x[2], x[3]));
            }
            four(m, x);
            store_f32<WHOLE>(pm, i, n, x);
            four(v, x);
            store_f32<WHOLE>(pv, i, n, x);
        }
        pg += kChunk * kG;
        pp += kChunk * kP;
        pm += kChunk * 4;
        pv += kChunk * 4;
        if (pc) pc += kChunk * 2;
        row += kChunk / kRow;
    }
}

// 8-bit moments, the same chunks.  Half a warp has a row, eight elements a lane: what is done once a row and lane (maximum, reciprocal, key of
// the random numbers, addresses) is done for twice as many elements: 62 -> 54 instructions an element, 659 -> 587 us.
template <bool PB, bool GB, bool WHOLE>
__device__ __forceinline__ void update_q8(const Tensor& t, const Coefficients& k, long long begin, int count, int n, int warp, int lane) {
    constexpr int kP = PB ? 2 : 4, kG = GB ? 2 : 4, kWide = 8;
    static_assert(kRows * kRow == 32 * kWide, "two rows a warp");
    const int own = warp * (kRows * kRow) + lane * kWide;      // (lanes 16 to 31 have the second row)
    const long long first = begin + own;
    const char* pg = static_cast<const char*>(t.g) + first * kG;
    char *pp = static_cast<char*>(t.p) + first * kP, *pm = static_cast<char*>(t.m) + first, *pv = static_cast<char*>(t.v) + first;
    char* pc = PB || !t.copy ? nullptr : static_cast<char*>(t.copy) + first * 2;
    uint32_t row = (uint32_t)(first / kRow);
    float *pms = t.ms + row, *pvs = t.vs + row;
    const float rate = k.lr * t.lr_mul, size = rate * k.inv1, shrink = rate * t.decay;
    const uint32_t key = mix32(k.key + t.number);
    const bool second = lane & 8;      // lanes of a row whose number has this bit go by the second moment where there is one value for both
    n -= own;
    struct Raw {
        uint4 g[2], p[2];      // (one each in bf16)
        uint2 m, v;
        float sm, sv;
    };
    auto load = [&](Raw& x, int ahead) {
        const int i = ahead * kChunk;
        if (GB && WHOLE) x.g[0] = load_f32<true>(pg + i * 2, 0, 0);      // (16 bytes)
        else if (GB) { const uint2 lo = load_bf16<false>(pg, 0, n), hi = load_bf16<false>(pg, 4, n); x.g[0] = make_uint4(lo.x, lo.y, hi.x, hi.y); }
        else { x.g[0] = load_f32<WHOLE>(pg, i, n); x.g[1] = load_f32<WHOLE>(pg, i + 4, n); }
        if (PB && WHOLE) x.p[0] = load_f32<true>(pp + i * 2, 0, 0);
        else if (PB) { const uint2 lo = load_bf16<false>(pp, 0, n), hi = load_bf16<false>(pp, 4, n); x.p[0] = make_uint4(lo.x, lo.y, hi.x, hi.y); }
        else { x.p[0] = load_f32<WHOLE>(pp, i, n); x.p[1] = load_f32<WHOLE>(pp, i + 4, n); }
        if (WHOLE) {
            x.m = load_bf16<true>(pm + i, 0, 0);      // (8 bytes)
            x.v = load_bf16<true>(pv + i, 0, 0);
        } else {
            x.m = make_uint2(load_b8<false>(pm, 0, n), load_b8<false>(pm, 4, n));
            x.v = make_uint2(load_b8<false>(pv, 0, n), load_b8<false>(pv, 4, n));
        }
        const bool some = WHOLE || n > 0;
        x.sm = some ? pms[i / kRow] : 0.f;
        x.sv = some ? pvs[i / kRow] : 0.f;
    };
    auto compute = [&](const Raw& raw, int ahead) {
        const int i = ahead * kChunk;
        P2 g[2][2], m[2][2], v[2][2], w[2][2];      // two fours
        if (GB) { unpack<true>(raw.g[0], g[0]); unpack<true>(make_uint4(raw.g[0].z, raw.g[0].w, 0, 0), g[1]); }
        else { unpack<false>(raw.g[0], g[0]); unpack<false>(raw.g[1], g[1]); }
        if (PB) { unpack<true>(raw.p[0], w[0]); unpack<true>(make_uint4(raw.p[0].z, raw.p[0].w, 0, 0), w[1]); }
        else { unpack<false>(raw.p[0], w[0]); unpack<false>(raw.p[1], w[1]); }
        const uint32_t cm[2] = {raw.m.x, raw.m.y}, cv[2] = {raw.v.x, raw.v.y};
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[f][j] = mul2(decode2(cm[f] >> (16 * j)), twice(raw.sm));
                v[f][j] = mul2(decode2(cv[f] >> (16 * j)), twice(raw.sv));
                advance2<false>(k, size, shrink, g[f][j], m[f][j], v[f][j], w[f][j]);
            }
        uint32_t bits[8];
        random_words<4>(key, row + ahead * (kChunk / kRow), (lane & 15) * 4, bits);
        uint32_t h[4];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            float x[4];
            four(w[f], x);
            if (PB) {
                const uint2 r = round_bf16(x, bits + 4 * f);
                h[2 * f] = r.x;
                h[2 * f + 1] = r.y;
            } else {
                store_f32<WHOLE>(pp, i + 4 * f, n, x);
                h[2 * f] = two_bf16(x[0], x[1]);
                h[2 * f + 1] = two_bf16(x[2], x[3]);
            }
        }
        char* low = PB ? pp : pc;
        if (PB || low) {
            if (WHOLE) *reinterpret_cast<uint4*>(low + i * 2) = make_uint4(h[0], h[1], h[2], h[3]);
            else { store_bf16<false>(low, 0, n, h[0], h[1]); store_bf16<false>(low, 4, n, h[2], h[3]); }
        }
        // the largest entries of the row: half of its lanes go on with the first moment, half with the second
        const float lm = most_of(m), lv = most_of(v);
        uint32_t bits_of = max(__float_as_uint(second ? lv : lm), __shfl_xor_sync(0xffffffffu, __float_as_uint(second ? lm : lv), 8));      // (bits of non-negative floats are ordered like them)
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) bits_of = max(bits_of, __shfl_xor_sync(0xffffffffu, bits_of, o));
        const float most = __uint_as_float(bits_of), per = __frcp_rn(most) * 448.f, other = __shfl_xor_sync(0xffffffffu, per, 8);
        const float per_m = second ? other : per, per_v = second ? per : other;
        float scale = most * (1.f / 448.f);
        uint2 qm = make_uint2(codes(m[0], per_m, bits), codes(m[1], per_m, bits + 4)), qv = make_uint2(codes_positive(v[0], per_v, bits), codes_positive(v[1], per_v, bits + 4));
        if (!__all_sync(0xffffffffu, held(most))) {
            // a row of next to nothing is zeros; one with an entry that is no number, or infinite, is no numbers throughout
            const bool mine = held(most), its = __shfl_xor_sync(0xffffffffu, (int)mine, 8);
            if (!(second ? its : mine)) qm = make_uint2(0, 0);
            if (!(second ? mine : its)) qv = make_uint2(0, 0);
            if (!mine) scale = most < kDead ? 0.f : __int_as_float(0x7fc00000);
        }
        if (WHOLE) {
            *reinterpret_cast<uint2*>(pm + i) = qm;
            *reinterpret_cast<uint2*>(pv + i) = qv;
        } else {
            store_b8<false>(pm, 0, n, qm.x);
            store_b8<false>(pm, 4, n, qm.y);
            store_b8<false>(pv, 0, n, qv.x);
            store_b8<false>(pv, 4, n, qv.y);
        }
        if ((lane & 7) == 0 && (WHOLE || n + (second ? 8 * kWide : 0) > 0)) (second ? pvs : pms)[i / kRow] = scale;      // (n counts from this lane's first element)
    };
    Raw x;
    if (WHOLE) {      // the next chunk is on its way during the arithmetic of this one, which takes as long as its bytes
        Raw y;
        load(x, 0);
        for (; count > 0; count -= 2) {
            if (count > 1) load(y, 1);
            compute(x, 0);
            if (count > 1) {
                if (count > 2) load(x, 2);
                compute(y, 1);
            }
            pg += 2 * kChunk * kG;
            pp += 2 * kChunk * kP;
            pm += 2 * kChunk;
            pv += 2 * kChunk;
            if (pc) pc += 2 * kChunk * 2;
            pms += 2 * kChunk / kRow;
            pvs += 2 * kChunk / kRow;
            row += 2 * kChunk / kRow;
        }
    } else {
        load(x, 0);
        compute(x, 0);
    }
}

template <int MANY, bool Q8, bool PB, bool GB>
__global__ void __launch_bounds__(kThreads, kBlocks<Q8>) step_kernel(const __grid_constant__ Args<MANY> a) {
    __shared__ double scratch[kWarps];
    __shared__ float hyper[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    wait_for_previous_kernel();
    const long long step = a.step_device ? *a.step_device : a.step;
    if (a.step_device && threadIdx.x == 0) {
        hyper[0] = (float)(-1.0 / expm1((double)step * log(a.beta1)));
        hyper[1] = (float)rsqrt(-expm1((double)step * log(a.beta2)));
    }
    Coefficients k;
    k.gain = a.grad_scale;
    if (a.norm_blocks) {
        const float norm = (float)(sqrt(block_total(a.part, a.norm_blocks, scratch)) * fabs((double)a.grad_scale));
        if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm_out) *a.norm_out = norm;
        if (!isfinite(norm)) return;      // nothing changes
        k.gain *= fminf(a.max_norm / (norm + 1e-6f), 1.f);
    }
    if (step < 1) return;      // (the host refuses such a step where it knows it)
    __syncthreads();
    k.b1 = a.b1; k.r1 = a.r1; k.b2 = a.b2; k.r2 = a.r2; k.eps = a.eps;
    k.lr = a.lr_device ? *a.lr_device : a.lr;
    k.inv1 = a.step_device ? hyper[0] : a.inv1;
    k.inv2 = a.step_device ? hyper[1] : a.inv2;
    k.key = mix32(mix32(mix32(a.seed_lo) ^ a.seed_hi) ^ (uint32_t)step);
    int at = 0;
    for (uint32_t c = blockIdx.x; c < a.units; c += gridDim.x) {
        at = tensor_of(a, c, at);
        const Tensor& t = a.t[at];
        const Share s(t, c, a.span);
        if (Q8) {
            if (s.whole) update_q8<PB, GB, true>(t, k, s.begin, s.whole, 0, warp, lane);
            if (s.rest) update_q8<PB, GB, false>(t, k, s.begin + s.whole * kChunk, 1, s.rest, warp, lane);
        } else {
            if (s.whole) update<PB, GB, true>(t, k, s.begin, s.whole, 0, warp, lane);
            if (s.rest) update<PB, GB, false>(t, k, s.begin + s.whole * kChunk, 1, s.rest, warp, lane);
        }
    }
}

}  // namespace adamw
}  // namespace hla

using namespace hla;

struct hla_adamw {
    hla_adamw_config cfg;
    std::vector<adamw::Tensor> t;      // those with weights in them; `first` within their launch
    int given;
    int sm_count;
};

namespace {

struct Span {
    uintptr_t at, end;
    bool written;
};

// Whether one of the tensors that a step writes shares memory with another one.
bool clash(std::vector<Span>& spans) {
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
    uintptr_t end = 0, written = 0;      // how far the spans so far reach, all and the written ones
    for (const Span& s : spans) {
        if (s.at < (s.written ? end : written)) return true;
        end = std::max(end, s.end);
        if (s.written) written = std::max(written, s.end);
    }
    return false;
}

hla_status check_spans(const hla_adamw* c) {
    const bool q8 = c->cfg.state == HLA_STATE_Q8;
    std::vector<Span> spans;
    auto add = [&](const void* p, long long bytes, bool written) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p) spans.push_back({at, at + (uintptr_t)bytes, written});
    };
    for (const adamw::Tensor& t : c->t) {
        const long long rows = (t.n + adamw::kRow - 1) / adamw::kRow;
        add(t.p, t.n * (t.p_bf16 ? 2 : 4), true);
        add(t.copy, t.n * 2, true);
        add(t.m, t.n * (q8 ? 1 : 4), true);
        add(t.v, t.n * (q8 ? 1 : 4), true);
        if (q8) add(t.ms, rows * 4, true), add(t.vs, rows * 4, true);
        add(t.g, t.n * (t.g_bf16 ? 2 : 4), false);
    }
    return clash(spans) ? HLA_ERR_INVALID_ARG : HLA_OK;
}

// Chunks that a block takes in one turn.  Finding a tensor and its pointers costs about 80 instructions, ten an element of a chunk; where
// every SM has at least 64 turns, up to kSpan chunks share them.
int span(const hla_adamw* c, int from, int n) {
    const int most = c->cfg.state == HLA_STATE_Q8 ? adamw::kSpan<true> : adamw::kSpan<false>;
    long long chunks = 0;
    for (int i = 0; i < n; ++i) chunks += (c->t[from + i].n + adamw::kChunk - 1) / adamw::kChunk;
    int s = 1;
    while (s < most && chunks >= 2ll * s * 64 * c->sm_count) s *= 2;
    return s;
}

template <int MANY>
void fill(adamw::Args<MANY>& a, const hla_adamw* c, int from, int n) {
    a.n = n;
    a.span = span(c, from, n);
    a.units = 0;
    const long long per = (long long)a.span * adamw::kChunk;
    for (int i = 0; i < n; ++i) {
        a.t[i] = c->t[from + i];
        a.t[i].first = a.units;
        a.units += (uint32_t)((a.t[i].n + per - 1) / per);
    }
}

// Tensors from `from` on that one launch takes: of the same types.
int batch(const hla_adamw* c, int from) {
    int n = 1;
    while (from + n < (int)c->t.size() && n < adamw::kMany && c->t[from + n].p_bf16 == c->t[from].p_bf16 && c->t[from + n].g_bf16 == c->t[from].g_bf16) ++n;
    return n;
}

template <int MANY, bool Q8>
void (*step_of(const adamw::Tensor& t))(adamw::Args<MANY>) {
    if (t.p_bf16) return t.g_bf16 ? adamw::step_kernel<MANY, Q8, true, true> : adamw::step_kernel<MANY, Q8, true, false>;
    return t.g_bf16 ? adamw::step_kernel<MANY, Q8, false, true> : adamw::step_kernel<MANY, Q8, false, false>;
}

int norm_blocks(const hla_adamw* c, uint32_t units) { return (int)std::min<uint32_t>(units, 8u * c->sm_count); }

template <typename A>
bool launch_step(void (*kern)(A), dim3 blocks, const A& a, cudaStream_t st) {
    if (a.norm_blocks) return launch_behind(kern, blocks, adamw::kThreads, st, a);
    kern<<<blocks, adamw::kThreads, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess;
}

template <int MANY>
hla_status step(const hla_adamw* c, const hla_adamw_step_args& s, double* part, cudaStream_t st) {
    adamw::Args<MANY> a;
    const hla_adamw_config& k = c->cfg;
    a.part = part;
    a.norm_out = s.norm;
    a.max_norm = s.max_norm;
    a.grad_scale = s.grad_scale == 0.f ? 1.f : s.grad_scale;
    a.b1 = (float)k.beta1; a.r1 = (float)(1.0 - k.beta1);
    a.b2 = (float)k.beta2; a.r2 = (float)(1.0 - k.beta2);
    a.eps = (float)k.eps;
    a.beta1 = k.beta1; a.beta2 = k.beta2;
    a.lr = (float)s.lr;
    a.step = s.step;
    a.inv1 = s.step_device ? 0.f : (float)(-1.0 / expm1((double)s.step * log(k.beta1)));
    a.inv2 = s.step_device ? 0.f : (float)(1.0 / sqrt(-expm1((double)s.step * log(k.beta2))));
    a.lr_device = s.lr_device;
    a.step_device = reinterpret_cast<const long long*>(s.step_device);
    a.seed_lo = (uint32_t)k.seed;
    a.seed_hi = (uint32_t)(k.seed >> 32);
    a.norm_blocks = 0;
    const int total = (int)c->t.size();
    if (s.max_norm > 0.f) {
        for (int from = 0; from < total; from += batch(c, from)) {
            fill(a, c, from, batch(c, from));
            const int blocks = norm_blocks(c, a.units);
            a.part = part + a.norm_blocks;
            if (c->t[from].g_bf16) adamw::norm_kernel<MANY, true><<<blocks, adamw::kThreads, 0, st>>>(a);
            else adamw::norm_kernel<MANY, false><<<blocks, adamw::kThreads, 0, st>>>(a);
            if (cudaGetLastError() != cudaSuccess) return HLA_ERR_CUDA;
            a.norm_blocks += blocks;
        }
        a.part = part;
    }
    for (int from = 0; from < total; from += batch(c, from)) {
        fill(a, c, from, batch(c, from));
        if (from) a.norm_out = nullptr;
        const dim3 blocks(std::min<uint32_t>(a.units, (k.state == HLA_STATE_Q8 ? adamw::kBlocks<true> : adamw::kBlocks<false>) * (uint32_t)c->sm_count));
        if (!launch_step(k.state == HLA_STATE_Q8 ? step_of<MANY, true>(c->t[from]) : step_of<MANY, false>(c->t[from]), blocks, a, st)) return HLA_ERR_CUDA;
    }
    return HLA_OK;
}

}  // namespace

extern "C" {

hla_status hla_adamw_create(const hla_adamw_config* cfg, const hla_adamw_tensor* tensors, int32_t n, hla_adamw** out) {
    if (out) *out = nullptr;
    if (!cfg || !out || !tensors || n <= 0) return HLA_ERR_INVALID_ARG;
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) || !(cfg->eps >= 0x1p-126) || !isfinite((float)cfg->eps))
        return HLA_ERR_INVALID_ARG;
    if (cfg->state != HLA_STATE_F32 && cfg->state != HLA_STATE_Q8) return HLA_ERR_INVALID_ARG;
    const bool q8 = cfg->state == HLA_STATE_Q8;
    if (q8 && cfg->eps < 0x1p-50) return HLA_ERR_INVALID_ARG;      // a row of second moments below 2^-100 is held as zeros: eps has to cover their roots
    if (n > (1 << 20)) return HLA_ERR_UNSUPPORTED;
    try {
        std::unique_ptr<hla_adamw> c(new hla_adamw());
        c->cfg = *cfg;
        c->given = n;
        c->sm_count = current_sm_count();
        hla_status st = HLA_OK;
        unsigned long long chunks = 0;
        for (int i = 0; i < n && st == HLA_OK; ++i) {
            const hla_adamw_tensor& t = tensors[i];
            if (t.n < 0 || (t.param_dtype != HLA_BF16 && t.param_dtype != HLA_F32) || (t.grad_dtype != HLA_BF16 && t.grad_dtype != HLA_F32) ||
                !isfinite(t.lr_mul) || !isfinite(t.weight_decay)) { st = HLA_ERR_INVALID_ARG; break; }
            if (t.n == 0) continue;
            const void* all[] = {t.param, t.grad, t.m, t.v, q8 ? t.m_scale : t.m, q8 ? t.v_scale : t.v};
            for (const void* p : all)
                if (!p || !aligned16(p)) st = HLA_ERR_INVALID_ARG;
            if (!aligned16(t.copy) || (t.copy && t.param_dtype != HLA_F32)) st = HLA_ERR_INVALID_ARG;
            if (t.n > (1ll << 38)) st = HLA_ERR_UNSUPPORTED;
            chunks += (unsigned long long)(t.n + adamw::kChunk - 1) / adamw::kChunk;
            adamw::Tensor d{};
            d.p = t.param; d.copy = t.copy; d.g = t.grad; d.m = t.m; d.v = t.v;
            d.ms = q8 ? static_cast<float*>(t.m_scale) : nullptr;
            d.vs = q8 ? static_cast<float*>(t.v_scale) : nullptr;
            d.n = t.n;
            d.number = (uint32_t)i;
            d.lr_mul = t.lr_mul == 0.f ? 1.f : t.lr_mul;
            d.decay = t.weight_decay;
            d.p_bf16 = t.param_dtype == HLA_BF16;
            d.g_bf16 = t.grad_dtype == HLA_BF16;
            c->t.push_back(d);
        }
        std::stable_sort(c->t.begin(), c->t.end(), [](const adamw::Tensor& a, const adamw::Tensor& b) { return 2 * a.p_bf16 + a.g_bf16 < 2 * b.p_bf16 + b.g_bf16; });
        if (st == HLA_OK && chunks >= (1ull << 31)) st = HLA_ERR_UNSUPPORTED;
        if (st == HLA_OK) st = check_spans(c.get());
        if (st == HLA_OK) *out = c.release();
        return st;
    } catch (...) {
        return HLA_ERR_NO_MEMORY;
    }
}

hla_status hla_adamw_set_grads(hla_adamw* c, const void* const* grads, int32_t n) {
    if (!c || !grads || n != c->given) return HLA_ERR_INVALID_ARG;
    for (const adamw::Tensor& t : c->t)
        if (!grads[t.number] || !aligned16(grads[t.number])) return HLA_ERR_INVALID_ARG;
    try {
        std::vector<adamw::Tensor> before = c->t;
        for (adamw::Tensor& t : c->t) t.g = grads[t.number];
        const hla_status st = check_spans(c);
        if (st != HLA_OK) c->t.swap(before);
        return st;
    } catch (...) {
        return HLA_ERR_NO_MEMORY;
    }
}

size_t hla_adamw_workspace_bytes(const hla_adamw* c) {
    if (!c) return 0;
    size_t n = 0;
    for (int from = 0; from < (int)c->t.size(); from += batch(c, from)) n += (size_t)8 * c->sm_count;
    return (n * 8 + 255) / 256 * 256;
}

hla_status hla_adamw_step(hla_adamw* c, const hla_adamw_step_args* s, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!c || !s) return HLA_ERR_INVALID_ARG;
    if (!(s->max_norm >= 0.f) || !isfinite(s->grad_scale) || !isfinite(s->lr)) return HLA_ERR_INVALID_ARG;
    if (!s->step_device && s->step < 1) return HLA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(s->step_device) & 7u) || (reinterpret_cast<uintptr_t>(s->lr_device) & 3u) || (reinterpret_cast<uintptr_t>(s->norm) & 3u))
        return HLA_ERR_INVALID_ARG;
    // blocks read the two scalars while one writes the norm
    if (s->max_norm > 0.f && s->norm && ((s->lr_device && overlap(s->norm, 4, s->lr_device, 4)) || (s->step_device && overlap(s->norm, 4, s->step_device, 8)))) return HLA_ERR_INVALID_ARG;
    if (c->t.empty())      // nothing but a norm of nothing
        return s->max_norm > 0.f && s->norm && cudaMemsetAsync(s->norm, 0, 4, static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess ? HLA_ERR_CUDA : HLA_OK;
    if (s->max_norm > 0.f) {
        if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HLA_ERR_INVALID_ARG;
        if (workspace_bytes < hla_adamw_workspace_bytes(c)) return HLA_ERR_WORKSPACE;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    double* part = static_cast<double*>(workspace);
    return (int)c->t.size() <= adamw::kFew ? step<adamw::kFew>(c, *s, part, st) : step<adamw::kMany>(c, *s, part, st);
}

hla_status hla_adamw_destroy(hla_adamw* c) {
    if (!c) return HLA_ERR_INVALID_ARG;
    delete c;
    return HLA_OK;
}

}  // extern "C"
