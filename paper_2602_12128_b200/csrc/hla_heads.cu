// Head preparation: what a projection [B,N,H,d] needs before it enters hla_forward (Algorithm 1 steps 1-3), and its backward.
//
//     y = s R(theta_n) (x r . w),   r = (mean x^2 + eps)^(-1/2),   theta_{n,p} = position_{axis(p)} inv_freq_p
//     g = s R(-theta_n) dy,   dw = sum g . x r,   dx = r (g . w - x r mean(g . w . x r))
//
// What bounds it: memory.  A row of d channels is read once (the backward: dy and x), about ten operations an element, and
// written once, at another place: the rows of one token lie together in the projection, those of one head in Q, K, V.  Forward of
// 24 x 32760 rows of 128 bf16 channels (q, k, v): 198 us, 6.1 TB/s; backward of twice as many 511 us, 6.3 TB/s.
//
// Layout: 16 bytes of a row per lane, so a row of 128 bf16 channels is half a warp and is summed with four shuffles; the two
// channels of every pair are in the same lane in both pairings.  Such a group of lanes takes one token and goes through the
// heads of one tensor: the angles of a token (a product and a reduction in 64 bits, one sincospi per pair) are computed once and
// stay in registers.  Neighbouring groups take neighbouring tokens, so a block reads rows of H d and writes runs of 16 tokens.  The next rows
// of a lane are on their way through shared memory: with as many in registers the forward took 207 us.
#include "../../include/hla.h"

#include <math.h>
#include <new>

#include "hla_heads_units.h"
#include "hla_ops_common.cuh"

namespace hla {
namespace heads {

constexpr int kThreads = 256;
constexpr int kMaxPairs = kMaxD / 2;
constexpr int kDwThreads = 1024, kDwChannels = 8;
constexpr int kStages = 4;          // rows of a group on their way in the backward

struct Tensor {
    const char *x, *dy;          // projection (strided); gradient of the prepared tensor (head-major)
    char* out;                   // forward: prepared tensor (head-major); backward: gradient of the projection (strided)
    long long x_batch, x_token, o_batch, o_token;    // strides in bytes; o_* of the backward's output
    const void* w;
    float scale;
    int rotate;                  // 0: the rows are only moved
};

struct Args {
    double turns[kMaxPairs];     // turns of a pair per unit of position
    int pair_end[3];             // first pair behind each axis; pairs behind the last do not turn
    int grid[3], stride[3], start[3], n_axes;
    const int* positions;
    long long pos_batch;         // elements
    int B, H, N, d;
    int log_lanes;
    int rot_lanes;               // lanes that hold rotated pairs of the half-split pairing; further lanes hold 16 bytes of the rest
    int half;                    // offset of the second channel of a pair of the half-split pairing
    float eps, inv_d;
    int n_tensors, chunks, per_chunk;                // every tensor's heads in `chunks` runs of `per_chunk`
    Units units;                 // forward
    Tensor t[3];
    float* part;                 // [tensor][chunk, block][d] partial sums of the weight gradients
    int want_dw;
};

// 16 bytes of a row as fp32: the first and the second channels of its NP pairs, two pairs in a register pair (rotation, norm and their
// gradients are then single instructions for two pairs).  Adjacent pairing: 16 consecutive bytes; half-split: 8 bytes at either place.
template <typename T, bool HALF> struct Vec;
template <bool HALF> struct Vec<__nv_bfloat16, HALF> {
    static constexpr int CH = 8, NP = 4, NQ = 2;
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ void unpack(const uint4& r, P2 (&a)[2], P2 (&b)[2]) {
        if (HALF) {
            a[0] = pair(lo(r.x), hi(r.x)); a[1] = pair(lo(r.y), hi(r.y));
            b[0] = pair(lo(r.z), hi(r.z)); b[1] = pair(lo(r.w), hi(r.w));
        } else {
            a[0] = pair(lo(r.x), lo(r.y)); a[1] = pair(lo(r.z), lo(r.w));
            b[0] = pair(hi(r.x), hi(r.y)); b[1] = pair(hi(r.z), hi(r.w));
        }
    }
    static __device__ __forceinline__ uint32_t two(float x, float y) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ uint4 pack(const P2 (&pa)[2], const P2 (&pb)[2]) {
        const float2 a0 = both(pa[0]), a1 = both(pa[1]), b0 = both(pb[0]), b1 = both(pb[1]);
        if (HALF) return make_uint4(two(a0.x, a0.y), two(a1.x, a1.y), two(b0.x, b0.y), two(b1.x, b1.y));
        return make_uint4(two(a0.x, b0.x), two(a0.y, b0.y), two(a1.x, b1.x), two(a1.y, b1.y));
    }
};
template <bool HALF> struct Vec<float, HALF> {
    static constexpr int CH = 4, NP = 2, NQ = 1;
    static __device__ __forceinline__ void unpack(const uint4& r, P2 (&a)[1], P2 (&b)[1]) {
        const float x = __uint_as_float(r.x), y = __uint_as_float(r.y), z = __uint_as_float(r.z), w = __uint_as_float(r.w);
        a[0] = HALF ? pair(x, y) : pair(x, z);
        b[0] = HALF ? pair(z, w) : pair(y, w);
    }
    static __device__ __forceinline__ uint4 pack(const P2 (&pa)[1], const P2 (&pb)[1]) {
        const float2 a = both(pa[0]), b = both(pb[0]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(HALF ? a.y : b.x), __float_as_uint(HALF ? b.x : a.y), __float_as_uint(b.y));
    }
};

// Where a lane's 16 bytes of a row are: off_a and off_b in bytes (off_b only counts in the half-split pairing).
template <typename T, bool HALF>
struct Place {
    int off_a, off_b;
    bool in;      // the lane has channels
    __device__ __forceinline__ Place(const Args& p, int l) {
        constexpr int CH = Vec<T, HALF>::CH, NP = Vec<T, HALF>::NP;
        in = l * CH < p.d;
        if (HALF && l < p.rot_lanes) {
            off_a = l * NP * (int)sizeof(T);
            off_b = off_a + p.half * (int)sizeof(T);
        } else {
            off_a = l * 16;
            off_b = off_a + 8;
        }
    }
    __device__ __forceinline__ uint4 load(const char* row) const {
        uint4 r;
        if (HALF) {
            const uint2 a = ld_once(reinterpret_cast<const uint2*>(row + off_a)), b = ld_once(reinterpret_cast<const uint2*>(row + off_b));
            r = make_uint4(a.x, a.y, b.x, b.y);
        } else {
            r = ld_once(reinterpret_cast<const uint4*>(row + off_a));
        }
        return r;
    }
    // Asynchronously into shared memory, both places next to one another.
    __device__ __forceinline__ void copy(uint4* to, const char* row) const {
        const uint32_t a = (uint32_t)__cvta_generic_to_shared(to);
        if (HALF) {
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(a), "l"(row + off_a) : "memory");
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(a + 8), "l"(row + off_b) : "memory");
        } else {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(a), "l"(row + off_a) : "memory");
        }
    }
    __device__ __forceinline__ void store(char* row, const uint4& r) const {
        if (HALF) {
            *reinterpret_cast<uint2*>(row + off_a) = make_uint2(r.x, r.y);
            *reinterpret_cast<uint2*>(row + off_b) = make_uint2(r.z, r.w);
        } else {
            *reinterpret_cast<uint4*>(row + off_a) = r;
        }
    }
};

// cos and sin of a lane's pairs at token n of batch b, times `scale`.  The angle is reduced to a fraction of a turn in 64 bits and the fraction, at
// most half a turn, rounded to fp32: 2^-26 turns, 9.4e-8 of the pair's length, hardly more than one of the roundings behind it (2^-24, 6e-8), and one
// sincospi in fp32 will do.  At position 2^31 the product's own rounding in 64 bits adds up to 2^-25 turns (frequencies up to 1).
template <typename T, bool HALF>
__device__ __forceinline__ void angles(const Args& p, const double* turns, int l, int b, int n, float scale, P2 (&c)[Vec<T, HALF>::NQ], P2 (&s)[Vec<T, HALF>::NQ]) {
    constexpr int NP = Vec<T, HALF>::NP;
    int pos[3] = {0, 0, 0};
#pragma unroll
    for (int a = 0; a < 3; ++a)
        if (a < p.n_axes) pos[a] = p.positions ? p.positions[b * p.pos_batch + (long long)n * p.n_axes + a] : n / p.stride[a] % p.grid[a] + p.start[a];
    float cs[NP], sn[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int pair_ = l * NP + i;
        cs[i] = 1.f;
        sn[i] = 0.f;
        if (pair_ < p.pair_end[2]) {
            const double x = (double)(pair_ < p.pair_end[0] ? pos[0] : pair_ < p.pair_end[1] ? pos[1] : pos[2]) * turns[pair_];
            sincospif(2.f * (float)(x - rint(x)), &sn[i], &cs[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < NP / 2; ++i) {
        c[i] = pair(cs[2 * i] * scale, cs[2 * i + 1] * scale);
        s[i] = pair(sn[2 * i] * scale, sn[2 * i + 1] * scale);
    }
}

// Sums over the lanes of a row of U values at once.  LOG: the lanes' number where it is known to the compiler (a loop costs as much as the
// shuffles), 0 else.
template <int LOG, int U>
__device__ __forceinline__ void lanes_sum(float (&v)[U], int log_lanes) {
    if (LOG) {
#pragma unroll
        for (int o = 1 << LOG >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] += __shfl_xor_sync(0xffffffffu, v[u], o);
    } else {
        for (int o = 1 << log_lanes >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] += __shfl_xor_sync(0xffffffffu, v[u], o);
    }
}

template <typename T, bool HALF>
__device__ __forceinline__ void norm_weights(const void* w, const Place<T, HALF>& at, P2 (&wa)[Vec<T, HALF>::NQ], P2 (&wb)[Vec<T, HALF>::NQ]) {
    if (w) {
        uint4 r = make_uint4(0, 0, 0, 0);
        if (at.in) r = at.load(static_cast<const char*>(w));
        Vec<T, HALF>::unpack(r, wa, wb);
    } else {
#pragma unroll
        for (int i = 0; i < Vec<T, HALF>::NQ; ++i) wa[i] = wb[i] = twice(1.f);
    }
}

template <typename T, bool HALF, bool NORM, int LOG>
__global__ void __launch_bounds__(kThreads, 4) forward_kernel(const __grid_constant__ Args p) {
    using V = Vec<T, HALF>;
    constexpr int NQ = V::NQ, U = 4;
    __shared__ double turns[kMaxPairs];
    if (threadIdx.x < kMaxPairs) turns[threadIdx.x] = p.turns[threadIdx.x];
    __syncthreads();
    const int log_lanes = LOG ? LOG : p.log_lanes;
    const int l = threadIdx.x & ((1 << log_lanes) - 1);
    const Unit unit = unit_of(p.units, blockIdx.x * (uint32_t)(kThreads >> log_lanes) + (threadIdx.x >> log_lanes));      // (without work: stays for the shuffles of its warp)
    const int b = unit.token / p.N, n = unit.token - b * p.N;
    const Tensor& t = p.t[unit.run / p.chunks];
    const int h0 = (unit.run % p.chunks) * p.per_chunk, count = min(p.H - h0, p.per_chunk);
    const Place<T, HALF> at(p, l);
    const bool mine = unit.live && at.in;
    const size_t row = (size_t)p.d * sizeof(T), head = row * p.N;
    const char* src = t.x + b * t.x_batch + n * t.x_token + h0 * row;
    char* dst = t.out + ((size_t)b * p.H + h0) * head + n * row;

    __shared__ uint4 staged[2][U][kThreads];
    auto fetch = [&](int h) {
        if (mine && h < count) {
            uint4(*to)[kThreads] = staged[h / U & 1];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u < count) at.copy(&to[u][threadIdx.x], src + u * row);
        }
        src += U * row;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fetch(0);      // (on their way while the angles are computed)
    fetch(U);
    P2 c[NQ], s[NQ], wa[NQ], wb[NQ];
    if (t.rotate) {
        angles<T, HALF>(p, turns, l, b, n, t.scale, c, s);
        if (NORM) norm_weights<T, HALF>(t.w, at, wa, wb);
    }
    for (int h = 0; h < p.per_chunk; h += U) {
        uint4 r[U];
        asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = mine && h + u < count ? staged[h / U & 1][u][threadIdx.x] : make_uint4(0, 0, 0, 0);
        if (t.rotate) {
            float scale[U];
            if (NORM) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    P2 x[NQ], y[NQ];
                    V::unpack(r[u], x, y);
                    P2 sum = mul2(x[0], x[0]);
#pragma unroll
                    for (int i = 1; i < NQ; ++i) sum = fma2(x[i], x[i], sum);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) sum = fma2(y[i], y[i], sum);
                    const float2 f = both(sum);
                    scale[u] = f.x + f.y;
                }
                lanes_sum<LOG, U>(scale, log_lanes);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                P2 x[NQ], y[NQ];
                V::unpack(r[u], x, y);
                if (NORM) {
                    const P2 q = twice(rsqrtf(fmaf(scale[u], p.inv_d, p.eps)));
#pragma unroll
                    for (int i = 0; i < NQ; ++i) {
                        x[i] = mul2(mul2(x[i], q), wa[i]);
                        y[i] = mul2(mul2(y[i], q), wb[i]);
                    }
                }
                P2 ya[NQ], yb[NQ];
#pragma unroll
                for (int i = 0; i < NQ; ++i) {
                    ya[i] = fma2(x[i], c[i], neg2(mul2(y[i], s[i])));
                    yb[i] = fma2(x[i], s[i], mul2(y[i], c[i]));
                }
                r[u] = V::pack(ya, yb);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (mine && h + u < count) at.store(dst + u * head, r[u]);
        fetch(h + 2 * U);
        dst += U * head;
    }
}

// The rows of a block's tokens one after the other: token tiles outside, the heads of its run inside.  Every group of lanes walks its own.
template <typename T, bool HALF>
struct Walk {
    const Args& p;
    const Tensor& t;
    uint32_t first;           // token of the block's first group
    int group, h, h0, count;
    bool in, mine;
    const char *dy, *x;
    __device__ __forceinline__ Walk(const Args& a, const Tensor& tensor, int g, int h0_, int count_, bool in_) : p(a), t(tensor), first(0), group(g), h(0), h0(h0_), count(count_), in(in_) {}
    __device__ __forceinline__ void tile(uint32_t at, int groups, uint32_t tokens, int& b, int& n) {
        first = at;
        h = 0;
        const bool live = first + group < tokens;
        mine = live && in;
        const uint32_t token = live ? first + group : first;
        b = token / p.N;
        n = token - b * p.N;
    }
    __device__ __forceinline__ void pointers(int b, int n, size_t row) {
        dy = t.dy + (((size_t)b * p.H + h0) * p.N + n) * row;
        x = t.x + b * t.x_batch + n * t.x_token + h0 * row;
    }
};

// A block stays with one run of heads of one tensor (blockIdx.y) and goes through tokens, so that its sums for the weight gradient
// can stay in registers until the end.  Rows come kStages ahead through shared memory, every lane its own 16 bytes (registers for as many
// rows in flight are not there): with two rows of registers ahead the backward of 2 x 24 x 32760 rows took 660 us.
template <typename T, bool HALF, bool NORM, int LOG>
__global__ void __launch_bounds__(kThreads, 3) backward_kernel(const __grid_constant__ Args p) {
    using V = Vec<T, HALF>;
    constexpr int NP = V::NP, NQ = V::NQ;
    __shared__ double turns[kMaxPairs];
    __shared__ float sums[kThreads * 2 * NP];
    __shared__ uint4 staged[kStages][NORM ? 2 : 1][kThreads];
    if (threadIdx.x < kMaxPairs) turns[threadIdx.x] = p.turns[threadIdx.x];
    __syncthreads();
    const int log_lanes = LOG ? LOG : p.log_lanes;
    const int l = threadIdx.x & ((1 << log_lanes) - 1), groups = kThreads >> log_lanes, group = threadIdx.x >> log_lanes;
    const int ti = blockIdx.y / p.chunks, chunk = blockIdx.y % p.chunks;
    const Tensor& t = p.t[ti];
    const int h0 = chunk * p.per_chunk, count = min(p.H - h0, p.per_chunk);
    const Place<T, HALF> at(p, l);
    const size_t row = (size_t)p.d * sizeof(T), head = row * p.N;
    const uint32_t tokens = (uint32_t)p.B * p.N, stride = gridDim.x * groups;
    const bool rotate = t.rotate;
    P2 wa[NQ], wb[NQ], da[NQ], db[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) da[i] = db[i] = 0;
    if (NORM && rotate) norm_weights<T, HALF>(t.w, at, wa, wb);

    Walk<T, HALF> ahead(p, t, group, h0, count, at.in);
    int ab, an;
    ahead.tile(blockIdx.x * groups, groups, tokens, ab, an);
    ahead.pointers(ab, an, row);
    auto fetch = [&](int stage) {
        if (ahead.first < tokens) {
            if (ahead.mine) {
                at.copy(&staged[stage][0][threadIdx.x], ahead.dy);
                if (NORM && rotate) at.copy(&staged[stage][NORM ? 1 : 0][threadIdx.x], ahead.x);
            }
            ahead.dy += head;
            ahead.x += row;
            if (++ahead.h == count) {
                ahead.tile(ahead.first + stride, groups, tokens, ab, an);
                if (ahead.first < tokens) ahead.pointers(ab, an, row);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i) fetch(i);
    int stage = 0;
    for (uint32_t first = blockIdx.x * groups; first < tokens; first += stride) {
        const bool live = first + group < tokens;
        const uint32_t token = live ? first + group : first;
        const int b = token / p.N, n = token - b * p.N;
        const bool mine = live && at.in;
        char* dst = t.out + b * t.o_batch + n * t.o_token + h0 * row;
        P2 c[NQ], s[NQ];
        if (rotate) angles<T, HALF>(p, turns, l, b, n, t.scale, c, s);
        for (int h = 0; h < count; ++h) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            uint4 r = make_uint4(0, 0, 0, 0), x = r;
            if (mine) {
                r = staged[stage][0][threadIdx.x];
                if (NORM && rotate) x = staged[stage][NORM ? 1 : 0][threadIdx.x];
            }
            if (rotate) {
                P2 ya[NQ], yb[NQ], ga[NQ], gb[NQ];
                V::unpack(r, ya, yb);
#pragma unroll
                for (int i = 0; i < NQ; ++i) {
                    ga[i] = fma2(ya[i], c[i], mul2(yb[i], s[i]));
                    gb[i] = fma2(yb[i], c[i], neg2(mul2(ya[i], s[i])));
                }
                if (NORM) {
                    P2 xa[NQ], xb[NQ], ss = 0, gx = 0;
                    V::unpack(x, xa, xb);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) {
                        ss = fma2(xb[i], xb[i], fma2(xa[i], xa[i], ss));
                        gx = fma2(mul2(gb[i], wb[i]), xb[i], fma2(mul2(ga[i], wa[i]), xa[i], gx));
                    }
                    const float2 f = both(ss), g = both(gx);
                    float sum[2] = {f.x + f.y, g.x + g.y};      // of x^2 and of g w x
                    lanes_sum<LOG, 2>(sum, log_lanes);
                    const float q = rsqrtf(fmaf(sum[0], p.inv_d, p.eps)), m = sum[1] * q * p.inv_d;
                    const P2 q2 = twice(q), less = twice(-m);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) {
                        const P2 ha = mul2(xa[i], q2), hb = mul2(xb[i], q2);
                        da[i] = fma2(ga[i], ha, da[i]);
                        db[i] = fma2(gb[i], hb, db[i]);
                        ga[i] = mul2(q2, fma2(ha, less, mul2(ga[i], wa[i])));
                        gb[i] = mul2(q2, fma2(hb, less, mul2(gb[i], wb[i])));
                    }
                }
                r = V::pack(ga, gb);
            }
            if (mine) at.store(dst, r);
            dst += row;
            fetch(stage);
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }
    }
    if (NORM && p.want_dw && rotate) {      // (uniform over the block)
        // Group after group: sums[group][channel].  A thread's rows (a few hundred) and the groups of a block (at most 256) are summed in fp32, the blocks in 64
        // bits (dw_kernel): a thread has eight sums and 80 registers in all, and in fp32 the error stays within 2^-24 a row of the sum of the magnitudes.
        constexpr int CH = V::CH;
        float* mine = sums + (size_t)group * CH * (1 << log_lanes);
        if (at.in) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int ca = HALF ? at.off_a / (int)sizeof(T) + i : l * CH + 2 * i, cb = HALF ? at.off_b / (int)sizeof(T) + i : ca + 1;
                const float2 fa = both(da[i / 2]), fb = both(db[i / 2]);
                mine[ca] = i & 1 ? fa.y : fa.x;
                mine[cb] = i & 1 ? fb.y : fb.x;
            }
        }
        __syncthreads();
        float* part = p.part + ((size_t)(ti * p.chunks + chunk) * gridDim.x + blockIdx.x) * p.d;
        for (int ch = threadIdx.x; ch < p.d; ch += kThreads) {
            float v = 0.f;
            for (int g = 0; g < groups; ++g) v += sums[(size_t)g * CH * (1 << log_lanes) + ch];
            part[ch] = v;
        }
    }
}

// Sums the partial rows of one tensor (blockIdx.y) for kDwChannels channels (blockIdx.x: a sector of every row) in a fixed order: rows by the
// block's slices, a warp's slices, warps.  What it takes is latency: all rows of a thread are on their way at once.
__global__ void __launch_bounds__(kDwThreads) dw_kernel(const float* part, int rows, int d, float* dw0, float* dw1) {
    constexpr int kSlices = kDwThreads / kDwChannels, kWarps = kDwThreads / 32;
    __shared__ double sums[kDwChannels][kWarps];
    const int ch = blockIdx.x * kDwChannels + threadIdx.x % kDwChannels, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    wait_for_previous_kernel();
    const float* mine = part + (size_t)blockIdx.y * rows * d;
    double v = 0.0;
    if (ch < d) {
#pragma unroll 8
        for (int r = threadIdx.x / kDwChannels; r < rows; r += kSlices) v += mine[(size_t)r * d + ch];
    }
#pragma unroll
    for (int o = 16; o >= kDwChannels; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane < kDwChannels) sums[lane][warp] = v;
    __syncthreads();
    if (warp < kDwChannels) {      // a channel a warp
        static_assert(kWarps == 32, "a warp has the sums of all warps");
        v = sums[warp][lane];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        float* dw = blockIdx.y ? dw1 : dw0;
        if (dw && lane == 0 && blockIdx.x * kDwChannels + warp < d) dw[blockIdx.x * kDwChannels + warp] = (float)v;
    }
}

}  // namespace heads
}  // namespace hla

using namespace hla;

struct hla_heads {
    hla_heads_config cfg;
    double turns[heads::kMaxPairs];
    int pair_end[3], rot;          // rotated channels
    bool grid_known;
    int log_lanes, sm_count;
};

namespace {

int elt_size(int dtype) { return dtype == HLA_BF16 ? 2 : 4; }

// How many blocks of the backward share the tokens, of `y` runs of heads.
int backward_blocks(const hla_heads* c, int y) {
    const long long tokens = (long long)c->cfg.B * c->cfg.N;
    const int groups = heads::kThreads >> c->log_lanes;
    const long long tiles = (tokens + groups - 1) / groups;
    // 16 blocks an SM in all, of which three run at once: V's blocks, which read half as much, and those with fewer tokens make room early.
    // 2 x 24 x 32760 rows: 492 us; with 12, four whole waves, 495 to 497 (without norm 190 and 192).
    const long long want = (16ll * c->sm_count + y - 1) / y;
    return (int)(tiles < want ? tiles : want);
}

// Heads that one group of lanes goes through.  All of a tensor's where the tokens alone fill the machine (the angles of a token are
// computed once per run); single heads for a few tokens.
int heads_per_run(const hla_heads* c, int tensors) {
    const long long tokens = (long long)c->cfg.B * c->cfg.N;
    const int groups = heads::kThreads >> c->log_lanes;
    int chunks = 1;
    while (chunks < c->cfg.H && chunks < 16384 && tokens * tensors * chunks < 4ll * c->sm_count * groups) chunks *= 2;      // (a grid has 65535 rows of blocks)
    if (chunks > c->cfg.H) chunks = c->cfg.H;
    return (c->cfg.H + chunks - 1) / chunks;
}

bool rows_ok(const hla_heads* c, const hla_rows* r) {
    const long long elt = elt_size(c->cfg.dtype);
    if (!r->data || (reinterpret_cast<uintptr_t>(r->data) & 15u)) return false;
    const long long width = (long long)c->cfg.H * c->cfg.d;
    const bool tokens = c->cfg.N > 1, batches = c->cfg.B > 1;      // a stride of one step is never taken
    constexpr long long most = 1ll << 56;      // (spans are computed in 64 bits)
    if (tokens && (r->token_stride < width || r->token_stride > most / c->cfg.N || (r->token_stride * elt & 15))) return false;
    if (batches && (r->batch_stride < width || r->batch_stride > most / c->cfg.B || (r->batch_stride * elt & 15))) return false;
    // rows do not share memory: a batch lies behind the one before, or a token's batches behind those of the token before
    if (tokens && batches && r->batch_stride < (c->cfg.N - 1) * r->token_stride + width && r->token_stride < (c->cfg.B - 1) * r->batch_stride + width) return false;
    return true;
}

size_t rows_span(const hla_heads* c, const hla_rows* r) {
    return (size_t)((c->cfg.B > 1 ? (c->cfg.B - 1) * r->batch_stride : 0) + (c->cfg.N > 1 ? (c->cfg.N - 1) * r->token_stride : 0) + (long long)c->cfg.H * c->cfg.d) *
           elt_size(c->cfg.dtype);
}

// Whether rows of a and rows of b, both written, may share memory.  Parts of one tensor do not: their strides are the same, the larger one a
// multiple of the smaller, and within the smaller one they lie side by side.
bool outputs_clash(const hla_heads* c, const hla_rows_out* a, const hla_rows_out* b) {
    const hla_rows x = {a->data, a->batch_stride, a->token_stride}, y = {b->data, b->batch_stride, b->token_stride};
    if (!overlap(x.data, rows_span(c, &x), y.data, rows_span(c, &y))) return false;
    const bool tokens = c->cfg.N > 1, batches = c->cfg.B > 1;
    if ((tokens && x.token_stride != y.token_stride) || (batches && x.batch_stride != y.batch_stride)) return true;
    const long long t = tokens ? x.token_stride : x.batch_stride, n = batches ? x.batch_stride : t;      // (with one row each, overlapping spans are the rows)
    const long long step = t < n ? t : n, elt = elt_size(c->cfg.dtype), width = (long long)c->cfg.H * c->cfg.d;
    if ((!tokens && !batches) || (t < n ? n : t) % step) return true;
    const uintptr_t from = reinterpret_cast<uintptr_t>(x.data), to = reinterpret_cast<uintptr_t>(y.data);
    const long long off = (long long)((from < to ? to - from : from - to) % (unsigned long long)(step * elt));
    return off < width * elt || step * elt - off < width * elt;
}

heads::Args common_args(const hla_heads* c, const int32_t* positions, int64_t pos_batch) {
    heads::Args a{};
    memcpy(a.turns, c->turns, sizeof(a.turns));
    int stride = 1;
    a.n_axes = c->rot ? c->cfg.n_axes : 0;
    for (int i = 2; i >= 0; --i) {
        a.pair_end[i] = c->pair_end[i];
        a.grid[i] = c->grid_known && i < c->cfg.n_axes ? c->cfg.grid[i] : 1;
        a.start[i] = c->cfg.start[i];
        a.stride[i] = stride;
        stride *= a.grid[i];
    }
    a.positions = positions;
    a.pos_batch = pos_batch;
    a.B = c->cfg.B; a.H = c->cfg.H; a.N = c->cfg.N; a.d = c->cfg.d;
    a.log_lanes = c->log_lanes;
    a.half = c->rot / 2;
    a.rot_lanes = c->rot * elt_size(c->cfg.dtype) / 16;
    a.eps = c->cfg.eps;
    a.inv_d = 1.f / (float)c->cfg.d;
    return a;
}

using Kernel = void (*)(heads::Args);

template <template <typename, bool, bool, int> class K, typename T, int LOG>
Kernel pick_of(bool half, bool norm) {
    return half ? (norm ? K<T, true, true, LOG>::get() : K<T, true, false, LOG>::get()) : (norm ? K<T, false, true, LOG>::get() : K<T, false, false, LOG>::get());
}
// Rows of 128 and 64 channels have kernels that know their lanes.
template <template <typename, bool, bool, int> class K>
Kernel pick(const hla_heads* c) {
    const bool half = c->cfg.pairing == HLA_PAIR_HALVES, norm = c->cfg.norm;
    if (c->cfg.dtype == HLA_BF16) {
        if (c->log_lanes == 4) return pick_of<K, __nv_bfloat16, 4>(half, norm);
        return c->log_lanes == 3 ? pick_of<K, __nv_bfloat16, 3>(half, norm) : pick_of<K, __nv_bfloat16, 0>(half, norm);
    }
    if (c->log_lanes == 5) return pick_of<K, float, 5>(half, norm);
    return c->log_lanes == 4 ? pick_of<K, float, 4>(half, norm) : pick_of<K, float, 0>(half, norm);
}
template <typename T, bool HALF, bool NORM, int LOG> struct Fwd { static Kernel get() { return heads::forward_kernel<T, HALF, NORM, LOG>; } };
template <typename T, bool HALF, bool NORM, int LOG> struct Bwd { static Kernel get() { return heads::backward_kernel<T, HALF, NORM, LOG>; } };

bool positions_ok(const hla_heads* c, const int32_t* positions, int64_t pos_batch) {
    if (!c->rot) return true;
    if (!positions) return c->grid_known;
    if (reinterpret_cast<uintptr_t>(positions) & 3u) return false;
    return pos_batch == 0 || (pos_batch >= (int64_t)c->cfg.N * c->cfg.n_axes && pos_batch < (1ll << 40));
}

// Whether n bytes at `out` share memory with a norm weight or with the positions that a call reads.
bool over_small_inputs(const hla_heads* c, const void* out, size_t n, const void* wq, const void* wk, const int32_t* positions, int64_t pos_batch) {
    const size_t weight = (size_t)c->cfg.d * elt_size(c->cfg.dtype);
    if ((wq && overlap(out, n, wq, weight)) || (wk && overlap(out, n, wk, weight))) return true;
    if (!positions || !c->rot) return false;
    const size_t read = ((size_t)(c->cfg.B - 1) * pos_batch + (size_t)c->cfg.N * c->cfg.n_axes) * sizeof(int32_t);
    return overlap(out, n, positions, read);
}

bool weight_ok(const hla_heads* c, const void* w) { return !w || (c->cfg.norm && aligned16(w)); }

}  // namespace

extern "C" {

hla_status hla_heads_create(const hla_heads_config* cfg, hla_heads** out) {
    if (out) *out = nullptr;
    if (!cfg || !out) return HLA_ERR_INVALID_ARG;
    const hla_heads_config& c = *cfg;
    if (c.B <= 0 || c.H <= 0 || c.N <= 0 || c.d <= 0) return HLA_ERR_INVALID_ARG;
    if (c.dtype != HLA_BF16 && c.dtype != HLA_F32) return HLA_ERR_INVALID_ARG;
    if (c.pairing != HLA_PAIR_ADJACENT && c.pairing != HLA_PAIR_HALVES) return HLA_ERR_INVALID_ARG;
    if (c.norm != 0 && c.norm != 1) return HLA_ERR_INVALID_ARG;
    if (c.n_axes < 0 || c.n_axes > 3) return HLA_ERR_INVALID_ARG;
    if (!isfinite(c.q_scale) || !isfinite(c.theta) || c.theta < 0.0 || !isfinite(c.eps) || c.eps < 0.f) return HLA_ERR_INVALID_ARG;
    int rot = 0;
    long long tokens = 1;
    bool any = false, all = true;
    for (int i = 0; i < c.n_axes; ++i) {
        if (c.axis_width[i] < 0 || (c.axis_width[i] & 1) || c.axis_width[i] > c.d || c.grid[i] < 0) return HLA_ERR_INVALID_ARG;
        rot += c.axis_width[i];
        any |= c.grid[i] > 0;
        all &= c.grid[i] > 0;
        if (c.grid[i] > 0 && tokens <= INT32_MAX) tokens *= c.grid[i];
        if (c.start[i] > INT32_MAX - (c.grid[i] > 0 ? c.grid[i] : 0)) return HLA_ERR_INVALID_ARG;
    }
    if (rot > c.d) return HLA_ERR_INVALID_ARG;
    if (any && (!all || tokens != c.N)) return HLA_ERR_INVALID_ARG;
    for (int p = 0; c.inv_freq && p < rot / 2; ++p)
        if (!isfinite(c.inv_freq[p])) return HLA_ERR_INVALID_ARG;
    const int per = 16 / elt_size(c.dtype);
    if (c.d > kMaxD || c.d % per) return HLA_ERR_UNSUPPORTED;                       // rows of whole 16-byte pieces
    if (c.pairing == HLA_PAIR_HALVES && rot % per) return HLA_ERR_UNSUPPORTED;
    if ((long long)c.B * c.H > 65535 || (long long)c.B * c.N > (1ll << 28)) return HLA_ERR_UNSUPPORTED;

    hla_heads* x = new (std::nothrow) hla_heads();
    if (!x) return HLA_ERR_NO_MEMORY;
    x->cfg = c;
    x->cfg.inv_freq = nullptr;
    if (c.eps == 0.f) x->cfg.eps = 1e-6f;
    if (c.q_scale == 0.f) x->cfg.q_scale = 1.f;
    if (c.theta == 0.0) x->cfg.theta = 10000.0;
    x->rot = rot;
    x->grid_known = any;
    for (int i = 0, pair = 0; i < 3; ++i) {
        const int np = i < c.n_axes ? c.axis_width[i] / 2 : 0;
        for (int j = 0; j < np; ++j, ++pair)
            x->turns[pair] = (c.inv_freq ? c.inv_freq[pair] : pow(x->cfg.theta, -(double)j / np)) / 6.283185307179586476925287;
        x->pair_end[i] = pair;
    }
    for (int p = 0; p < rot / 2; ++p)
        if (!isfinite(x->turns[p] * 0x1p31)) {      // (the farthest position; a product that is not finite has no fraction)
            delete x;
            return HLA_ERR_INVALID_ARG;
        }
    x->log_lanes = 0;
    while ((per << x->log_lanes) < c.d) ++x->log_lanes;
    x->sm_count = current_sm_count();
    *out = x;
    return HLA_OK;
}

size_t hla_heads_workspace_bytes(const hla_heads* c) {
    if (!c || !c->cfg.norm) return 0;
    // rows of partial sums: runs x blocks of the two normed tensors, whichever of the three are passed
    size_t most = 0;
    for (int tensors = 1; tensors <= 3; ++tensors) {
        const int per = heads_per_run(c, tensors), chunks = (c->cfg.H + per - 1) / per;
        const size_t rows = (size_t)(tensors < 2 ? tensors : 2) * chunks * backward_blocks(c, tensors * chunks);
        if (rows > most) most = rows;
    }
    return (most * c->cfg.d * 4 + 255) / 256 * 256;
}

hla_status hla_heads_forward(hla_heads* c, const hla_rows* q, const hla_rows* k, const hla_rows* v, const void* wq, const void* wk,
                             const int32_t* positions, int64_t positions_batch_stride, void* Q, void* K, void* V, void* cuda_stream) {
    if (!c || (!q && !k && !v)) return HLA_ERR_INVALID_ARG;
    const hla_rows* in[3] = {q, k, v};
    void* to[3] = {Q, K, V};
    const void* w[3] = {wq, wk, nullptr};
    if (!weight_ok(c, wq) || !weight_ok(c, wk) || !positions_ok(c, positions, positions_batch_stride)) return HLA_ERR_INVALID_ARG;
    const size_t dense = (size_t)c->cfg.B * c->cfg.H * c->cfg.N * c->cfg.d * elt_size(c->cfg.dtype);
    heads::Args a = common_args(c, positions, positions_batch_stride);
    const int elt = elt_size(c->cfg.dtype);
    for (int i = 0; i < 3; ++i) {
        if (!in[i] != !to[i]) return HLA_ERR_INVALID_ARG;
        if (!in[i]) continue;
        if (!rows_ok(c, in[i]) || !aligned16(to[i])) return HLA_ERR_INVALID_ARG;
        if (over_small_inputs(c, to[i], dense, wq, wk, positions, positions_batch_stride)) return HLA_ERR_INVALID_ARG;
        for (int j = 0; j < 3; ++j) {      // an output over an input, or over another output
            if (in[j] && in[j]->data && overlap(to[i], dense, in[j]->data, rows_span(c, in[j]))) return HLA_ERR_INVALID_ARG;
            if (j != i && to[j] && overlap(to[i], dense, to[j], dense)) return HLA_ERR_INVALID_ARG;
        }
        heads::Tensor& t = a.t[a.n_tensors++];
        t.x = static_cast<const char*>(in[i]->data);
        t.x_batch = in[i]->batch_stride * elt;
        t.x_token = in[i]->token_stride * elt;
        t.out = static_cast<char*>(to[i]);
        t.w = w[i];
        t.scale = i == 0 ? c->cfg.q_scale : 1.f;
        t.rotate = i < 2;
    }
    a.per_chunk = heads_per_run(c, a.n_tensors);
    a.chunks = (a.H + a.per_chunk - 1) / a.per_chunk;
    a.units = heads::units_of((uint32_t)a.B * a.N, a.n_tensors * a.chunks, a.log_lanes);
    const uint32_t groups = heads::kThreads >> a.log_lanes;
    const Kernel kern = pick<Fwd>(c);
    kern<<<(a.units.all + groups - 1) / groups, heads::kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    return cudaGetLastError() == cudaSuccess ? HLA_OK : HLA_ERR_CUDA;
}

hla_status hla_heads_backward(hla_heads* c, const void* dQ, const void* dK, const void* dV, const hla_rows* q, const hla_rows* k,
                              const void* wq, const void* wk, const int32_t* positions, int64_t positions_batch_stride,
                              const hla_rows_out* dq, const hla_rows_out* dk, const hla_rows_out* dv, void* dwq, void* dwk,
                              void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!c || (!dQ && !dK && !dV)) return HLA_ERR_INVALID_ARG;
    const void* dy[3] = {dQ, dK, dV};
    const hla_rows* x[3] = {q, k, nullptr};
    const hla_rows_out* to[3] = {dq, dk, dv};
    const void* w[3] = {wq, wk, nullptr};
    void* dw[2] = {dwq, dwk};
    if (!weight_ok(c, wq) || !weight_ok(c, wk) || !positions_ok(c, positions, positions_batch_stride)) return HLA_ERR_INVALID_ARG;
    const size_t dense = (size_t)c->cfg.B * c->cfg.H * c->cfg.N * c->cfg.d * elt_size(c->cfg.dtype);
    heads::Args a = common_args(c, positions, positions_batch_stride);
    const int elt = elt_size(c->cfg.dtype);
    float* sums[2] = {nullptr, nullptr};
    int normed = 0;
    for (int i = 0; i < 3; ++i) {
        if (!dy[i] != !to[i]) return HLA_ERR_INVALID_ARG;
        if (i < 2 && dw[i] && (!c->cfg.norm || !dy[i] || (reinterpret_cast<uintptr_t>(dw[i]) & 3u))) return HLA_ERR_INVALID_ARG;
        if (!dy[i]) continue;
        const bool needs_x = i < 2 && c->cfg.norm;
        const hla_rows o = {to[i]->data, to[i]->batch_stride, to[i]->token_stride};
        if (!aligned16(dy[i]) || !rows_ok(c, &o)) return HLA_ERR_INVALID_ARG;
        if (needs_x && (!x[i] || !rows_ok(c, x[i]))) return HLA_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (dy[j] && outputs_clash(c, to[i], to[j])) return HLA_ERR_INVALID_ARG;
        for (int j = 0; j < 3; ++j) {
            if (dy[j] && overlap(o.data, rows_span(c, &o), dy[j], dense)) return HLA_ERR_INVALID_ARG;
            if (j < 2 && c->cfg.norm && x[j] && x[j]->data && dy[j] && overlap(o.data, rows_span(c, &o), x[j]->data, rows_span(c, x[j]))) return HLA_ERR_INVALID_ARG;
        }
        heads::Tensor& t = a.t[a.n_tensors++];
        t.dy = static_cast<const char*>(dy[i]);
        t.out = static_cast<char*>(to[i]->data);
        t.o_batch = o.batch_stride * elt;
        t.o_token = o.token_stride * elt;
        if (needs_x) {
            t.x = static_cast<const char*>(x[i]->data);
            t.x_batch = x[i]->batch_stride * elt;
            t.x_token = x[i]->token_stride * elt;
            sums[normed++] = static_cast<float*>(dw[i]);
        }
        t.w = w[i];
        t.scale = i == 0 ? c->cfg.q_scale : 1.f;
        t.rotate = i < 2;
    }
    a.want_dw = sums[0] || sums[1];
    const size_t weights = (size_t)c->cfg.d * sizeof(float);
    if (dwq && dwk && overlap(dwq, weights, dwk, weights)) return HLA_ERR_INVALID_ARG;
    if (a.want_dw) {
        if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HLA_ERR_INVALID_ARG;
        if (workspace_bytes < hla_heads_workspace_bytes(c)) return HLA_ERR_WORKSPACE;
        a.part = static_cast<float*>(workspace);
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    a.per_chunk = heads_per_run(c, a.n_tensors);
    a.chunks = (a.H + a.per_chunk - 1) / a.per_chunk;
    const int blocks = backward_blocks(c, a.n_tensors * a.chunks);
    const Kernel kern = pick<Bwd>(c);
    kern<<<dim3(blocks, a.n_tensors * a.chunks), heads::kThreads, 0, st>>>(a);
    if (cudaGetLastError() != cudaSuccess) return HLA_ERR_CUDA;
    if (a.want_dw && !launch_behind(heads::dw_kernel, dim3((a.d + heads::kDwChannels - 1) / heads::kDwChannels, normed), heads::kDwThreads, st, (const float*)a.part, a.chunks * blocks, a.d, sums[0], sums[1]))
        return HLA_ERR_CUDA;
    return HLA_OK;
}

hla_status hla_heads_destroy(hla_heads* c) {
    if (!c) return HLA_ERR_INVALID_ARG;
    delete c;
    return HLA_OK;
}

}  // extern "C"
