// Gated linear recurrence over the tokens of a sequence, every channel for itself, and its backward.
//
//     h_t = a_t h_{t-1} + u_t,   a_t = exp(g_t) or 1 / (1 + exp(-g_t)),   u_t = x_t or (1 - a_t) x_t
//     lambda_t = dh_t + mu_{t+1},   mu_t = a_t lambda_t:   dx_t = lambda_t [(1 - a_t)],   dg_t = lambda_t (h_{t-1} [- x_t]) da_t/dg_t
//
// A step is the affine map h -> a h + u, and maps compose: (A2, H2) o (A1, H1) = (A2 A1, A2 H1 + H2).  The backward is the same
// recurrence in mu (mu_t = a_t mu_{t+1} + a_t dh_t) from the last token to the first, with the rest pointwise.
//
// What bounds it: memory would, if every input is read once; a channel is sequential and there are too few channels to fill the machine, so
// a sequence is cut.  A thread takes two channels of kRun consecutive tokens and composes their maps in registers; one warp of a block
// composes those of its runs; a cluster of up to eight blocks takes neighbouring pieces of the sequence and hands the maps of its blocks
// round through distributed shared memory, once for every kPieceOf tokens of a block.  The tokens stay in registers meanwhile and are gone
// through once more from the state that comes in; the next pieces are on their way into shared memory.  All orders are fixed: results
// do not depend on timing.  (Where the sequence is cut can depend on the GPU: the clusters that fit on it are counted.)  States, maps and sums are fp32.
//
// Forward of 32760 tokens, 1536 channels, bf16, sigmoid gates, convex: 70 to 74 us from GPU to GPU, 4.1 to 4.3 TB/s of 6.5, 24.5 instructions an
// element, 54 % of the issue slots.  The rest is the wait for the slowest block of a cluster (384 blocks on 148 SMs: three on some, two on others) and the round
// through the cluster.  Backward of two such sequences, log gates: 197 to 216 us, 4.7 to 5.1 TB/s, 30 instructions an element at 47 %; of one, sigmoid
// gates, convex: 147 to 151 us, 4.0 to 4.1 TB/s, two blocks an SM in 192 blocks of clusters of four.
#include "../../include/hla.h"

#include <algorithm>
#include <new>
#include <type_traits>

#include "hla_ops_common.cuh"
#include "hla_tc_prim.cuh"

namespace hla {
namespace scan {

constexpr int kThreads = 256;                    // and a warp that exchanges states
constexpr int kLanes = 16;                       // threads side by side on channels, two each
constexpr int kRuns = kThreads / kLanes;
template <typename T> constexpr int kRunOf = sizeof(T) == 2 ? 8 : 4;            // tokens of a thread: as many as its registers hold
template <typename T> constexpr int kPieceOf = kRuns * kRunOf<T>;               // tokens of a block between two exchanges
constexpr int kTile = 2 * kLanes;                // channels of a block
constexpr int kMaxCluster = 8;
constexpr int kBlocks = 3;                       // on an SM, where shared memory has room for them (kBlocksBack), and of the backward with many channels:
// With three its time depends on where the clusters come to lie (2 x 32760 x 1536, log gates: 199 to 285 us, with two 197).  Where clusters of
// eight fit at once three are better (32760 x 1536, log gates: 94 us, with two 123).
constexpr int kBlocksMany = 2;
constexpr int kSharedOfSm = 228 << 10, kSharedOfRuntime = 1 << 10;      // bytes of shared memory of an SM, and what a block takes beside its own

enum { kLog = 0, kSigmoid = 1 };

struct Args {
    int N, C, pieces;                            // pieces: exchanges of a block
    const char *x, *g, *h, *dh;
    char *out0, *out1;                           // forward: h, -; backward: dx, dg
    long long x_batch, x_token, g_batch, g_token;      // elements
    const float *in;                             // state that comes in (forward h0, backward dlast), or null
    const float *h0;                             // backward: the state before the first token, or null
    float* last;                                 // state that goes out (forward h_N, backward dh0), or null
    int segments, summary;                       // parts of a sequence that run side by side; 1: only their maps are wanted
    float2* maps;                                // [segment][B][C] maps of the segments, and the state that comes in
    unsigned long long* status;                  // becomes kTimedOut when a wait runs out, or null
};
// No call clears the record (that would be a launch more, and calls of other streams may be under way): it is a value that memory hardly holds by
// chance, and reading it takes it back.
constexpr unsigned long long kTimedOut = 0x8c5f3a9d17e264b1ull;
__device__ __forceinline__ void record_timeout(unsigned long long* status) {
    if (status) *status = kTimedOut;
}

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_blocks() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
// The .aligned barriers want all lanes of a warp at once, and so do bar.sync and bar.arrive; lanes may come here apart (one of them has prepared
// something, or a wait ended for one before the others), so each of them is behind a __syncwarp.
__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t of_block(uint32_t local, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
    return r;
}

__device__ __forceinline__ P2 one_minus(P2 x) { return fma2(x, twice(-1.f), twice(1.f)); }

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Two neighbouring channels of one token.  VEC: they are one aligned word of the outputs; else they go one by one, and `second` says whether
// the second channel exists.
template <typename T> struct Two;
template <> struct Two<__nv_bfloat16> {
    using Raw = uint32_t;
    static __device__ __forceinline__ P2 get(Raw r) { return pair(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u)); }
    template <bool VEC> static __device__ __forceinline__ void store(char* at, bool second, P2 v) {
        const float2 f = both(v);
        __nv_bfloat16* p = reinterpret_cast<__nv_bfloat16*>(at);
        if (VEC) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(f.x, f.y); return; }
        p[0] = __float2bfloat16_rn(f.x);
        if (second) p[1] = __float2bfloat16_rn(f.y);
    }
};
template <> struct Two<float> {
    using Raw = P2;
    static __device__ __forceinline__ P2 get(Raw r) { return r; }
    template <bool VEC> static __device__ __forceinline__ void store(char* at, bool second, P2 v) {
        if (VEC) { *reinterpret_cast<P2*>(at) = v; return; }
        const float2 f = both(v);
        float* p = reinterpret_cast<float*>(at);
        p[0] = f.x;
        if (second) p[1] = f.y;
    }
};

// Tokens on their way into shared memory.  Each warp has kStages buffers of its own for the tokens of its two runs (so that nothing but the
// warp waits for them), each of a row of kTile channels per token and input; a lane copies two pieces of 16 bytes of every input.
template <typename T>
struct Stage {
    static constexpr int kRowBytes = kTile * (int)sizeof(T), kRun = kRunOf<T>;
    static constexpr int kRunBytes = kRun * kRowBytes + (kRowBytes < 128 ? kRowBytes : 0);      // the two runs on different banks
    static constexpr int kBytes = 2 * kRunBytes;                                                // one input, one stage
    static constexpr int kPerRow = kRowBytes / 16, kHalf = 32 / kPerRow;                        // pieces of a row; rows that the warp copies at once
};
static_assert(Stage<float>::kHalf * 2 == 2 * kRunOf<float> && Stage<__nv_bfloat16>::kHalf * 2 == 2 * kRunOf<__nv_bfloat16>, "two pieces a lane");

// 16 bytes from global to shared memory, the first `elements` of them (the rest zeros), in words of WIDE bytes (16, or 4 where rows are only
// aligned to that).
template <typename T, int WIDE>
__device__ __forceinline__ void copy16(uint32_t to, const char* from, int elements) {
    if (WIDE == 16) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(elements > 0 ? 16 : 0) : "memory");
    } else {
        constexpr int per = 4 / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4 * i), "l"(elements > i * per ? from + 4 * i : from), "r"(elements > i * per ? 4 : 0) : "memory");
    }
}
// The same through registers, for 16-bit types whose rows are not aligned to four bytes.
__device__ __forceinline__ uint4 gather16(const char* from, int elements) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < elements) w[i / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(from)[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void put16(uint32_t to, const uint4& w) { asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory"); }
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void arrived() {
    asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
    __syncwarp();
}
template <typename R> __device__ __forceinline__ R read(uint32_t at);
template <> __device__ __forceinline__ uint32_t read<uint32_t>(uint32_t at) { uint32_t r; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(at)); return r; }
template <> __device__ __forceinline__ P2 read<P2>(uint32_t at) { P2 r; asm volatile("ld.shared.u64 %0, [%1];" : "=l"(r) : "r"(at)); return r; }

// One input of a block: where this lane's pieces are, token by token forwards (step > 0) or backwards.
template <typename T, int WIDE>
struct Input {
    using S = Stage<T>;
    static_assert(S::kHalf == S::kRun, "the second piece of a lane belongs to the second run");
    const char* at;
    long long step;           // bytes from a token to the next one in this order
    uint4 held[2];            // WIDE 2: between get and put
    __device__ __forceinline__ Input(const char* base, long long token0, long long step_, int lane32) : at(base + token0 * step_ + (lane32 / S::kPerRow) * step_ + (lane32 % S::kPerRow) * 16), step(step_) {}
    // Copies the tokens first + (0 .. 2 kRun - 1) of the warp; tokens at `end` or behind are zeros, channels behind the last too.
    __device__ __forceinline__ void fetch(uint32_t to, int first, int end, int channels, int lane32, int stride) {
        const int row = lane32 / S::kPerRow, col = lane32 % S::kPerRow;
        to += row * S::kRowBytes + col * 16;
        if (WIDE == 16 && first + 2 * S::kRun <= end && channels >= kTile) {
            copy16<T, 16>(to, at, 16);
            copy16<T, 16>(to + S::kRunBytes, at + S::kHalf * step, 16);
        } else {
            const int left = channels - col * (16 / (int)sizeof(T));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool in = first + row + i * S::kHalf < end && left > 0;
                const char* from = in ? at + i * S::kHalf * step : at;
                if (WIDE == 2) held[i] = gather16(from, in ? left : 0);
                else copy16<T, WIDE>(to + i * S::kRunBytes, from, in ? left : 0);
            }
        }
        at += stride * step;
    }
    // WIDE 2: what fetch has read goes into shared memory (behind the fetches of the other inputs, so that their latencies are one).
    __device__ __forceinline__ void put(uint32_t to, int lane32) {
        if (WIDE != 2) return;
        to += lane32 / S::kPerRow * S::kRowBytes + lane32 % S::kPerRow * 16;
        put16(to, held[0]);
        put16(to + S::kRunBytes, held[1]);
    }
};

// fp32 values of a state [B][C].
__device__ __forceinline__ P2 load_state(const float* p, size_t i, bool live, bool second) {
    return p && live ? pair(p[i], second ? p[i + 1] : 0.f) : 0;
}
// a and 1 - a.  Where the memory is long a is near 1, and an error of a relative 2^-22 of every a would add up over it; so the smaller of
// the two is formed first, with an error of its own size, and the larger is its difference to 1, correctly rounded.
template <int GATE>
__device__ __forceinline__ void gate(P2 g, P2& a, P2& rest) {
    if (GATE == kLog) {
        // 1 - exp(g) = -g (1 + g/2 (1 + g/3 (1 + ...))): six terms leave 5e-8 of it up to 1/4; beyond, a memory is at most four tokens
        P2 p = fma2(g, twice(1.f / 720), twice(1.f / 120));
        p = fma2(g, p, twice(1.f / 24));
        p = fma2(g, p, twice(1.f / 6));
        p = fma2(g, p, twice(0.5f));
        p = fma2(g, p, twice(1.f));
        const float2 x = both(g), near = both(mul2(mul2(g, twice(-1.f)), p)), t = both(mul2(g, twice(1.4426950408889634f)));
        const float2 e = make_float2(exp2_fast(t.x), exp2_fast(t.y));
        const bool nx = fabsf(x.x) < 0.25f, ny = fabsf(x.y) < 0.25f;
        rest = pair(nx ? near.x : 1.f - e.x, ny ? near.y : 1.f - e.y);
        a = pair(nx ? 1.f - near.x : e.x, ny ? 1.f - near.y : e.y);
    } else {
        // r = 1 / (1 + exp(-g)): the smaller of the two is e r or r, the larger its difference to 1
        const float2 x = both(g), t = both(mul2(g, twice(-1.4426950408889634f)));
        const P2 e = pair(exp2_fast(t.x), exp2_fast(t.y));
        const float2 d = both(add2(e, twice(1.f)));
        const P2 r = pair(reciprocal(d.x), reciprocal(d.y));
        const bool px = x.x >= 0.f, py = x.y >= 0.f;
        const float2 er = both(mul2(e, r)), rr = both(r);
        const P2 small = pair(px ? er.x : rr.x, py ? er.y : rr.y);
        const float2 v = both(small), w = both(one_minus(small));
        a = pair(px ? w.x : v.x, py ? w.y : v.y);
        rest = pair(px ? v.x : w.x, py ? v.y : w.y);
    }
}

struct Exchange {
    float2 warps_a[kRuns / 2][kLanes], warps_h[kRuns / 2][kLanes];      // maps (A, H) of this block's warps, two runs each
    float2 before[kRuns / 2][kLanes];                                   // the state before each warp's tokens
    float2 blocks[2][kMaxCluster][kTile];                               // maps of the cluster's blocks, of this piece and the next
    uint64_t full[2];                                                   // barriers: the maps of all blocks are there
};

__device__ __forceinline__ void arrive_at(int barrier) { __syncwarp(); asm volatile("bar.arrive %0, %1;" ::"r"(barrier), "n"(kThreads + 32) : "memory"); }
__device__ __forceinline__ void wait_at(int barrier) { __syncwarp(); asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(kThreads + 32) : "memory"); }
constexpr int kMapsThere = 1, kStatesThere = 2;

// The last warp of a block: a channel per lane.  It composes the maps of the block's warps, hands the result to the blocks of the cluster and,
// from theirs, finds the state before each warp's tokens.  (Done by every thread for itself, this was five instructions of 34 an element.)
// The other warps wait for it, so that what it reads it reads at once, ahead of the chain of products: 1 % of the whole.
//
// Every map of a piece is written by its block straight into the shared memory of all blocks of the cluster and counted by their barriers.
// A buffer is written again two pieces later: by then its writer has had this block's map of the piece between, which this block sends
// behind its reads of the buffer.
//
// A lane whose wait has run out takes no further part: it neither announces nor sends maps, its outputs from there on are not numbers, and
// the blocks that wait for it give up as well.  Going on, it would write over maps that others still wait for, arrive twice in one phase of a barrier, or
// end with maps on their way to it.
__device__ __forceinline__ float2 exchange(Exchange& e, int pieces, int rank, int blocks, float carry, unsigned long long* status) {
    const int lane = threadIdx.x & 31;
    const float *wa = &e.warps_a[0][0].x + lane, *wh = &e.warps_h[0][0].x + lane;
    float* before = &e.before[0][0].x + lane;
    bool lost = false;
    float product = 1.f;      // of all factors: (product, carry) is the map of all pieces
    uint32_t there[kMaxCluster], bars[kMaxCluster];      // where this block's maps go in every block, and their barriers
#pragma unroll
    for (int i = 0; i < kMaxCluster; ++i) {
        const int to = i < blocks ? i : 0;
        there[i] = of_block(tc::smem_u32(&e.blocks[0][rank][lane]), to);
        bars[i] = of_block(tc::smem_u32(&e.full[0]), to);
    }
    for (int s = 0; s < pieces; ++s) {
        const int buffer = s & 1;
        if (!lost && lane == 0) tc::mbar_arrive_expect_tx(&e.full[buffer], blocks * kTile * (int)sizeof(float2));
        wait_at(kMapsThere);
        float a[kRuns / 2], h[kRuns / 2], PA[kRuns / 2], PH[kRuns / 2], A = 1.f, H = 0.f;
#pragma unroll
        for (int w = 0; w < kRuns / 2; ++w) {
            a[w] = wa[w * kTile];
            h[w] = wh[w * kTile];
        }
#pragma unroll
        for (int w = 0; w < kRuns / 2; ++w) {
            PA[w] = A;
            PH[w] = H;
            H = fmaf(a[w], H, h[w]);
            A *= a[w];
        }
        if (!lost) {
#pragma unroll
            for (int i = 0; i < kMaxCluster; ++i)
                if (i < blocks)
                    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(there[i] + buffer * (uint32_t)sizeof(e.blocks[0])), "f"(A), "f"(H),
                                 "r"(bars[i] + buffer * (uint32_t)sizeof(uint64_t))
                                 : "memory");
        }
        if (!lost && !tc::mbar_wait(&e.full[buffer], (s >> 1) & 1)) {      // (two seconds)
            record_timeout(status);
            lost = true;
            carry = __int_as_float(0x7fc00000);
        }
        float2 q[kMaxCluster];
#pragma unroll
        for (int i = 0; i < kMaxCluster; ++i) q[i] = e.blocks[buffer][i][lane];      // (those behind the last block's are not used)
        float mine = carry;
#pragma unroll
        for (int i = 0; i < kMaxCluster; ++i) {
            if (i == rank) mine = carry;
            if (i < blocks) {
                carry = fmaf(q[i].x, carry, q[i].y);
                product *= q[i].x;
            }
        }
#pragma unroll
        for (int w = 0; w < kRuns / 2; ++w) before[w * kTile] = fmaf(PA[w], mine, PH[w]);
        arrive_at(kStatesThere);
    }
    return make_float2(product, carry);
}

// A warp's part of it: from the map (A, H) of this thread's run the state before its first token.  `during` runs while the maps are under way.
template <typename F>
__device__ __forceinline__ P2 state_before(Exchange& e, P2 A, P2 H, int warp, int lane, bool second, F during) {
    // the other run of the warp: (qa, qh); the second run's thread forms the map of both
    const P2 qa = __shfl_xor_sync(0xffffffffu, A, kLanes), qh = __shfl_xor_sync(0xffffffffu, H, kLanes);
    if (second) {
        e.warps_a[warp][lane] = both(mul2(A, qa));
        e.warps_h[warp][lane] = both(fma2(A, qh, H));
    }
    arrive_at(kMapsThere);
    during();
    wait_at(kStatesThere);
    const float2 f = e.before[warp][lane];
    const P2 h = pair(f.x, f.y);
    return second ? fma2(qa, h, qh) : h;
}

__device__ __forceinline__ void start(Exchange& e) {
    if (threadIdx.x == 0) {
        tc::mbar_init(&e.full[0], 1);
        tc::mbar_init(&e.full[1], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_sync();
}

// The state that goes into this block's part of a channel (the exchanging warp's lane), through the maps of the segments before its own.  Read
// before the cluster's first barrier: the state that goes out may lie over it.  (With segments, which end in any order, its copy from the first
// pass is read.)
__device__ __forceinline__ float state_in(const Args& p, int b, int segment) {
    const int c = blockIdx.y * kTile + (threadIdx.x & 31);
    if (p.summary || threadIdx.x < kThreads || c >= p.C) return 0.f;
    const size_t at = (size_t)b * p.C + c, all = (size_t)(gridDim.z / p.segments) * p.C;
    float carry = 0.f;
    if (p.in) carry = p.segments > 1 ? p.maps[p.segments * all + at].x : p.in[at];
    for (int i = 0; i < segment; ++i) {
        const float2 m = p.maps[i * all + at];
        carry = fmaf(m.x, carry, m.y);
    }
    return carry;
}
__device__ __forceinline__ void exchange_warp(Exchange& e, const Args& p, int rank, int blocks, int b, int segment, float carry) {
    const int c = blockIdx.y * kTile + (threadIdx.x & 31);
    const size_t at = (size_t)b * p.C + c, all = (size_t)(gridDim.z / p.segments) * p.C;
    const float2 map = exchange(e, p.pieces, rank, blocks, carry, p.status);
    if (rank != 0 || c >= p.C) return;
    if (p.summary) {
        p.maps[segment * all + at] = map;
        if (segment == 0 && p.in) p.maps[p.segments * all + at] = make_float2(p.in[at], 0.f);
    } else if (p.last && segment == p.segments - 1) {
        p.last[at] = map.y;
    }
}

template <typename T, int GATE, bool CONVEX, int WIDE>
__global__ void __launch_bounds__(kThreads + 32, kBlocks) forward_kernel(const __grid_constant__ Args p) {
    using V = Two<T>;
    constexpr bool VEC = WIDE >= 2 * (int)sizeof(T);      // two channels of the outputs are one word
    using S = Stage<T>;
    constexpr int kRun = kRunOf<T>, kPiece = kPieceOf<T>, kInputs = 2, kStages = 3;
    __shared__ Exchange e;
    extern __shared__ __align__(128) char staged[];
    const int lane32 = threadIdx.x & 31, lane = lane32 % kLanes, warp = threadIdx.x >> 5, rank = cluster_rank(), blocks = cluster_blocks();
    const bool late = lane32 >= kLanes;      // the second run of the warp
    const int c = blockIdx.y * kTile + 2 * lane, b = blockIdx.z / p.segments, segment = blockIdx.z % p.segments;
    const int channels = p.C - (int)blockIdx.y * kTile;
    const bool live = c < p.C, second = c + 1 < p.C;
    const long long gs = p.g_token * (int)sizeof(T), xs = p.x_token * (int)sizeof(T), os = (long long)p.C * (int)sizeof(T);
    const int stride = blocks * kPiece, tile = (int)blockIdx.y * kTile;
    int w0 = segment * p.pieces * stride + rank * kPiece + warp * 2 * kRun, t0 = w0 + late * kRun;      // first token of the warp, of the thread
    Input<T, WIDE> g(p.g + (b * p.g_batch + tile) * (int)sizeof(T), w0, gs, lane32), x(p.x + (b * p.x_batch + tile) * (int)sizeof(T), w0, xs, lane32);
    char* po = p.out0 + ((long long)b * p.N * p.C + c) * (int)sizeof(T) + t0 * os;
    const uint32_t mine = tc::smem_u32(staged) + warp * (kStages * kInputs * S::kBytes), own = late * S::kRunBytes + lane * 2 * (int)sizeof(T);
    auto fetch = [&](int piece, int stage) {
        if (piece < p.pieces) {
            const uint32_t to = mine + stage * (kInputs * S::kBytes);
            g.fetch(to, w0 + piece * stride, p.N, channels, lane32, stride);
            x.fetch(to + S::kBytes, w0 + piece * stride, p.N, channels, lane32, stride);
            g.put(to, lane32);
            x.put(to + S::kBytes, lane32);
        }
        commit();
    };
    if (warp < kThreads / 32) {
#pragma unroll
        for (int i = 0; i < kStages; ++i) fetch(i, i);
    }
    const float carry = state_in(p, b, segment);
    start(e);
    if (warp == kThreads / 32) {
        exchange_warp(e, p, rank, blocks, b, segment, carry);
        cluster_sync();      // no block leaves while another may still write into its shared memory
        return;
    }
    for (int s = 0, stage = 0; s < p.pieces; ++s) {
        arrived<kStages - 1>();
        const uint32_t from = mine + stage * (kInputs * S::kBytes) + own;
        P2 a[kRun], u[kRun];
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            P2 rest;
            gate<GATE>(V::get(read<typename V::Raw>(from + k * S::kRowBytes)), a[k], rest);
            u[k] = V::get(read<typename V::Raw>(from + S::kBytes + k * S::kRowBytes));
            if (CONVEX) u[k] = mul2(rest, u[k]);
        }
        const bool whole = live && t0 + kRun <= p.N;
        if (!whole) {      // behind the end nothing changes
#pragma unroll
            for (int k = 0; k < kRun; ++k)
                if (t0 + k >= p.N) { a[k] = twice(1.f); u[k] = 0; }
        }
        P2 A = a[0], H = u[0];
#pragma unroll
        for (int k = 1; k < kRun; ++k) {
            H = fma2(a[k], H, u[k]);
            A = mul2(a[k], A);
        }
        P2 h = state_before(e, A, H, warp, lane, late, [&] {
            __syncwarp();
            fetch(s + kStages, stage);
            stage = stage + 1 == kStages ? 0 : stage + 1;
        });
        if (p.summary) {
        } else if (whole) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                h = fma2(a[k], h, u[k]);
                V::template store<VEC>(po + k * os, second, h);
            }
        } else if (live) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                h = fma2(a[k], h, u[k]);
                if (t0 + k < p.N) V::template store<VEC>(po + k * os, second, h);
            }
        }
        po += stride * os;
        t0 += stride;
    }
    cluster_sync();
}

// Tokens are counted from the end: i = N - 1 - t; pointers go down.
template <typename T, int GATE, bool CONVEX, int WIDE, int BLOCKS>
__global__ void __launch_bounds__(kThreads + 32, BLOCKS) backward_kernel(const __grid_constant__ Args p) {
    using V = Two<T>;
    constexpr bool VEC = WIDE >= 2 * (int)sizeof(T);      // two channels of the outputs are one word
    using Raw = typename V::Raw;
    using S = Stage<T>;
    constexpr int kRun = kRunOf<T>, kPiece = kPieceOf<T>, kInputs = CONVEX ? 4 : 3, kStages = 2;
    __shared__ Exchange e;
    extern __shared__ __align__(128) char staged[];
    const int lane32 = threadIdx.x & 31, lane = lane32 % kLanes, warp = threadIdx.x >> 5, rank = cluster_rank(), blocks = cluster_blocks();
    const bool late = lane32 >= kLanes;      // the second run of the warp
    const int c = blockIdx.y * kTile + 2 * lane, b = blockIdx.z / p.segments, segment = blockIdx.z % p.segments;
    const int channels = p.C - (int)blockIdx.y * kTile;
    const bool live = c < p.C, second = c + 1 < p.C;
    const P2 h0 = load_state(p.h0, (size_t)b * p.C + c, live, second);
    const long long gs = p.g_token * (int)sizeof(T), xs = p.x_token * (int)sizeof(T), os = (long long)p.C * (int)sizeof(T);
    const int stride = blocks * kPiece, tile = (int)blockIdx.y * kTile;
    int w0 = segment * p.pieces * stride + rank * kPiece + warp * 2 * kRun, i0 = w0 + late * kRun;
    const long long dense = ((long long)b * p.N * p.C + tile) * (int)sizeof(T), end = p.N - 1;
    Input<T, WIDE> g(p.g + (b * p.g_batch + tile) * (int)sizeof(T) + end * gs, w0, -gs, lane32), d(p.dh + dense + end * os, w0, -os, lane32),
        h(p.h + dense + (end - 1) * os, w0, -os, lane32), x(CONVEX ? p.x + (b * p.x_batch + tile) * (int)sizeof(T) + end * xs : nullptr, w0, -xs, lane32);
    const long long out = dense + 2 * lane * (int)sizeof(T) + (end - i0) * os;
    char *po0 = p.out0 + out, *po1 = p.out1 + out;
    const uint32_t mine = tc::smem_u32(staged) + warp * (kStages * kInputs * S::kBytes), own = late * S::kRunBytes + lane * 2 * (int)sizeof(T);
    auto fetch = [&](int piece, int stage) {
        if (piece < p.pieces) {
            const uint32_t to = mine + stage * (kInputs * S::kBytes);
            const int first = w0 + piece * stride;
            g.fetch(to, first, p.N, channels, lane32, stride);
            d.fetch(to + S::kBytes, first, p.N, channels, lane32, stride);
            if (!p.summary) h.fetch(to + 2 * S::kBytes, first, p.N - 1, channels, lane32, stride);      // (the state before token 0 is h0)
            if (CONVEX && !p.summary) x.fetch(to + 3 * S::kBytes, first, p.N, channels, lane32, stride);
            g.put(to, lane32);
            d.put(to + S::kBytes, lane32);
            if (!p.summary) h.put(to + 2 * S::kBytes, lane32);
            if (CONVEX && !p.summary) x.put(to + 3 * S::kBytes, lane32);
        }
        commit();
    };
    if (warp < kThreads / 32) {
#pragma unroll
        for (int i = 0; i < kStages; ++i) fetch(i, i);
    }
    const float carry = state_in(p, b, segment);
    start(e);
    if (warp == kThreads / 32) {
        exchange_warp(e, p, rank, blocks, b, segment, carry);
        cluster_sync();      // no block leaves while another may still write into its shared memory
        return;
    }
    // one piece; WHOLE: the warp's tokens and channels are all there, and the sequence's first token is not among them
    auto piece = [&](auto whole_, int stage) {
        constexpr bool WHOLE = decltype(whole_)::value;
        const uint32_t from = mine + stage * (kInputs * S::kBytes) + own;
        P2 a[kRun], rest[kRun], A, M;
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            gate<GATE>(V::get(read<Raw>(from + k * S::kRowBytes)), a[k], rest[k]);
            if (!WHOLE && i0 + k >= p.N) a[k] = twice(1.f);      // (its dh was not read and is zero)
            const P2 dk = V::get(read<Raw>(from + S::kBytes + k * S::kRowBytes));
            M = mul2(a[k], k ? add2(dk, M) : dk);
            A = k ? mul2(a[k], A) : a[k];
        }
        P2 mu = state_before(e, A, M, warp, lane, late, [] {});
        if (p.summary) return;
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const P2 lam = add2(V::get(read<Raw>(from + S::kBytes + k * S::kRowBytes)), mu);
            mu = mul2(a[k], lam);
            P2 w = V::get(read<Raw>(from + 2 * S::kBytes + k * S::kRowBytes));
            if (!WHOLE && i0 + k == p.N - 1) w = h0;
            if (CONVEX) w = fma2(V::get(read<Raw>(from + 3 * S::kBytes + k * S::kRowBytes)), twice(-1.f), w);
            P2 dg = mul2(mu, w);      // lambda a (h_{t-1} - x)
            if (GATE == kSigmoid) dg = mul2(dg, rest[k]);
            const P2 dx = CONVEX ? mul2(lam, rest[k]) : lam;
            if (WHOLE || (live && i0 + k < p.N)) {
                V::template store<VEC>(po0 - k * os, WHOLE || second, dx);
                V::template store<VEC>(po1 - k * os, WHOLE || second, dg);
            }
        }
    };
    for (int s = 0, stage = 0; s < p.pieces; ++s) {
        arrived<kStages - 1>();
        if (w0 + s * stride + 2 * kRun < p.N && channels >= kTile) piece(std::true_type{}, stage);
        else piece(std::false_type{}, stage);
        __syncwarp();
        fetch(s + kStages, stage);
        stage ^= 1;
        po0 -= stride * os;
        po1 -= stride * os;
        i0 += stride;
    }
    cluster_sync();
}

// Waits, with a limit, for a barrier that nothing arrives at.
__global__ void wait_selftest_kernel(unsigned long long* status, unsigned long long limit_ns) {
    __shared__ uint64_t bar;
    if (threadIdx.x == 0) tc::mbar_init(&bar, 1);
    __syncwarp();
    if (!tc::mbar_wait(&bar, 0, limit_ns)) record_timeout(status);
}

template <typename T> constexpr int forward_bytes() { return kThreads / 32 * 3 * 2 * Stage<T>::kBytes; }
template <typename T> constexpr int backward_bytes(bool convex) { return kThreads / 32 * 2 * (convex ? 4 : 3) * Stage<T>::kBytes; }

// Blocks that shared memory has room for: three, but two of the convex backward of a 16-bit type (four inputs, 73728 bytes of stages a block).
constexpr int blocks_in_shared(int staged) {
    return kSharedOfSm / (staged + ((int)sizeof(Exchange) + 127) / 128 * 128 + kSharedOfRuntime);
}
template <typename T> constexpr int kBlocksForward = kBlocks < blocks_in_shared(forward_bytes<T>()) ? kBlocks : blocks_in_shared(forward_bytes<T>());
template <typename T, bool CONVEX> constexpr int kBlocksBack = kBlocks < blocks_in_shared(backward_bytes<T>(CONVEX)) ? kBlocks : blocks_in_shared(backward_bytes<T>(CONVEX));
static_assert(kBlocksForward<__nv_bfloat16> == kBlocks && kBlocksForward<float> == kBlocks, "what the forward's launch bounds say");
static_assert(kBlocksBack<__nv_bfloat16, true> >= kBlocksMany && kBlocksBack<float, true> >= kBlocksMany, "what the launch bounds of the backward with many channels say");

}  // namespace scan
}  // namespace hla

using namespace hla;

struct hla_scan {
    hla_scan_config cfg;
    int sm_count;
    void (*ready[2])(scan::Args);      // forward and backward kernels that were given their shared memory, on `device`
    int device;
    int blocks;                        // of a cluster of the backward
};

namespace {

using Kernel = void (*)(scan::Args);

template <template <typename, int, bool, int> class K, typename T, int WIDE>
Kernel pick_of(bool sigmoid, bool convex) {
    if (sigmoid) return convex ? K<T, scan::kSigmoid, true, WIDE>::get() : K<T, scan::kSigmoid, false, WIDE>::get();
    return convex ? K<T, scan::kLog, true, WIDE>::get() : K<T, scan::kLog, false, WIDE>::get();
}
template <template <typename, int, bool, int> class K>
Kernel pick(const hla_scan_config& c, int wide) {
    const bool s = c.gate == HLA_GATE_SIGMOID, v = c.convex;
    if (c.dtype == HLA_F32) return wide == 16 ? pick_of<K, float, 16>(s, v) : pick_of<K, float, 4>(s, v);
    return wide == 16 ? pick_of<K, __nv_bfloat16, 16>(s, v) : wide == 4 ? pick_of<K, __nv_bfloat16, 4>(s, v) : pick_of<K, __nv_bfloat16, 2>(s, v);
}
template <typename T, int GATE, bool CONVEX, int WIDE> struct Fwd { static Kernel get() { return scan::forward_kernel<T, GATE, CONVEX, WIDE>; } };
template <typename T, int GATE, bool CONVEX, int WIDE> struct Bwd { static Kernel get() { return scan::backward_kernel<T, GATE, CONVEX, WIDE, scan::kBlocksBack<T, CONVEX>>; } };
template <typename T, int GATE, bool CONVEX, int WIDE> struct BwdMany { static Kernel get() { return scan::backward_kernel<T, GATE, CONVEX, WIDE, scan::kBlocksMany>; } };

int elt_size(int dtype) { return dtype == HLA_BF16 ? 2 : 4; }

size_t dense_bytes(const hla_scan* c) { return (size_t)c->cfg.B * c->cfg.N * c->cfg.C * elt_size(c->cfg.dtype); }
size_t span(const hla_scan* c, long long batch, long long token) { return (size_t)((c->cfg.B - 1) * batch + (c->cfg.N - 1) * token + c->cfg.C) * elt_size(c->cfg.dtype); }

scan::Args common_args(const hla_scan* c) {
    scan::Args a{};
    a.N = c->cfg.N;
    a.C = c->cfg.C;
    a.x_batch = c->cfg.x_batch_stride; a.x_token = c->cfg.x_token_stride;
    a.g_batch = c->cfg.g_batch_stride; a.g_token = c->cfg.g_token_stride;
    return a;
}

// The words in which rows can be copied: 16 bytes where all rows are aligned to that, else 4, else (16-bit types, odd rows) 2.  (The dense
// tensors' rows, C elements, are told by C.)
int width(const hla_scan* c, const scan::Args& a) {
    const long long at = (long long)(reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.g));
    const long long bits = (a.C | a.x_batch | a.x_token | a.g_batch | a.g_token) * elt_size(c->cfg.dtype) | at;
    return !(bits & 15) ? 16 : !(bits & 3) ? 4 : 2;
}

long long columns_of(const hla_scan* c) { return (long long)((c->cfg.C + scan::kTile - 1) / scan::kTile) * c->cfg.B; }

// Blocks that run at once, as shared memory and launch bounds allow.
long long places_of(const hla_scan* c, bool back) {
    const int forward = c->cfg.dtype == HLA_BF16 ? scan::kBlocksForward<__nv_bfloat16> : scan::kBlocksForward<float>;
    const int convex = c->cfg.dtype == HLA_BF16 ? scan::kBlocksBack<__nv_bfloat16, true> : scan::kBlocksBack<float, true>;
    const int plain = c->cfg.dtype == HLA_BF16 ? scan::kBlocksBack<__nv_bfloat16, false> : scan::kBlocksBack<float, false>;
    return (long long)(!back ? forward : c->cfg.convex ? convex : plain) * c->sm_count;
}

// Parts of a sequence that run side by side: a first pass finds the map of each, and the pass proper starts every part from the states that the
// maps before it give.  It reads the inputs twice, so it is taken where at least three parts fit on the machine next to one another (75600 tokens:
// 64 channels 78 us in one part, 29 in 27; 512 channels backward 158 and 131 in three; 32760 tokens of 768 channels 49 and 70 in two, which
// is not taken).
int segments_of(const hla_scan* c, bool back, int blocks, long long pieces) {
    long long n = places_of(c, back) / (blocks * columns_of(c));
    if (n > pieces / 2) n = pieces / 2;
    return n < 3 ? 1 : (int)n;
}

int piece_of(const hla_scan* c) { return c->cfg.dtype == HLA_BF16 ? scan::kPieceOf<__nv_bfloat16> : scan::kPieceOf<float>; }

// Blocks of a cluster: as many as sequences and channels leave room for.  A second wave would wait for the first, and with fewer
// blocks an exchange is shorter.  Forward of 32760 tokens of 1536 channels: two sequences 123 us with four blocks, 133 with eight; three 166 with
// two, 192 with eight; four 231 with two, 252 with eight.  (Clusters do not fill the groups of SMs that they have to lie in: of eight blocks
// 48 run at once on 148 SMs, of four 104.)
int cluster_of(const hla_scan* c, bool back) {
    const long long columns = columns_of(c), room = places_of(c, back);
    auto fits = [&](int b) { return b * columns <= room - (b == 8 ? room / 8 : b == 4 ? room / 16 : 0); };
    int blocks = 1;
    while (blocks < scan::kMaxCluster && blocks * piece_of(c) < c->cfg.N && fits(2 * blocks)) blocks *= 2;
    return blocks;
}
// The backward has many channels where longer clusters would have been of use and found no room.
bool many(const hla_scan* c) {
    const int blocks = cluster_of(c, true);
    return blocks < scan::kMaxCluster && blocks * piece_of(c) < c->cfg.N;
}
// The parts of a call.
long long pieces_of(const hla_scan* c, int blocks) { return ((long long)c->cfg.N + blocks * piece_of(c) - 1) / (blocks * piece_of(c)); }
int parts_of(const hla_scan* c, bool back) {
    if (back && many(c)) return 1;
    const int blocks = cluster_of(c, back);
    return segments_of(c, back, blocks, pieces_of(c, blocks));
}

// With many channels the backward's clusters are those with the least waves x tokens a block, the fewest blocks where it is the same.  Two sequences (three waves of clusters of
// eight): 195 us, with four blocks (two waves) 200, with two (one) 225; three: 254 with two blocks, 307 with eight; four: 365 with four, 457 with two.
bool backward_cluster(const hla_scan* c, Kernel kern, int bytes, int& blocks) {
    long long best = 0;
    for (int b = 1; b <= scan::kMaxCluster && (b == 1 || b / 2 * piece_of(c) < c->cfg.N); b *= 2) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(b);
        cfg.blockDim = dim3(scan::kThreads + 32);
        cfg.dynamicSmemBytes = bytes;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = b;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        int active = 0;
        if (cudaOccupancyMaxActiveClusters(&active, kern, &cfg) != cudaSuccess || active <= 0) return false;
        const long long cost = (columns_of(c) + active - 1) / active * (scan::kMaxCluster / b);
        if (b == 1 || cost < best) {
            best = cost;
            blocks = b;
        }
    }
    return true;
}

hla_status launch(hla_scan* c, bool back, Kernel kern, int bytes, scan::Args& a, void* workspace, size_t workspace_bytes, cudaStream_t st) {
    const bool choose = back && many(c);
    int blocks = cluster_of(c, back);
    a.segments = parts_of(c, back);
    if (a.segments > 1) {
        if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HLA_ERR_INVALID_ARG;
        if (workspace_bytes < hla_scan_workspace_bytes(c)) return HLA_ERR_WORKSPACE;
        a.maps = reinterpret_cast<float2*>(static_cast<char*>(workspace) + HLA_SCAN_STATUS_BYTES);
    }
    if (workspace && !(reinterpret_cast<uintptr_t>(workspace) & 255u) && workspace_bytes >= HLA_SCAN_STATUS_BYTES) a.status = static_cast<unsigned long long*>(workspace);
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return HLA_ERR_CUDA;
    if (c->ready[back] != kern || c->device != dev) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return HLA_ERR_CUDA;
        if (choose && !backward_cluster(c, kern, bytes, c->blocks)) return HLA_ERR_CUDA;
        if (c->device != dev) c->ready[!back] = nullptr;
        c->ready[back] = kern;
        c->device = dev;
    }
    if (choose) blocks = c->blocks;
    const long long total = pieces_of(c, blocks);
    a.pieces = (int)((total + a.segments - 1) / a.segments);
    a.segments = (int)((total + a.pieces - 1) / a.pieces);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, (a.C + scan::kTile - 1) / scan::kTile, c->cfg.B * a.segments);
    cfg.blockDim = dim3(scan::kThreads + 32);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = blocks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (a.segments > 1) {
        a.summary = 1;
        if (cudaLaunchKernelEx(&cfg, kern, a) != cudaSuccess) return HLA_ERR_CUDA;
        a.summary = 0;
    }
    return cudaLaunchKernelEx(&cfg, kern, a) == cudaSuccess ? HLA_OK : HLA_ERR_CUDA;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool aligned_elt(const hla_scan* c, const void* p) { return reinterpret_cast<uintptr_t>(p) % elt_size(c->cfg.dtype) == 0; }

}  // namespace

extern "C" {

hla_status hla_scan_create(const hla_scan_config* cfg, hla_scan** out) {
    if (out) *out = nullptr;
    if (!cfg || !out) return HLA_ERR_INVALID_ARG;
    hla_scan_config c = *cfg;
    if (c.B <= 0 || c.N <= 0 || c.C <= 0) return HLA_ERR_INVALID_ARG;
    if (c.dtype != HLA_BF16 && c.dtype != HLA_F32) return HLA_ERR_INVALID_ARG;
    if (c.gate != HLA_GATE_LOG && c.gate != HLA_GATE_SIGMOID) return HLA_ERR_INVALID_ARG;
    if (c.convex != 0 && c.convex != 1) return HLA_ERR_INVALID_ARG;
    if (c.B > 65535 || c.N > (1 << 30) || c.C > 65535 * scan::kTile || (long long)c.B * c.N > (1ll << 48) / c.C) return HLA_ERR_UNSUPPORTED;
    if (c.x_token_stride == 0) c.x_token_stride = c.C;
    if (c.g_token_stride == 0) c.g_token_stride = c.C;
    if (c.x_batch_stride == 0) c.x_batch_stride = c.N * c.x_token_stride;
    if (c.g_batch_stride == 0) c.g_batch_stride = c.N * c.g_token_stride;
    const long long strides[4] = {c.x_token_stride, c.g_token_stride, c.x_batch_stride, c.g_batch_stride};
    for (int i = 0; i < 4; ++i)
        if (strides[i] < c.C || strides[i] > (1ll << 56) / (i < 2 ? c.N : c.B)) return HLA_ERR_INVALID_ARG;      // (spans are computed in 64 bits)
    hla_scan* x = new (std::nothrow) hla_scan();
    if (!x) return HLA_ERR_NO_MEMORY;
    x->cfg = c;
    x->sm_count = current_sm_count();
    x->device = -1;
    *out = x;
    return HLA_OK;
}

size_t hla_scan_workspace_bytes(const hla_scan* c) {
    if (!c) return 0;
    const size_t parts = std::max(parts_of(c, false), parts_of(c, true));
    return HLA_SCAN_STATUS_BYTES + (parts > 1 ? ((parts + 1) * c->cfg.B * c->cfg.C * sizeof(float2) + 255) / 256 * 256 : 0);
}

hla_status hla_scan_forward(hla_scan* c, const void* x, const void* g, const void* h0, void* h, void* h_last, void* workspace, size_t workspace_bytes,
                            void* cuda_stream) {
    if (!c || !x || !g || !h || !aligned_elt(c, x) || !aligned_elt(c, g) || !aligned16(h) || !aligned4(h0) || !aligned4(h_last)) return HLA_ERR_INVALID_ARG;
    scan::Args a = common_args(c);
    const size_t out = dense_bytes(c), state = (size_t)c->cfg.B * c->cfg.C * 4;
    if (overlap(h, out, x, span(c, a.x_batch, a.x_token)) || overlap(h, out, g, span(c, a.g_batch, a.g_token))) return HLA_ERR_INVALID_ARG;
    if ((h0 && overlap(h, out, h0, state)) || (h_last && overlap(h, out, h_last, state))) return HLA_ERR_INVALID_ARG;
    if (h_last && (overlap(h_last, state, x, span(c, a.x_batch, a.x_token)) || overlap(h_last, state, g, span(c, a.g_batch, a.g_token)))) return HLA_ERR_INVALID_ARG;
    if (h_last && h0 && h_last != h0 && overlap(h_last, state, h0, state)) return HLA_ERR_INVALID_ARG;
    a.x = static_cast<const char*>(x);
    a.g = static_cast<const char*>(g);
    a.out0 = static_cast<char*>(h);
    a.in = static_cast<const float*>(h0);
    a.last = static_cast<float*>(h_last);
    return launch(c, false, pick<Fwd>(c->cfg, width(c, a)), c->cfg.dtype == HLA_BF16 ? scan::forward_bytes<__nv_bfloat16>() : scan::forward_bytes<float>(), a, workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

hla_status hla_scan_backward(hla_scan* c, const void* x, const void* g, const void* h0, const void* h, const void* dh, const void* dh_last,
                             void* dx, void* dg, void* dh0, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!c || !g || !h || !dh || !dx || !dg || (c->cfg.convex && !x)) return HLA_ERR_INVALID_ARG;
    const void* dense[] = {h, dh, dx, dg};
    for (const void* p : dense)
        if (!aligned16(p)) return HLA_ERR_INVALID_ARG;
    if (!aligned_elt(c, x) || !aligned_elt(c, g) || !aligned4(h0) || !aligned4(dh_last) || !aligned4(dh0)) return HLA_ERR_INVALID_ARG;
    scan::Args a = common_args(c);
    const size_t n = dense_bytes(c), state = (size_t)c->cfg.B * c->cfg.C * 4;
    if (overlap(dx, n, dg, n)) return HLA_ERR_INVALID_ARG;
    for (void* o : {dx, dg}) {
        if ((c->cfg.convex && overlap(o, n, x, span(c, a.x_batch, a.x_token))) || overlap(o, n, g, span(c, a.g_batch, a.g_token)) || overlap(o, n, h, n) ||
            overlap(o, n, dh, n))
            return HLA_ERR_INVALID_ARG;
        for (const void* s : {h0, dh_last, (const void*)dh0})
            if (s && overlap(o, n, s, state)) return HLA_ERR_INVALID_ARG;
    }
    if (dh0) {
        if (overlap(dh0, state, h, n) || overlap(dh0, state, dh, n) || overlap(dh0, state, g, span(c, a.g_batch, a.g_token)) ||
            (c->cfg.convex && overlap(dh0, state, x, span(c, a.x_batch, a.x_token))))
            return HLA_ERR_INVALID_ARG;
        for (const void* s : {h0, dh_last})
            if (s && s != dh0 && overlap(dh0, state, s, state)) return HLA_ERR_INVALID_ARG;
    }
    a.x = static_cast<const char*>(c->cfg.convex ? x : nullptr);
    a.g = static_cast<const char*>(g);
    a.h = static_cast<const char*>(h);
    a.dh = static_cast<const char*>(dh);
    a.out0 = static_cast<char*>(dx);
    a.out1 = static_cast<char*>(dg);
    a.in = static_cast<const float*>(dh_last);
    a.h0 = static_cast<const float*>(h0);
    a.last = static_cast<float*>(dh0);
    return launch(c, true, many(c) ? pick<BwdMany>(c->cfg, width(c, a)) : pick<Bwd>(c->cfg, width(c, a)), c->cfg.dtype == HLA_BF16 ? scan::backward_bytes<__nv_bfloat16>(c->cfg.convex) : scan::backward_bytes<float>(c->cfg.convex), a, workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream));
}

hla_status hla_scan_last_device_status(hla_scan* c, void* workspace, void* cuda_stream) {
    if (!c || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HLA_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    unsigned long long word = 0;
    if (cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return HLA_ERR_CUDA;
    if (word != scan::kTimedOut) return HLA_OK;
    return cudaMemsetAsync(workspace, 0, sizeof(word), st) == cudaSuccess ? HLA_ERR_DEVICE_TIMEOUT : HLA_ERR_CUDA;
}

hla_status hla_scan_selftest_bounded_wait(hla_scan* c, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!c || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return HLA_ERR_INVALID_ARG;
    if (workspace_bytes < HLA_SCAN_STATUS_BYTES) return HLA_ERR_WORKSPACE;
    scan::wait_selftest_kernel<<<1, 32, 0, static_cast<cudaStream_t>(cuda_stream)>>>(static_cast<unsigned long long*>(workspace), 1000000ull);      // gives up after 1 ms
    return cudaGetLastError() == cudaSuccess ? HLA_OK : HLA_ERR_CUDA;
}

hla_status hla_scan_destroy(hla_scan* c) {
    if (!c) return HLA_ERR_INVALID_ARG;
    delete c;
    return HLA_OK;
}

}  // extern "C"
