// Gated linear recurrence over the tokens of a sequence, every channel for itself, and its backward.
//
//     h_t = a_t h_{t-1} + u_t,   a_t = exp(g_t) or 1 / (1 + exp(-g_t)),   u_t = x_t or (1 - a_t) x_t
//     lambda_t = dh_t + mu_{t+1},   mu_t = a_t lambda_t:   dx_t = lambda_t [(1 - a_t)],   dg_t = lambda_t (h_{t-1} [- x_t]) da_t/dg_t
//
// A step is the affine map h -> a h + u, and maps compose: (A2, H2) o (A1, H1) = (A2 A1, A2 H1 + H2).  The backward is the same
// recurrence in mu (mu_t = a_t mu_{t+1} + a_t dh_t) from the last token to the first, with the rest pointwise.
//
// What bounds it: memory, if every input is read once.  A channel is sequential and there are too few channels to fill the machine, so a
// sequence is cut: a thread takes two channels of kRun consecutive tokens, composes them in registers, and composes the runs before its
// own from shared memory; a cluster of up to eight blocks takes neighbouring pieces of the sequence and hands the maps of its blocks
// round through distributed shared memory, once for every kPiece tokens of a block.  The tokens stay in registers meanwhile and are gone
// through once more from the state that comes in; the next piece is loaded before the exchange.  All orders are fixed: results do not
// depend on timing.  States, maps and sums are fp32.
#include "../../include/hla.h"

#include <new>

#include "hla_ops_common.cuh"

namespace hla {
namespace scan {

constexpr int kThreads = 256;
constexpr int kLanes = 16;                       // threads side by side on channels, two each
constexpr int kRuns = kThreads / kLanes;
constexpr int kRun = 8;                          // tokens of a thread
constexpr int kPiece = kRuns * kRun;             // tokens of a block between two exchanges
constexpr int kTile = 2 * kLanes;                // channels of a block
constexpr int kMaxCluster = 8;

enum { kLog = 0, kSigmoid = 1 };

struct Args {
    int N, C, pieces;                            // pieces: exchanges of a block
    int vec;                                     // two channels can be moved as one word
    const char *x, *g, *h, *dh;
    char *out0, *out1;                           // forward: h, -; backward: dx, dg
    long long x_batch, x_token, g_batch, g_token;      // elements
    const float *in;                             // state that comes in (forward h0, backward dlast), or null
    const float *h0;                             // backward: the state before the first token, or null
    float* last;                                 // state that goes out (forward h_N, backward dh0), or null
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_blocks() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_remote(float4* local, uint32_t rank, const float4& v) {
    uint32_t a = (uint32_t)__cvta_generic_to_shared(local), r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(r), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// Two neighbouring channels of one token, as they are in memory.
template <typename T> struct Two;
template <> struct Two<__nv_bfloat16> {
    using Raw = uint32_t;
    static __device__ __forceinline__ Raw none() { return 0; }
    static __device__ __forceinline__ Raw load(const char* base, long long i, bool vec, bool second) {
        const unsigned short* p = reinterpret_cast<const unsigned short*>(base) + i;
        if (vec) return *reinterpret_cast<const uint32_t*>(p);
        return p[0] | (second ? (uint32_t)p[1] << 16 : 0u);
    }
    static __device__ __forceinline__ float2 get(Raw r) { return make_float2(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u)); }
    static __device__ __forceinline__ void store(char* base, long long i, bool vec, bool second, float2 v) {
        __nv_bfloat16* p = reinterpret_cast<__nv_bfloat16*>(base) + i;
        if (vec) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v.x, v.y); return; }
        p[0] = __float2bfloat16_rn(v.x);
        if (second) p[1] = __float2bfloat16_rn(v.y);
    }
};
template <> struct Two<float> {
    using Raw = float2;
    static __device__ __forceinline__ Raw none() { return make_float2(0.f, 0.f); }
    static __device__ __forceinline__ Raw load(const char* base, long long i, bool vec, bool second) {
        const float* p = reinterpret_cast<const float*>(base) + i;
        if (vec) return *reinterpret_cast<const float2*>(p);
        return make_float2(p[0], second ? p[1] : 0.f);
    }
    static __device__ __forceinline__ float2 get(Raw r) { return r; }
    static __device__ __forceinline__ void store(char* base, long long i, bool vec, bool second, float2 v) {
        float* p = reinterpret_cast<float*>(base) + i;
        if (vec) { *reinterpret_cast<float2*>(p) = v; return; }
        p[0] = v.x;
        if (second) p[1] = v.y;
    }
};

// a and 1 - a.  Where the memory is long a is near 1, and an error of a relative 2^-22 of every a would add up over it: expf, not the
// fast form; and 1 - a is formed without the difference.
template <int GATE, bool REST>
__device__ __forceinline__ void gate1(float g, float& a, float& rest) {
    if (GATE == kLog) {
        a = expf(g);
        if (REST) rest = -expm1f(g);
    } else {
        const float e = expf(-fabsf(g)), r = 1.f / (1.f + e), s = e * r;      // the larger and the smaller of the two
        a = g >= 0.f ? r : s;
        if (REST) rest = g >= 0.f ? s : r;
    }
}
template <int GATE, bool REST>
__device__ __forceinline__ void gate(float2 g, float2& a, float2& rest) {
    gate1<GATE, REST>(g.x, a.x, rest.x);
    gate1<GATE, REST>(g.y, a.y, rest.y);
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }

struct Exchange {
    float4 runs[kRuns][kLanes];                          // maps (A, A, H, H) of this block's runs
    float4 blocks[2][kMaxCluster][kLanes];               // of the cluster's blocks, of this piece and the next
};

// From the map (A, H) of this thread's run: the state before its first token; `carry`, the state before the cluster's piece, becomes
// the one behind it.  Every thread of the cluster calls this once a piece.
__device__ __forceinline__ float2 state_before(Exchange& e, float2 A, float2 H, float2& carry, int parity, int lane, int run, int rank, int blocks) {
    e.runs[run][lane] = make_float4(A.x, A.y, H.x, H.y);
    __syncthreads();
    float2 PA = make_float2(1.f, 1.f), PH = make_float2(0.f, 0.f);
    for (int r = 0; r < run; ++r) {
        const float4 q = e.runs[r][lane];
        const float2 qa = make_float2(q.x, q.y);
        PH = fma2(qa, PH, make_float2(q.z, q.w));
        PA = mul2(qa, PA);
    }
    if (run == kRuns - 1) {
        const float2 TA = mul2(A, PA), TH = fma2(A, PH, H);
        for (int i = 0; i < blocks; ++i) store_remote(&e.blocks[parity][rank][lane], i, make_float4(TA.x, TA.y, TH.x, TH.y));
    }
    cluster_arrive();
    cluster_wait();
    float2 mine = carry;
    for (int i = 0; i < blocks; ++i) {
        if (i == rank) mine = carry;
        const float4 q = e.blocks[parity][i][lane];
        carry = fma2(make_float2(q.x, q.y), carry, make_float2(q.z, q.w));
    }
    return fma2(PA, mine, PH);
}

template <typename T, int GATE, bool CONVEX>
__global__ void __launch_bounds__(kThreads) forward_kernel(const __grid_constant__ Args p) {
    using V = Two<T>;
    __shared__ Exchange e;
    const int lane = threadIdx.x % kLanes, run = threadIdx.x / kLanes, rank = cluster_rank(), blocks = cluster_blocks();
    const int c = blockIdx.y * kTile + 2 * lane, b = blockIdx.z;
    const bool live = c < p.C, second = c + 1 < p.C;
    const long long xo = b * p.x_batch + c, go = b * p.g_batch + c, oo = (long long)b * p.N * p.C + c;
    float2 carry = make_float2(0.f, 0.f);
    if (p.in && live) {
        carry.x = p.in[(size_t)b * p.C + c];
        if (second) carry.y = p.in[(size_t)b * p.C + c + 1];
    }
    typename V::Raw rg[kRun], rx[kRun];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            rg[k] = rx[k] = V::none();
            if (live && t0 + k < p.N) {
                rg[k] = V::load(p.g, go + (long long)(t0 + k) * p.g_token, p.vec, second);
                rx[k] = V::load(p.x, xo + (long long)(t0 + k) * p.x_token, p.vec, second);
            }
        }
    };
    int t0 = rank * kPiece + run * kRun;
    fetch(t0);
    for (int s = 0; s < p.pieces; ++s) {
        float2 a[kRun], u[kRun], A = make_float2(1.f, 1.f), H = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            float2 rest;
            gate<GATE, CONVEX>(V::get(rg[k]), a[k], rest);
            u[k] = V::get(rx[k]);
            if (CONVEX) u[k] = mul2(rest, u[k]);
            if (t0 + k >= p.N) { a[k] = make_float2(1.f, 1.f); u[k] = make_float2(0.f, 0.f); }      // behind the end nothing changes
            H = fma2(a[k], H, u[k]);
            A = mul2(a[k], A);
        }
        const int next = t0 + blocks * kPiece;
        if (s + 1 < p.pieces) fetch(next);
        float2 h = state_before(e, A, H, carry, s & 1, lane, run, rank, blocks);
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            h = fma2(a[k], h, u[k]);
            if (live && t0 + k < p.N) V::store(p.out0, oo + (long long)(t0 + k) * p.C, p.vec, second, h);
        }
        t0 = next;
    }
    if (p.last && rank == 0 && run == 0 && live) {
        p.last[(size_t)b * p.C + c] = carry.x;
        if (second) p.last[(size_t)b * p.C + c + 1] = carry.y;
    }
}

// Tokens are counted from the end: i = N - 1 - t.
template <typename T, int GATE, bool CONVEX>
__global__ void __launch_bounds__(kThreads) backward_kernel(const __grid_constant__ Args p) {
    using V = Two<T>;
    using Raw = typename V::Raw;
    __shared__ Exchange e;
    const int lane = threadIdx.x % kLanes, run = threadIdx.x / kLanes, rank = cluster_rank(), blocks = cluster_blocks();
    const int c = blockIdx.y * kTile + 2 * lane, b = blockIdx.z;
    const bool live = c < p.C, second = c + 1 < p.C;
    const long long xo = b * p.x_batch + c, go = b * p.g_batch + c, oo = (long long)b * p.N * p.C + c;
    float2 carry = make_float2(0.f, 0.f), h0 = make_float2(0.f, 0.f);
    if (live) {
        const size_t at = (size_t)b * p.C + c;
        if (p.in) { carry.x = p.in[at]; if (second) carry.y = p.in[at + 1]; }
        if (p.h0) { h0.x = p.h0[at]; if (second) h0.y = p.h0[at + 1]; }
    }
    Raw rg[kRun], rd[kRun], rh[kRun], rx[kRun];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const int t = p.N - 1 - (i0 + k);
            rg[k] = rd[k] = rh[k] = rx[k] = V::none();
            if (live && t >= 0) {
                rg[k] = V::load(p.g, go + (long long)t * p.g_token, p.vec, second);
                rd[k] = V::load(p.dh, oo + (long long)t * p.C, p.vec, second);
                if (t > 0) rh[k] = V::load(p.h, oo + (long long)(t - 1) * p.C, p.vec, second);
                if (CONVEX) rx[k] = V::load(p.x, xo + (long long)t * p.x_token, p.vec, second);
            }
        }
    };
    int i0 = rank * kPiece + run * kRun;
    fetch(i0);
    for (int s = 0; s < p.pieces; ++s) {
        constexpr bool REST = CONVEX || GATE == kSigmoid;
        float2 a[kRun], rest[kRun], d[kRun], w[kRun], A = make_float2(1.f, 1.f), M = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            gate<GATE, REST>(V::get(rg[k]), a[k], rest[k]);
            d[k] = V::get(rd[k]);
            w[k] = i0 + k == p.N - 1 ? h0 : V::get(rh[k]);
            if (CONVEX) { const float2 x = V::get(rx[k]); w[k].x -= x.x; w[k].y -= x.y; }
            if (i0 + k >= p.N) { a[k] = make_float2(1.f, 1.f); d[k] = make_float2(0.f, 0.f); }
            M = mul2(a[k], make_float2(d[k].x + M.x, d[k].y + M.y));
            A = mul2(a[k], A);
        }
        const int next = i0 + blocks * kPiece;
        if (s + 1 < p.pieces) fetch(next);
        float2 mu = state_before(e, A, M, carry, s & 1, lane, run, rank, blocks);
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const float2 lam = make_float2(d[k].x + mu.x, d[k].y + mu.y);
            mu = mul2(a[k], lam);
            float2 dg = mul2(mu, w[k]);      // lambda a (h_{t-1} - x)
            if (GATE == kSigmoid) dg = mul2(dg, rest[k]);
            const float2 dx = CONVEX ? mul2(lam, rest[k]) : lam;
            const int t = p.N - 1 - (i0 + k);
            if (live && t >= 0) {
                V::store(p.out0, oo + (long long)t * p.C, p.vec, second, dx);
                V::store(p.out1, oo + (long long)t * p.C, p.vec, second, dg);
            }
        }
        i0 = next;
    }
    if (p.last && rank == 0 && run == 0 && live) {
        p.last[(size_t)b * p.C + c] = carry.x;
        if (second) p.last[(size_t)b * p.C + c + 1] = carry.y;
    }
}

}  // namespace scan
}  // namespace hla

using namespace hla;

struct hla_scan {
    hla_scan_config cfg;
    int sm_count;
};

namespace {

using Kernel = void (*)(scan::Args);

template <template <typename, int, bool> class K, typename T>
Kernel pick_of(bool sigmoid, bool convex) {
    if (sigmoid) return convex ? K<T, scan::kSigmoid, true>::get() : K<T, scan::kSigmoid, false>::get();
    return convex ? K<T, scan::kLog, true>::get() : K<T, scan::kLog, false>::get();
}
template <template <typename, int, bool> class K>
Kernel pick(const hla_scan_config& c) {
    return c.dtype == HLA_BF16 ? pick_of<K, __nv_bfloat16>(c.gate == HLA_GATE_SIGMOID, c.convex) : pick_of<K, float>(c.gate == HLA_GATE_SIGMOID, c.convex);
}
template <typename T, int GATE, bool CONVEX> struct Fwd { static Kernel get() { return scan::forward_kernel<T, GATE, CONVEX>; } };
template <typename T, int GATE, bool CONVEX> struct Bwd { static Kernel get() { return scan::backward_kernel<T, GATE, CONVEX>; } };

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

// Whether two channels lie in one aligned word everywhere.
int vectors(const hla_scan* c, const scan::Args& a) {
    const uintptr_t word = 2 * elt_size(c->cfg.dtype), at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.g);
    return !((a.C | a.x_batch | a.x_token | a.g_batch | a.g_token) & 1) && at % word == 0;
}

hla_status launch(const hla_scan* c, Kernel kern, scan::Args& a, cudaStream_t st) {
    a.vec = vectors(c, a);
    int blocks = 1;      // of a cluster
    while (blocks < scan::kMaxCluster && blocks * scan::kPiece < a.N) blocks *= 2;
    a.pieces = (int)((a.N + (long long)blocks * scan::kPiece - 1) / (blocks * scan::kPiece));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, (a.C + scan::kTile - 1) / scan::kTile, c->cfg.B);
    cfg.blockDim = dim3(scan::kThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = blocks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
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
    if (c.B > 65535 || c.N > (1 << 30) || c.C > 65535 * scan::kTile) return HLA_ERR_UNSUPPORTED;
    if (c.x_token_stride == 0) c.x_token_stride = c.C;
    if (c.g_token_stride == 0) c.g_token_stride = c.C;
    if (c.x_batch_stride == 0) c.x_batch_stride = c.N * c.x_token_stride;
    if (c.g_batch_stride == 0) c.g_batch_stride = c.N * c.g_token_stride;
    const long long strides[4] = {c.x_token_stride, c.g_token_stride, c.x_batch_stride, c.g_batch_stride};
    for (int i = 0; i < 4; ++i)
        if (strides[i] < c.C || strides[i] > (i < 2 ? 1ll << 30 : 1ll << 46)) return HLA_ERR_INVALID_ARG;
    hla_scan* x = new (std::nothrow) hla_scan();
    if (!x) return HLA_ERR_NO_MEMORY;
    x->cfg = c;
    x->sm_count = current_sm_count();
    *out = x;
    return HLA_OK;
}

hla_status hla_scan_forward(hla_scan* c, const void* x, const void* g, const void* h0, void* h, void* h_last, void* cuda_stream) {
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
    return launch(c, pick<Fwd>(c->cfg), a, static_cast<cudaStream_t>(cuda_stream));
}

hla_status hla_scan_backward(hla_scan* c, const void* x, const void* g, const void* h0, const void* h, const void* dh, const void* dh_last,
                             void* dx, void* dg, void* dh0, void* cuda_stream) {
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
    return launch(c, pick<Bwd>(c->cfg), a, static_cast<cudaStream_t>(cuda_stream));
}

hla_status hla_scan_destroy(hla_scan* c) {
    if (!c) return HLA_ERR_INVALID_ARG;
    delete c;
    return HLA_OK;
}

}  // extern "C"
