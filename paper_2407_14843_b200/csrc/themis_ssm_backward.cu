// Gradients of the selective state space scan.
//
// With e_t = dy_t silu(z_t) and the adjoint state p_t[n] = C_t[n] e_t + a_{t+1}[n] p_{t+1}[n]
// (a_t = exp(s_t A)), everything follows from p_t and h_{t-1} of the same time:
//     dC_t = sum_d e_t h_t                 dB_t = sum_d s_t u_t p_t
//     ds_t = sum_n p_t (A a_t h_{t-1} + u_t B_t)       dA = sum_t p_t s_t a_t h_{t-1}
//     du_t = s_t sum_n p_t B_t + skip e_t              dz_t = dy_t v_t silu'(z_t)
// and dx, dconv from dc_t = du_t silu'(c_t) by the convolution read backwards.
//
// h runs forwards and p backwards, and h cannot be run backwards (a_t may be tiny), so it is
// recomputed: the forward pass left the state before every 16th time; a block takes one chunk of
// 16 times after the other from the end, walks it forwards once keeping every 4th state in shared
// memory, and then takes the sub-chunks of 4 times from the last to the first with their states and
// factors in registers.  That is two exponentials per state and time instead of a state table of
// 4 N bytes per time and channel in memory.
//
// A lane has two channels (for the paired 32-bit arithmetic) by four states, LPC lanes a channel.
// So B and C are fetched once for two channels, the sums over channels (dB, dC)
// begin inside the lane, and both they and the sums over states (v, sum p B, sum p a h A) end in
// reduce-scatters over few lanes.  Warps add their dB and dC through shared memory, blocks through
// partial sums that a second kernel adds in a fixed order (no atomics).
//
// Where rows x channels are few the time axis is cut into parts of whole chunks.  The adjoint
// after a part is linear in what follows it, so a first pass computes every part's own share and
// its steps' sum, and a small kernel joins them from the end.
#include <algorithm>

#include "themis_ssm.cuh"

namespace themis {
namespace {

constexpr int kChunk = THEMIS_SSM_CHUNK;
constexpr int kSub = 4;                  // times whose states are in registers at once
constexpr int kSubs = kChunk / kSub;
constexpr int kParExtra = 8;             // per channel beside dA: dconv (4), dconv_bias, dskip, ddt_bias, unused

// A channel's parameters in shared memory, in this order; the convolution's taps aligned at the newest.
enum { kW0, kW1, kW2, kW3, kConvBias, kDtBias, kSkip, kPars };

// Main kernel: LPC lanes to a channel, four states and two channels to a lane.  Four channels need
// 500 instructions for 32 channels and a time instead of 690 but leave half the warps, which take as
// long for them: 8 x 1024 x 1024 x 16 in bf16, 311 us against 316 when both were built; two channels
// stayed, whose kernel is 293 now.
template <typename T, int LPC> struct Shape {
    static constexpr int NP = 4 * LPC;                           // states, padded
    static constexpr int WARPS = LPC == 4 || LPC == 8 ? 8 : 4;
    static constexpr int THREADS = 32 * WARPS;
    static constexpr int CT = THREADS / LPC * 2;                 // channels of a block
    static constexpr int PAIRS = CT / 2;                         // element-wise parts: two channels to a thread ...
    static constexpr int TG = THREADS / PAIRS;                   // ... in this many groups of times
    static constexpr int E = kChunk / TG;
    static constexpr int PART = kSub * 2 * NP;                   // dB and dC of a warp and sub-chunk
    static constexpr int SLOT = THREADS * 8;                     // states before a sub-chunk
    static constexpr bool IN_SLOT = PART <= SLOT / WARPS;        // dB and dC fit a slot whose states have been used ...
    static constexpr bool SHARE = 2 * PART <= SLOT / WARPS;      // ... those of two sub-chunks do
    static constexpr int PARTS = (!IN_SLOT ? kSubs : SHARE ? 1 : 2) * WARPS * PART;
    // u, s, e; states before sub-chunks 1 .. kSubs - 2; B and C; partial sums; carry; parameters; dA
    static constexpr int FLOATS = 3 * kChunk * CT + (kSubs - 2) * SLOT + kChunk * 2 * NP + PARTS + (3 + kPars) * CT + SLOT;
    // The inputs of a chunk as they are; 16-bit ones twice, the next chunk's arriving meanwhile (two
    // buffers of 32-bit ones would leave room for one block to a multiprocessor).
    struct Raw {                                                 // (every array on the 16 bytes of a copy)
        alignas(16) T x[kChunk + 3][CT];                         // the three times before the chunk first
        alignas(16) T dt[kChunk][CT];
        alignas(16) T z[kChunk][CT];
        alignas(16) T dy[kChunk][CT];
        alignas(16) T b[kChunk][NP];
        alignas(16) T c[kChunk][NP];
    };
    static constexpr int BUFS = sizeof(T) == 4 ? 1 : 2;
    static constexpr size_t BYTES = FLOATS * sizeof(float) + BUFS * sizeof(Raw);
    // Blocks of a multiprocessor: by registers (128 a thread in blocks of 256, 168 in blocks of 128) and by
    // the shared memory that each takes with its reserved kilobyte, which leaves two for up to 8 states.  (A
    // training step 16 x 2048 x 1024 with 4 states, bf16: 1348 us compiled and planned for three, 1276 for two.)
    static constexpr int RESIDENT = std::min<int>(WARPS == 8 ? 2 : 3, 228 * 1024 / (BYTES + 1024));
};

// First pass over split parts: NPT states to a lane, LPC lanes to a channel, as in the forward kernel.
template <typename T, int NPT, int LPC> struct LocalShape {
    static constexpr int THREADS = 128;
    static constexpr int NP = NPT * LPC;
    static constexpr int CT = THREADS / LPC;
    static constexpr int PAIRS = CT / 2;
    static constexpr int E = kChunk * PAIRS / THREADS;
    struct Tile {
        struct Raw {                                             // (every array on the 16 bytes of a copy)
            alignas(16) T dt[kChunk][CT];
            alignas(16) T z[kChunk][CT];
            alignas(16) T dy[kChunk][CT];
            alignas(16) T c[kChunk][NP];
        } raw[2];
        alignas(16) float2 se[kChunk][CT];                       // s_t and e_t
        alignas(16) float c[kChunk][NP];
    };
};

// Reduce-scatter of 8 values over the G = 32 / LPC lanes of a warp that have the same states (LPC lanes
// apart): afterwards lane group c has values first(c) .. first(c) + LEFT - 1.
template <int LPC> struct GroupSum {
    static constexpr int G = 32 / LPC;
    static constexpr int LEFT = G >= 8 ? 1 : 8 / G;
    __device__ __forceinline__ static int first(int c)
    {
        return (c & 1) * 4 + (G > 2 ? ((c >> 1) & 1) * 2 : 0) + (G > 4 ? (c >> 2) & 1 : 0);
    }
    __device__ __forceinline__ static void run(float (&v)[8], int c)
    {
        int left = 8, bit = 1;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            if (bit < G) {
                const bool up = c & bit;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left / 2) {
                        const float give = up ? v[i] : v[i + left / 2], keep = up ? v[i + left / 2] : v[i];
                        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, bit * LPC);
                    }
                left /= 2;
                bit *= 2;
            }
        }
#pragma unroll
        for (; bit < G; bit *= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], bit * LPC);
    }
};

// Sum of 3 values of 2 channels over a channel's LPC lanes: afterwards lane `part` has those of channel
// part & 1 (in v[0]).
template <int LPC> struct StateSum {
    __device__ __forceinline__ static void run(float (&v)[2][3], int part)
    {
        const bool up = part & 1;
#pragma unroll
        for (int m = 0; m < 3; ++m) {
            const float give = up ? v[0][m] : v[1][m], keep = up ? v[1][m] : v[0][m];
            v[0][m] = keep + __shfl_xor_sync(0xffffffffu, give, 1);
        }
#pragma unroll
        for (int bit = 2; bit < LPC; bit *= 2)
#pragma unroll
            for (int m = 0; m < 3; ++m) v[0][m] += __shfl_xor_sync(0xffffffffu, v[0][m], bit);
    }
};

__device__ __forceinline__ float channel_par(const SsmParams &p, int m, int d)
{
    const int W = p.pr.conv_width;
    if (m <= kW3) return m - (4 - W) >= 0 ? p.in.conv_weight[(size_t)d * W + m - (4 - W)] : 0.0f;
    const float *v = m == kConvBias ? p.in.conv_bias : m == kDtBias ? p.in.dt_bias : p.in.skip;
    return v ? v[d] : 0.0f;
}

// the same order of additions as the forward kernel
__device__ __forceinline__ float conv_at(int width, float w0, float w1, float w2, float w3, float bias, float x0, float x1, float x2, float x3)
{
    float c = fmaf(w3, x3, bias);
    c = fmaf(w2, x2, c);
    if (width > 2) c = fmaf(w1, x1, c);
    if (width > 3) c = fmaf(w0, x0, c);
    return c;
}

// First pass over split parts: every part's share of the adjoint that it hands to the part before,
// sum_t exp(A sum_{r<=t} s_r) C_t e_t over its times (r, t from the part's first), and its steps' sum.
// (Times that do not exist add 0.)
template <typename T, int NPT, int LPC>
__global__ __launch_bounds__(128, sizeof(T) == 4 ? 3 : 4) void ssm_adjoint_local_kernel(const SsmParams p)
{
    using S = LocalShape<T, NPT, LPC>;
    constexpr int CT = S::CT, NP = S::NP, E = S::E, THREADS = S::THREADS;
    extern __shared__ __align__(16) float smem[];
    using Tile = typename S::Tile;
    using Raw = typename Tile::Raw;
    static_assert(sizeof(Raw) % 16 == 0 && offsetof(Raw, dt) % 16 == 0 && offsetof(Raw, z) % 16 == 0 && offsetof(Raw, dy) % 16 == 0 &&
                      offsetof(Raw, c) % 16 == 0 && offsetof(Tile, raw) % 16 == 0 && offsetof(Tile, se) % 16 == 0 && offsetof(Tile, c) % 16 == 0,
                  "rows are copied and read 16 bytes at a time");
    auto &s = *reinterpret_cast<Tile *>(smem);

    const int D = p.pr.channels, N = p.pr.state, tid = threadIdx.x;
    const int b = blockIdx.x, split = blockIdx.z + 1;       // nothing needs the first part's share
    int g, d0, nd;
    tile_of_block(p, blockIdx.y, CT, g, d0, nd);
    const int t_begin = split * p.split_len, t_end = min(row_length(p, b), min(p.pr.length, t_begin + p.split_len));
    const T *dtp = (const T *)p.in.dt + (size_t)b * p.pr.dt_row + d0, *dyp = (const T *)p.dy + (size_t)b * p.pr.length * D + d0;
    const T *zp = p.in.z ? (const T *)p.in.z + (size_t)b * p.pr.z_row + d0 : nullptr;
    const T *cp = (const T *)p.in.c + (size_t)b * p.pr.c_row + (size_t)g * p.pr.c_group;
    const int pc = 2 * (tid % S::PAIRS), tg = tid / S::PAIRS;
    float db[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) db[j] = p.in.dt_bias ? p.in.dt_bias[d0 + min(pc + j, nd - 1)] : 0.0f;
    const int rc = tid / LPC, part = tid % LPC, dr = d0 + min(rc, nd - 1), n0 = part * NPT;
    f32x2 a2[NPT / 2], acc[NPT / 2];
#pragma unroll
    for (int i = 0; i < NPT / 2; ++i) {
        const int n = n0 + 2 * i;
        a2[i] = pack2(n < N ? log2_rate(p.in.a[(size_t)dr * N + n]) : 0.0f, n + 1 < N ? log2_rate(p.in.a[(size_t)dr * N + n + 1]) : 0.0f);
        acc[i] = pack2(0.0f, 0.0f);
    }
    float sum = 0.0f;

    const RowCopy<T, CT, kChunk, THREADS> copy_dt(dtp, p.pr.dt_time, nd, tid), copy_z(zp, p.pr.z_time, nd, tid), copy_dy(dyp, D, nd, tid);
    const RowCopy<T, NP, kChunk, THREADS> copy_c(cp, p.pr.c_time, N, tid);
    auto fetch = [&](int t0) {
        auto &r = s.raw[(t0 - t_begin) / kChunk & 1];
        copy_dt.run(&r.dt[0][0], t0, t_end, tid);
        if (zp) copy_z.run(&r.z[0][0], t0, t_end, tid);
        copy_dy.run(&r.dy[0][0], t0, t_end, tid);
        copy_c.run(&r.c[0][0], t0, t_end, tid);
        copy_commit();
    };
    if (N < NP) {                                        // the padded states' C stays 0
        for (int i = tid; i < 2 * kChunk * NP; i += THREADS) (&s.raw[i / (kChunk * NP)].c[0][0])[i % (kChunk * NP)] = from_f32<T>(0.0f);
        __syncthreads();
    }
    if (t_begin < t_end) fetch(t_begin);
    for (int t0 = t_begin; t0 < t_end; t0 += kChunk) {
        copy_wait<0>();
        __syncthreads();
        if (t0 + kChunk < t_end) fetch(t0 + kChunk);
        const auto &r = s.raw[(t0 - t_begin) / kChunk & 1];
        const int live = min(kChunk, t_end - t0);
#pragma unroll 4
        for (int i = 0; i < E; ++i) {
            const int t = tg * E + i;
            float dv[2], e[2], z[2], st[2];
            get_pair(&r.dt[t][pc], dv);
            get_pair(&r.dy[t][pc], e);
            if (zp) get_pair(&r.z[t][pc], z);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                st[j] = t < live ? softplus(dv[j] + db[j]) : 0.0f;
                if (zp) e[j] *= silu(z[j]);
                if (t >= live) e[j] = 0.0f;
            }
            *reinterpret_cast<float4 *>(&s.se[t][pc]) = make_float4(st[0], e[0], st[1], e[1]);
        }
        for (int i = tid; i < kChunk * NP / 2; i += THREADS) {
            float v[2];
            get_pair(&r.c[0][0] + 2 * i, v);
            *reinterpret_cast<float2 *>(&s.c[0][0] + 2 * i) = make_float2(v[0], v[1]);
        }
        __syncthreads();
#pragma unroll 4
        for (int t = 0; t < kChunk; ++t) {
            const float2 se = s.se[t][rc];
            sum += se.x;
            const f32x2 ss = pack2(sum, sum), ee = pack2(se.y, se.y);
            const float4 *C = reinterpret_cast<const float4 *>(&s.c[t][n0]);
#pragma unroll
            for (int i = 0; i < NPT / 4; ++i) {
                const float4 c = C[i];
                acc[2 * i] = fma2(decay2(ss, a2[2 * i]), mul2(ee, pack2(c.x, c.y)), acc[2 * i]);
                acc[2 * i + 1] = fma2(decay2(ss, a2[2 * i + 1]), mul2(ee, pack2(c.z, c.w)), acc[2 * i + 1]);
            }
        }
    }
    if (rc < nd) {
        float *to = p.split_state + (((size_t)b * p.splits + split) * D + dr) * N + n0;
#pragma unroll
        for (int i = 0; i < NPT / 2; ++i) {
            float lo, hi;
            unpack2(acc[i], lo, hi);
            if (n0 + 2 * i < N) to[2 * i] = lo;
            if (n0 + 2 * i + 1 < N) to[2 * i + 1] = hi;
        }
        if (part == 0) p.split_step[((size_t)b * p.splits + split) * D + dr] = sum;
    }
}

// Joins the parts from the end: split_state[s] holds part s's share and gets the adjoint (already
// multiplied by the next time's factor) that enters part s from its right.
__global__ void ssm_adjoint_join_kernel(const SsmParams p)
{
    const int DN = p.pr.channels * p.pr.state, N = p.pr.state, D = p.pr.channels;
    const int e = blockIdx.y * blockDim.x + threadIdx.x, b = blockIdx.x;
    if (e >= DN) return;
    const int d = e / N;
    const float a = log2_rate(p.in.a[e]);
    float *st = p.split_state + (size_t)b * p.splits * DN + e;
    const float *sum = p.split_step + (size_t)b * p.splits * D + d;
    float q = 0.0f;
    constexpr int U = 8;
    for (int s0 = p.splits - 1; s0 >= 0; s0 -= U) {
        float own[U], step[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool in = s0 - i >= 1;
            own[i] = in ? st[(size_t)(s0 - i) * DN] : 0.0f;
            step[i] = in ? sum[(size_t)(s0 - i) * D] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (s0 - i < 0) break;
            st[(size_t)(s0 - i) * DN] = q;
            q = fmaf(exp2f(a * step[i]), q, own[i]);
        }
    }
}

template <typename T, int LPC>
__global__ __launch_bounds__(Shape<T, LPC>::THREADS, Shape<T, LPC>::RESIDENT) void ssm_backward_kernel(const SsmParams p)
{
    using S = Shape<T, LPC>;
    constexpr int CT = S::CT, NP = S::NP, E = S::E, THREADS = S::THREADS, WARPS = S::WARPS, PAIRS = S::PAIRS;
    extern __shared__ __align__(16) float smem[];
    float *at_ = smem;
    auto take = [&](int n) { float *q = at_; at_ += n; return q; };
    float(*s_u)[CT] = reinterpret_cast<float(*)[CT]>(take(kChunk * CT));        // u_t, then s_t sum_n p B, then dc_t
    float(*s_step)[CT] = reinterpret_cast<float(*)[CT]>(take(kChunk * CT));     // s_t, then ds_t
    float(*s_e)[CT] = reinterpret_cast<float(*)[CT]>(take(kChunk * CT));        // e_t, then sum_n C h
    float *s_h = take((kSubs - 2) * S::SLOT);                                   // states before sub-chunks 1 .. kSubs - 2
    float(*s_bc)[2 * NP] = reinterpret_cast<float(*)[2 * NP]>(take(kChunk * 2 * NP));
    float *s_part = take(S::PARTS);                                             // dB and dC of sub-chunks without a slot
    float *s_dA = take(S::SLOT);
    float(*s_carry)[CT] = reinterpret_cast<float(*)[CT]>(take(3 * CT));         // dc of the next chunk's first times
    float(*s_par)[CT] = reinterpret_cast<float(*)[CT]>(take(kPars * CT));
    using Raw = typename S::Raw;
    static_assert(S::RESIDENT == Shape<float, LPC>::RESIDENT && S::CT == Shape<float, LPC>::CT, "the plan takes both from the 32-bit shape");
    static_assert(sizeof(Raw) % 16 == 0 && offsetof(Raw, x) % 16 == 0 && offsetof(Raw, dt) % 16 == 0 && offsetof(Raw, z) % 16 == 0 &&
                      offsetof(Raw, dy) % 16 == 0 && offsetof(Raw, b) % 16 == 0 && offsetof(Raw, c) % 16 == 0,
                  "rows are copied and read 16 bytes at a time");
    static_assert(CT % 4 == 0 && S::SLOT % 4 == 0 && NP % 4 == 0 && S::PARTS % 4 == 0 && S::FLOATS % 4 == 0, "so are the arrays before it");
    Raw *s_raw = reinterpret_cast<Raw *>(at_);

    const int D = p.pr.channels, N = p.pr.state, W = p.pr.conv_width, L = p.pr.length, G = p.pr.groups;
    const int b = blockIdx.x, split = blockIdx.z, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    int g, d0, nd;
    tile_of_block(p, blockIdx.y, CT, g, d0, nd);
    const int tile_in_group = blockIdx.y % p.tiles_per_group;
    const int len = row_length(p, b);
    const int t_begin = split * p.split_len, t_end = min(L, t_begin + p.split_len);

    // element-wise role: two channels, E consecutive times
    const int pc = 2 * (tid % PAIRS), tg = tid / PAIRS, de = d0 + min(pc, (nd - 1) & ~1);
    const bool own = pc < nd, two = pc + 1 < nd;
    const T *xp = (const T *)p.in.x + (size_t)b * p.pr.x_row + d0, *dtp = (const T *)p.in.dt + (size_t)b * p.pr.dt_row + d0;
    const T *zp = p.in.z ? (const T *)p.in.z + (size_t)b * p.pr.z_row + d0 : nullptr, *dyp = (const T *)p.dy + (size_t)b * L * D + d0;
    const T *cs = p.in.conv_state ? (const T *)p.in.conv_state + (size_t)b * (W - 1) * D + d0 : nullptr;
    const T *bp = (const T *)p.in.b + (size_t)b * p.pr.b_row + (size_t)g * p.pr.b_group;
    const T *cp = (const T *)p.in.c + (size_t)b * p.pr.c_row + (size_t)g * p.pr.c_group;
    for (int i = tid; i < kPars * CT; i += THREADS) s_par[i / CT][i % CT] = channel_par(p, i / CT, d0 + min(i % CT, nd - 1));
    __syncthreads();
    auto pars = [&](int m, float (&v)[2]) {
        const float2 w = *reinterpret_cast<const float2 *>(&s_par[m][pc]);
        v[0] = w.x;
        v[1] = w.y;
    };
    const size_t out_at = (size_t)b * L * D + de;
    const bool out_pair = two && ((((uintptr_t)p.grads.x | (uintptr_t)p.grads.dt | (uintptr_t)p.grads.z) & (2 * sizeof(T) - 1)) == 0) &&
                          (D & 1) == 0 && (out_at & 1) == 0;

    // recurrence role: channels c0 and c0 + 1 (a pair), states n0 .. n0 + 3
    const int part = lane % LPC, grp = lane / LPC, c0 = (tid / LPC) * 2, n0 = part * 4;
    f32x2 A2[4], q[4];                   // A log2(e); the adjoint that enters a time from its right, a_{t+1} p_{t+1}
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float av[2], qv[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool in = n0 + i < N && c0 + j < nd;
            const size_t at = (size_t)(d0 + c0 + j) * N + n0 + i;
            av[j] = in ? log2_rate(p.in.a[at]) : 0.0f;
            qv[j] = in && p.splits > 1 ? p.split_state[((size_t)b * p.splits + split) * D * N + at] : 0.0f;
        }
        A2[i] = pack2(av[0], av[1]);
        q[i] = pack2(qv[0], qv[1]);
    }
    // sums over this block's times: of a chunk, then of all (keeps the rounding of long sums small)
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float2 *>(s_dA)[i * THREADS + tid] = make_float2(0.0f, 0.0f);
    float sums[7][2] = {};               // dconv (oldest tap first), dconv_bias, dskip, ddt_bias
    for (int i = tid; i < 3 * CT; i += THREADS) (&s_carry[0][0])[i] = 0.0f;

    // where a warp leaves dB and dC of sub-chunk j: over its states before it, which have been used by then
    auto part_of = [&](int j, int w) {
        if (!S::IN_SLOT) return s_part + (j * WARPS + w) * S::PART;
        if (j == kSubs - 1) return s_part + w * S::PART;
        if (j == 0) return S::SHARE ? s_h + w * (S::SLOT / WARPS) + S::PART : s_part + (WARPS + w) * S::PART;
        return s_h + (j - 1) * S::SLOT + w * (S::SLOT / WARPS);
    };
    auto load_states = [&](int t0, f32x2 (&h)[4]) {
        const float *from = p.checkpoints + (((size_t)b * p.n_chunks + t0 / kChunk) * D + d0 + c0) * N + n0;
        float v[2][4];                   // [channel][state]
        const bool vec = N % 4 == 0 && ((uintptr_t)p.checkpoints & 15u) == 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (c0 + j < nd && vec && n0 < N) {
                const float4 w = *reinterpret_cast<const float4 *>(from + (size_t)j * N);
                v[j][0] = w.x; v[j][1] = w.y; v[j][2] = w.z; v[j][3] = w.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] = c0 + j < nd && n0 + i < N ? from[(size_t)j * N + i] : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = pack2(v[0][i], v[1][i]);
    };
    auto fetch = [&](int t0, Raw &r) {
        RowCopy<T, CT, kChunk + 3, THREADS>(xp, p.pr.x_time, nd, tid).run(&r.x[0][0], t0 - 3, len, tid);
        RowCopy<T, CT, kChunk, THREADS>(dtp, p.pr.dt_time, nd, tid).run(&r.dt[0][0], t0, len, tid);
        if (zp) RowCopy<T, CT, kChunk, THREADS>(zp, p.pr.z_time, nd, tid).run(&r.z[0][0], t0, len, tid);
        RowCopy<T, CT, kChunk, THREADS>(dyp, D, nd, tid).run(&r.dy[0][0], t0, len, tid);
        RowCopy<T, NP, kChunk, THREADS>(bp, p.pr.b_time, N, tid).run(&r.b[0][0], t0, len, tid);
        RowCopy<T, NP, kChunk, THREADS>(cp, p.pr.c_time, N, tid).run(&r.c[0][0], t0, len, tid);
        if (t0 < 3 && cs) {                              // x before time 0, over the zeros
            __syncthreads();
            for (int i = tid; i < 3 * CT; i += THREADS) {
                const int k = i / CT, c = i % CT, from = t0 - 3 + k + W - 1;
                if (t0 - 3 + k < 0 && from >= 0 && c < nd) r.x[k][c] = cs[(size_t)from * D + c];
            }
        }
        copy_commit();
    };
    if (N < NP) {                                        // the padded states' B and C stay 0
        for (int i = tid; i < S::BUFS * kChunk * NP; i += THREADS) {
            auto &r = s_raw[i / (kChunk * NP)];
            (&r.b[0][0])[i % (kChunk * NP)] = (&r.c[0][0])[i % (kChunk * NP)] = from_f32<T>(0.0f);
        }
        __syncthreads();
    }

    const int n_chunks = (t_end - t_begin + kChunk - 1) / kChunk;
    if (S::BUFS == 2) fetch(t_begin + (n_chunks - 1) * kChunk, s_raw[(n_chunks - 1) & 1]);
    for (int cidx = n_chunks - 1; cidx >= 0; --cidx) {
        const int t0 = t_begin + cidx * kChunk;
        const int span = min(kChunk, t_end - t0);                    // times of the chunk
        const int live = max(0, min(kChunk, min(len, t_end) - t0));  // that exist in this row
        if (S::BUFS == 1) {
            __syncthreads();
            fetch(t0, s_raw[0]);
        }
        copy_wait<0>();
        __syncthreads();                                             // the inputs are here, the chunk after this one is done
        if (S::BUFS == 2 && cidx > 0) fetch(t0 - kChunk, s_raw[(cidx - 1) & 1]);
        const auto &r = s_raw[S::BUFS == 2 ? cidx & 1 : 0];
        f32x2 h[4];
        if (live > 0) load_states(t0, h);
        // element-wise: u, s, e (0 beyond the row's end: nothing flows there, and the factors are 1)
        {
            float w0[2], w1[2], w2[2], w3[2], cb[2], db[2];
            pars(kW0, w0); pars(kW1, w1); pars(kW2, w2); pars(kW3, w3); pars(kConvBias, cb); pars(kDtBias, db);
            float x0[2], x1[2], x2[2];
            get_pair(&r.x[tg * E][pc], x0);
            get_pair(&r.x[tg * E + 1][pc], x1);
            get_pair(&r.x[tg * E + 2][pc], x2);
#pragma unroll 4
            for (int i = 0; i < E; ++i) {
                const int k = tg * E + i;
                float u[2], s[2], e[2], x3[2], dtv[2], z[2];
                get_pair(&r.x[k + 3][pc], x3);
                get_pair(&r.dt[k][pc], dtv);
                get_pair(&r.dy[k][pc], e);
                if (zp) get_pair(&r.z[k][pc], z);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bool in = k < live && pc + j < nd;
                    u[j] = in ? silu(conv_at(W, w0[j], w1[j], w2[j], w3[j], cb[j], x0[j], x1[j], x2[j], x3[j])) : 0.0f;
                    s[j] = in ? softplus(dtv[j] + db[j]) : 0.0f;
                    if (zp) e[j] *= silu(z[j]);
                    if (!in) e[j] = 0.0f;
                    x0[j] = x1[j];
                    x1[j] = x2[j];
                    x2[j] = x3[j];
                }
                *reinterpret_cast<float2 *>(&s_u[k][pc]) = make_float2(u[0], u[1]);
                *reinterpret_cast<float2 *>(&s_step[k][pc]) = make_float2(s[0], s[1]);
                *reinterpret_cast<float2 *>(&s_e[k][pc]) = make_float2(e[0], e[1]);
            }
        }
        for (int i = tid; i < kChunk * NP / 2; i += THREADS) {
            const int k = i / (NP / 2), n = 2 * (i % (NP / 2));
            float v[2];
            get_pair(&r.b[k][n], v);
            *reinterpret_cast<float2 *>(&s_bc[k][n]) = make_float2(v[0], v[1]);
            get_pair(&r.c[k][n], v);
            *reinterpret_cast<float2 *>(&s_bc[k][NP + n]) = make_float2(v[0], v[1]);
        }
        __syncthreads();

        const int subs = (live + kSub - 1) / kSub;
        // one time forwards: a (its factors) and h from the state before it
        auto forward = [&](int t, const f32x2 (&from)[4], f32x2 (&a)[4], f32x2 (&to)[4]) {
            const float2 s2 = *reinterpret_cast<const float2 *>(&s_step[t][c0]), u2 = *reinterpret_cast<const float2 *>(&s_u[t][c0]);
            const float4 B4 = *reinterpret_cast<const float4 *>(&s_bc[t][n0]);
            const f32x2 s = pack2(s2.x, s2.y), du = mul2(s, pack2(u2.x, u2.y));
            const float Bv[4] = {B4.x, B4.y, B4.z, B4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = decay2(s, A2[i]);
                to[i] = fma2(a[i], from[i], mul2(du, pack2(Bv[i], Bv[i])));
            }
        };
        auto slot = [&](int j) { return reinterpret_cast<float2 *>(s_h + (j - 1) * S::SLOT + warp * (S::SLOT / WARPS)) + lane; };
        // forwards through the chunk, keeping the state before the middle sub-chunks
#pragma unroll 1
        for (int j = 0; j + 1 < subs; ++j) {
            if (j > 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 v;
                    unpack2(h[i], v.x, v.y);
                    slot(j)[i * 32] = v;
                }
            }
#pragma unroll
            for (int k = 0; k < kSub; ++k) {
                f32x2 a[4];
                forward(j * kSub + k, h, a, h);
            }
        }

        f32x2 dA[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) dA[i] = pack2(0.0f, 0.0f);
#pragma unroll 1
        for (int j = subs - 1; j >= 0; --j) {
            f32x2 a[kSub][4], hh[kSub + 1][4];
            if (j == subs - 1) {             // the walk ended here
#pragma unroll
                for (int i = 0; i < 4; ++i) hh[0][i] = h[i];
            } else if (j == 0) {
                load_states(t0, hh[0]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 v = slot(j)[i * 32];
                    hh[0][i] = pack2(v.x, v.y);
                }
            }
            __syncwarp();                    // the slot takes this sub-chunk's dB and dC
#pragma unroll
            for (int k = 0; k < kSub; ++k) forward(j * kSub + k, hh[k], a[k], hh[k + 1]);
            float *s_mine = part_of(j, warp);
#pragma unroll
            for (int k = kSub - 1; k >= 0; --k) {
                const int t = j * kSub + k;
                const float2 s2 = *reinterpret_cast<const float2 *>(&s_step[t][c0]), u2 = *reinterpret_cast<const float2 *>(&s_u[t][c0]);
                const float2 e2 = *reinterpret_cast<const float2 *>(&s_e[t][c0]);
                const float4 B4 = *reinterpret_cast<const float4 *>(&s_bc[t][n0]), C4 = *reinterpret_cast<const float4 *>(&s_bc[t][NP + n0]);
                const f32x2 s = pack2(s2.x, s2.y), e = pack2(e2.x, e2.y), su = mul2(s, pack2(u2.x, u2.y));
                const float Bv[4] = {B4.x, B4.y, B4.z, B4.w}, Cv[4] = {C4.x, C4.y, C4.z, C4.w};
                f32x2 pB, pAh, v;
                float bc[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x2 bb = pack2(Bv[i], Bv[i]), cc = pack2(Cv[i], Cv[i]);
                    const f32x2 pt = fma2(cc, e, q[i]);              // p_t
                    q[i] = mul2(pt, a[k][i]);                        // what the time before gets
                    const f32x2 qh = mul2(q[i], hh[k][i]);           // p a h_{t-1}
                    pB = i ? fma2(pt, bb, pB) : mul2(pt, bb);
                    pAh = i ? fma2(qh, A2[i], pAh) : mul2(qh, A2[i]);
                    v = i ? fma2(cc, hh[k + 1][i], v) : mul2(cc, hh[k + 1][i]);
                    dA[i] = fma2(qh, s, dA[i]);
                    float lo, hi;
                    unpack2(mul2(su, pt), lo, hi);
                    bc[i] = lo + hi;
                    unpack2(mul2(e, hh[k + 1][i]), lo, hi);
                    bc[4 + i] = lo + hi;
                }
                float cs[2][3];
                unpack2(pB, cs[0][0], cs[1][0]);
                unpack2(pAh, cs[0][1], cs[1][1]);
                unpack2(v, cs[0][2], cs[1][2]);
                StateSum<LPC>::run(cs, part);
                GroupSum<LPC>::run(bc, grp);
                // (the shuffles: all lanes of a channel have read this time's values)
                if (part < 2) {
                    const float st = part ? s2.y : s2.x, ut = part ? u2.y : u2.x;
                    s_u[t][c0 + part] = st * cs[0][0];                                       // du but for the skip's share
                    s_step[t][c0 + part] = fmaf(ut, cs[0][0], cs[0][1] * 0.6931471806f);     // ds (A2 is A log2 e)
                    s_e[t][c0 + part] = cs[0][2];                                            // sum_n C h
                }
                if (grp < 8) {
                    const int f = GroupSum<LPC>::first(grp);
#pragma unroll
                    for (int i = 0; i < GroupSum<LPC>::LEFT; ++i) {
                        const int m = f + i;                     // 0..3: dB of state n0 + m, 4..7: dC
                        s_mine[k * 2 * NP + (m < 4 ? 0 : NP) + n0 + (m & 3)] = bc[i];
                    }
                }
            }
            __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 &to = reinterpret_cast<float2 *>(s_dA)[i * THREADS + tid];
            float lo, hi;
            unpack2(dA[i], lo, hi);
            to = make_float2(to.x + lo, to.y + hi);
        }
        __syncthreads();
        // dB and dC of the chunk: the warps' sums in their order
        for (int at = tid; at < span * 2 * NP; at += THREADS) {
            const int k = at / (2 * NP), n = at % (2 * NP), m = n < NP ? n : n - NP, j = k / kSub;
            if (m >= N) continue;
            float s = 0.0f;
            if (k < subs * kSub) {
#pragma unroll
                for (int w = 0; w < WARPS; ++w) s += part_of(j, w)[(k % kSub) * 2 * NP + n];
            }
            p.part_bc[((((size_t)tile_in_group * p.pr.batch + b) * L + t0 + k) * G + g) * 2 * N + (n < NP ? m : N + m)] = s;
        }

        // element-wise: dz, ddt, dc and the parameters' sums
        {
            float w0[2], w1[2], w2[2], w3[2], cb[2], db[2], skip[2];
            pars(kW0, w0); pars(kW1, w1); pars(kW2, w2); pars(kW3, w3); pars(kConvBias, cb); pars(kDtBias, db); pars(kSkip, skip);
            float x0[2], x1[2], x2[2];
            get_pair(&r.x[tg * E][pc], x0);
            get_pair(&r.x[tg * E + 1][pc], x1);
            get_pair(&r.x[tg * E + 2][pc], x2);
            size_t at = out_at + (size_t)(t0 + tg * E) * D;
            float acc[7][2] = {};
#pragma unroll 4
            for (int i = 0; i < E; ++i) {
                const int k = tg * E + i;
                float dc[2] = {}, ddt[2] = {}, dz[2] = {};
                if (k < live && own) {
                    float x3[2], dtv[2], dyv[2], z[2];
                    get_pair(&r.x[k + 3][pc], x3);
                    get_pair(&r.dt[k][pc], dtv);
                    get_pair(&r.dy[k][pc], dyv);
                    if (zp) get_pair(&r.z[k][pc], z);
                    const float2 duv = *reinterpret_cast<const float2 *>(&s_u[k][pc]), dsv = *reinterpret_cast<const float2 *>(&s_step[k][pc]);
                    const float2 vv = *reinterpret_cast<const float2 *>(&s_e[k][pc]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float c = conv_at(W, w0[j], w1[j], w2[j], w3[j], cb[j], x0[j], x1[j], x2[j], x3[j]), sc = sigmoid(c), u = c * sc;
                        float e = dyv[j];
                        if (zp) {
                            const float sz = sigmoid(z[j]);
                            dz[j] = dyv[j] * fmaf(skip[j], u, j ? vv.y : vv.x) * silu_slope(z[j], sz);
                            e = dyv[j] * (z[j] * sz);
                        }
                        ddt[j] = (j ? dsv.y : dsv.x) * sigmoid(dtv[j] + db[j]);
                        dc[j] = fmaf(skip[j], e, j ? duv.y : duv.x) * silu_slope(c, sc);
                        acc[5][j] = fmaf(e, u, acc[5][j]);
                        acc[6][j] += ddt[j];
                        acc[4][j] += dc[j];
                        acc[3][j] = fmaf(dc[j], x3[j], acc[3][j]);
                        acc[2][j] = fmaf(dc[j], x2[j], acc[2][j]);
                        acc[1][j] = fmaf(dc[j], x1[j], acc[1][j]);
                        acc[0][j] = fmaf(dc[j], x0[j], acc[0][j]);
                        x0[j] = x1[j];
                        x1[j] = x2[j];
                        x2[j] = x3[j];
                    }
                }
                if (k < span && own) {
                    if (p.grads.dt) store_pair((T *)p.grads.dt + at, ddt, out_pair, two);
                    if (p.grads.z) store_pair((T *)p.grads.z + at, dz, out_pair, two);
                }
                at += D;
                *reinterpret_cast<float2 *>(&s_u[k][pc]) = make_float2(dc[0], dc[1]);
            }
#pragma unroll
            for (int m = 0; m < 7; ++m) {
                sums[m][0] += acc[m][0];
                sums[m][1] += acc[m][1];
            }
        }
        __syncthreads();
        // dx_t = sum_j w[W-1-j] dc_{t+j}; the chunk's last times reach into the chunk after it
        {
            auto dc_at = [&](int k) {
                return k < kChunk ? *reinterpret_cast<const float2 *>(&s_u[k][pc]) : *reinterpret_cast<const float2 *>(&s_carry[k - kChunk][pc]);
            };
            float w0[2], w1[2], w2[2], w3[2];
            pars(kW0, w0); pars(kW1, w1); pars(kW2, w2); pars(kW3, w3);
            const int first = tg * E;
            float2 c0v = dc_at(first), c1v = dc_at(first + 1), c2v = dc_at(first + 2);
            const bool hands_over = split + 1 < p.splits && cidx == n_chunks - 1;   // the next part's dc is added later
#pragma unroll 4
            for (int i = 0; i < E; ++i) {
                const int k = first + i;
                const float2 c3v = dc_at(k + 3);
                float dx[2];
                dx[0] = fmaf(w0[0], c3v.x, fmaf(w1[0], c2v.x, fmaf(w2[0], c1v.x, w3[0] * c0v.x)));
                dx[1] = fmaf(w0[1], c3v.y, fmaf(w1[1], c2v.y, fmaf(w2[1], c1v.y, w3[1] * c0v.y)));
                if (k < span && own) {
                    if (hands_over && k >= kChunk - (W - 1)) {
                        float *to = p.conv_tail + (((size_t)b * p.splits + split) * (W - 1) + k - (kChunk - (W - 1))) * D + de;
                        to[0] = dx[0];
                        if (two) to[1] = dx[1];
                    } else if (p.grads.x) {
                        if (k >= live) dx[0] = dx[1] = 0.0f;
                        store_pair((T *)p.grads.x + out_at + (size_t)(t0 + k) * D, dx, out_pair, two);
                    }
                }
                c0v = c1v;
                c1v = c2v;
                c2v = c3v;
            }
        }
        __syncthreads();
        for (int i = tid; i < 3 * CT; i += THREADS) (&s_carry[0][0])[i] = (&s_u[0][0])[i];
    }
    __syncthreads();
    // what the part before needs of this part's first dc
    if (p.splits > 1) {
        for (int i = tid; i < (W - 1) * CT; i += THREADS) {
            const int k = i / CT, c = i % CT;
            if (c < nd) p.conv_head[(((size_t)b * p.splits + split) * (W - 1) + k) * D + d0 + c] = s_carry[k][c];
        }
    }

    // parameters' partial sums: dA by its lanes, the others over the groups of times through shared memory
    float *pa = p.part_par + ((size_t)b * p.splits + split) * D * (N + kParExtra);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = reinterpret_cast<const float2 *>(s_dA)[i * THREADS + tid];
        if (n0 + i < N && c0 < nd) pa[(size_t)(d0 + c0) * N + n0 + i] = v.x;
        if (n0 + i < N && c0 + 1 < nd) pa[(size_t)(d0 + c0 + 1) * N + n0 + i] = v.y;
    }
    float *s_sum = smem;                 // [TG][7][CT]
#pragma unroll
    for (int m = 0; m < 7; ++m) *reinterpret_cast<float2 *>(s_sum + (tg * 7 + m) * CT + pc) = make_float2(sums[m][0], sums[m][1]);
    __syncthreads();
    for (int i = tid; i < 7 * CT; i += THREADS) {
        const int m = i / CT, c = i % CT;
        if (c >= nd) continue;
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < S::TG; ++k) s += s_sum[(k * 7 + m) * CT + c];
        pa[(size_t)D * N + (size_t)m * D + d0 + c] = s;
    }
}

// dx of the last W-1 times of every part but the last: the next part's dc were not known there.
template <typename T> __global__ void ssm_conv_join_kernel(const SsmParams p)
{
    const int D = p.pr.channels, W = p.pr.conv_width;
    const int d = blockIdx.y * blockDim.x + threadIdx.x, b = blockIdx.x, split = blockIdx.z;
    if (d >= D) return;
    const int len = row_length(p, b), t_last = (split + 1) * p.split_len;
    const float *w = p.in.conv_weight + (size_t)d * W;
    for (int k = 0; k < W - 1; ++k) {
        const int t = t_last - (W - 1) + k;
        float dx = p.conv_tail[(((size_t)b * p.splits + split) * (W - 1) + k) * D + d];
        // dc_{t+j} with t + j >= t_last: head index t + j - t_last = k + j - (W - 1)
        for (int j = W - 1 - k; j < W; ++j)
            dx = fmaf(w[W - 1 - j], p.conv_head[(((size_t)b * p.splits + split + 1) * (W - 1) + k + j - (W - 1)) * D + d], dx);
        ((T *)p.grads.x)[((size_t)b * p.pr.length + t) * D + d] = from_f32<T>(t < len ? dx : 0.0f);
    }
}

// dB and dC: the channel tiles' partial sums, in the order of the tiles.
template <typename T> __global__ void ssm_bc_sum_kernel(const SsmParams p)
{
    const int N = p.pr.state;
    const size_t per = (size_t)p.pr.batch * p.pr.length * p.pr.groups * 2 * N;
    const size_t at = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (at >= per) return;
    float s = 0.0f;
    for (int k = 0; k < p.tiles_per_group; ++k) s += p.part_bc[k * per + at];
    const size_t row = at / (2 * N);
    const int n = (int)(at - row * 2 * N);
    if (n < N) {
        if (p.grads.b) ((T *)p.grads.b)[row * N + n] = from_f32<T>(s);
    } else if (p.grads.c) {
        ((T *)p.grads.c)[row * N + n - N] = from_f32<T>(s);
    }
}

// Parameters' gradients: the partial sums of rows and parts.  A block takes 32 values, its warps
// every 8th slot each, and adds the warps' sums.
__global__ __launch_bounds__(256) void ssm_par_sum_kernel(const SsmParams p)
{
    __shared__ float s_sum[8][32];
    const int D = p.pr.channels, N = p.pr.state, W = p.pr.conv_width;
    const int stride = D * (N + kParExtra), total = D * (N + 7), slots = p.pr.batch * p.splits;
    const int at = blockIdx.x * 32 + threadIdx.x % 32, w = threadIdx.x / 32;
    float s = 0.0f;
    if (at < total)
        for (int k = w; k < slots; k += 8) s += p.part_par[(size_t)k * stride + at];
    s_sum[w][threadIdx.x % 32] = s;
    __syncthreads();
    if (w > 0 || at >= total) return;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += s_sum[k][threadIdx.x];
    if (at < D * N) {
        if (p.grads.a) p.grads.a[at] = s;
        return;
    }
    const int m = (at - D * N) / D, d = (at - D * N) % D;
    if (m < 4) {
        // the four taps are aligned at the newest
        const int k = m - (4 - W);
        if (k >= 0 && p.grads.conv_weight) p.grads.conv_weight[(size_t)d * W + k] = s;
    } else {
        float *to = m == 4 ? p.grads.conv_bias : m == 5 ? p.grads.skip : p.grads.dt_bias;
        if (to) to[d] = s;
    }
}

template <typename T, int NPT, int LPC> cudaError_t launch_local(SsmParams p, cudaStream_t st)
{
    using S = LocalShape<T, NPT, LPC>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = allow_max_smem((const void *)ssm_adjoint_local_kernel<T, NPT, LPC>, done);
    if (e != cudaSuccess) return e;
    p.tiles_per_group = (p.pr.channels / p.pr.groups + S::CT - 1) / S::CT;
    ssm_adjoint_local_kernel<T, NPT, LPC><<<dim3(p.pr.batch, p.tiles_per_group * p.pr.groups, p.splits - 1), S::THREADS, sizeof(typename S::Tile), st>>>(p);
    return cudaGetLastError();
}

template <typename T, int LPC> cudaError_t launch(const SsmParams &p, cudaStream_t st)
{
    using S = Shape<T, LPC>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = allow_max_smem((const void *)ssm_backward_kernel<T, LPC>, done);
    if (e != cudaSuccess) return e;
    if (p.splits > 1) {
        e = LPC == 2 ? launch_local<T, 8, 1>(p, st) : launch_local<T, 16, (LPC < 4 ? 1 : LPC / 4)>(p, st);
        if (e != cudaSuccess) return e;
        const int DN = p.pr.channels * p.pr.state;
        ssm_adjoint_join_kernel<<<dim3(p.pr.batch, (DN + 127) / 128), 128, 0, st>>>(p);
    }
    ssm_backward_kernel<T, LPC><<<dim3(p.pr.batch, p.tiles_per_group * p.pr.groups, p.splits), S::THREADS, S::BYTES, st>>>(p);
    if (p.splits > 1 && p.grads.x)
        ssm_conv_join_kernel<T><<<dim3(p.pr.batch, (p.pr.channels + 127) / 128, p.splits - 1), 128, 0, st>>>(p);
    if (p.grads.b || p.grads.c) {
        const size_t per = (size_t)p.pr.batch * p.pr.length * p.pr.groups * 2 * p.pr.state;
        ssm_bc_sum_kernel<T><<<(unsigned)((per + 255) / 256), 256, 0, st>>>(p);
    }
    ssm_par_sum_kernel<<<(p.pr.channels * (p.pr.state + 7) + 31) / 32, 256, 0, st>>>(p);
    return cudaGetLastError();
}

template <typename T> cudaError_t launch_shape(const SsmParams &p, cudaStream_t st)
{
    if (p.pr.state <= 8) return launch<T, 2>(p, st);
    if (p.pr.state <= 16) return launch<T, 4>(p, st);
    return p.pr.state <= 32 ? launch<T, 8>(p, st) : launch<T, 16>(p, st);
}

}  // namespace

void ssm_backward_plan(const themis_ssm_problem_t *pr, SsmParams *p)
{
    // (the two are the same for every type: two 16-bit input buffers are as large as one of 32 bits)
    const int ct = pr->state <= 8 ? Shape<float, 2>::CT : pr->state <= 16 ? Shape<float, 4>::CT : pr->state <= 32 ? Shape<float, 8>::CT : Shape<float, 16>::CT;
    const int resident = pr->state <= 8    ? Shape<float, 2>::RESIDENT
                         : pr->state <= 16 ? Shape<float, 4>::RESIDENT
                         : pr->state <= 32 ? Shape<float, 8>::RESIDENT
                                           : Shape<float, 16>::RESIDENT;
    p->tiles_per_group = (pr->channels / pr->groups + ct - 1) / ct;
    p->n_chunks = (pr->length + kChunk - 1) / kChunk;
    const long long blocks = (long long)p->tiles_per_group * pr->groups * pr->batch;
    // Time of a part's chunk with k blocks on a multiprocessor, measured on 16 and 64 x 2048 and 1024
    // x 1024 with 16 states in bf16 and used for every shape (one block 14 us, two 23 us); split parts repeat the
    // steps and gates in the first pass (0.17 with the joins).  Many short parts even out the last wave: in the
    // form of the kernel that these were measured with, 16 x 2048 x 1024 took 2140 us whole, 1990 in 2 parts and 1740
    // in 16 (the present one: 1270 in 16), but rows that fill the GPU twice were fastest whole.
    auto chunk_time = [&](long long n) {
        const long long places = (long long)resident * kSMs;
        return n <= places ? 4.7 + 9.2 * ((n + kSMs - 1) / kSMs) : ((double)n / places + 0.35) * (4.7 + 9.2 * resident);
    };
    double least = 0.0;
    const int most = (int)std::min<long long>(p->n_chunks, 8LL * resident * kSMs / blocks + 1);
    for (int s = 1; s <= most; s += s < 16 ? 1 : s / 8) {
        const int chunks = (p->n_chunks + s - 1) / s, splits = (p->n_chunks + chunks - 1) / chunks;
        const double t = chunk_time(blocks * splits) * chunks * (splits > 1 ? 1.17 : 1.0) + (splits > 1 ? 8.0 + 0.2 * splits : 0.0);
        if (least == 0.0 || t < least) {
            least = t;
            p->splits = splits;
            p->split_len = chunks * kChunk;
        }
    }
}

cudaError_t launch_ssm_backward(const SsmParams &p, cudaStream_t st)
{
    switch (p.pr.dtype) {
        case THEMIS_DTYPE_F32: return launch_shape<float>(p, st);
        case THEMIS_DTYPE_BF16: return launch_shape<__nv_bfloat16>(p, st);
        default: return launch_shape<__half>(p, st);
    }
}

}  // namespace themis
