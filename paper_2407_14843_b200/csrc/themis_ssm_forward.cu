// Selective state space scan over whole histories, forward.
//
// A block takes a tile of channels of one row and walks its times in tiles.  Per tile: the
// convolution and the step, element by element (channels across a warp); then the recurrence, NPT
// states of a channel in the registers of a lane and LPC lanes to a channel, B and C of the tile
// broadcast from shared memory; then gate and output.  The tiles arrive by asynchronous copies, the
// next one while this one is worked on.
//
// The time axis is a chain, so rows x channels alone give the parallelism.  Where they are too
// few to fill the GPU, the axis is cut into parts: a first pass runs every part from a zero state
// (h is linear in the state before the part: h_end = exp(A sum s) h_start + h_local), a small
// kernel joins the parts, and the main pass runs every part from its true start.  That costs the
// recurrence twice, so no more parts are made than are needed.
#include <algorithm>

#include "themis_ssm.cuh"

namespace themis {
namespace {

constexpr int kThreads = 128;
constexpr int kGroup = 4;                    // times of the recurrence that are worked on at once

template <typename T, int NPT, int LPC> struct Shape {
    static constexpr int CT = kThreads / LPC;            // channels of a block
    static constexpr int TT = LPC == 1 ? 16 : 32;        // times of a tile
    static constexpr int PAIRS = CT / 2;                 // element-wise parts: a thread has two channels ...
    static constexpr int E = TT * PAIRS / kThreads;      // ... of this many consecutive times
    static constexpr int NP = NPT * LPC;                 // states, padded (A = B = C = 0 beyond N)
};

// Shared memory of a block.  x, dt, B and C of the next tile arrive while this one is worked on.  Every array
// starts on the 16 bytes of an asynchronous copy, in both buffers (four 16-bit values of an unused C would
// put the second buffer 8 bytes off).
template <typename T, int NPT, int LPC, bool LOCAL> struct Tile {
    using S = Shape<T, NPT, LPC>;
    struct Raw {
        alignas(16) T x[S::TT + 3][S::CT];               // the three times before the tile first
        alignas(16) T dt[S::TT][S::CT];
        alignas(16) T b[S::TT][S::NP];
        alignas(16) T c[LOCAL ? 1 : S::TT][S::NP];
    } raw[2];
    alignas(16) T z[LOCAL ? 1 : S::TT][S::CT];
    alignas(16) float2 su[S::TT][S::CT];                 // s_t and u_t, then v_t
    alignas(16) float bc[S::TT][2 * S::NP];
};

// blocks of a multiprocessor (registers)
template <typename T> constexpr int kPlaces = sizeof(T) == 4 ? 3 : 4;

// LOCAL: first pass over split parts (no y): the part's state from zero and the sum of its steps.
// SAVE: checkpoints for the backward pass.
template <typename T, int NPT, int LPC, bool LOCAL, bool SAVE>
__global__ __launch_bounds__(kThreads, kPlaces<T>) void ssm_scan_kernel(const SsmParams p)
{
    using S = Shape<T, NPT, LPC>;
    constexpr int CT = S::CT, E = S::E, TT = S::TT, NP = S::NP;
    extern __shared__ __align__(16) uint8_t smem[];
    using Buffers = Tile<T, NPT, LPC, LOCAL>;
    using Raw = typename Buffers::Raw;
    static_assert(sizeof(Raw) % 16 == 0 && offsetof(Raw, x) % 16 == 0 && offsetof(Raw, dt) % 16 == 0 && offsetof(Raw, b) % 16 == 0 &&
                      offsetof(Raw, c) % 16 == 0 && offsetof(Buffers, raw) % 16 == 0 && offsetof(Buffers, z) % 16 == 0 &&
                      offsetof(Buffers, su) % 16 == 0 && offsetof(Buffers, bc) % 16 == 0,
                  "rows are copied and read 16 bytes at a time");
    auto &s = *reinterpret_cast<Buffers *>(smem);

    const int D = p.pr.channels, N = p.pr.state, W = p.pr.conv_width, L = p.pr.length;
    const int b = blockIdx.x, split = blockIdx.z, tid = threadIdx.x;
    int g, d0, nd;
    tile_of_block(p, blockIdx.y, CT, g, d0, nd);
    const int t_begin = split * p.split_len, t_end = min(L, t_begin + p.split_len);
    const int t_live = min(row_length(p, b), t_end);     // times from here on do not exist

    const T *xp = (const T *)p.in.x + (size_t)b * p.pr.x_row + d0;
    const T *dtp = (const T *)p.in.dt + (size_t)b * p.pr.dt_row + d0;
    const T *zp = !LOCAL && p.in.z ? (const T *)p.in.z + (size_t)b * p.pr.z_row + d0 : nullptr;
    const T *cs = p.in.conv_state ? (const T *)p.in.conv_state + (size_t)b * (W - 1) * D + d0 : nullptr;
    const T *bp = (const T *)p.in.b + (size_t)b * p.pr.b_row + (size_t)g * p.pr.b_group;
    const T *cp = (const T *)p.in.c + (size_t)b * p.pr.c_row + (size_t)g * p.pr.c_group;

    // element-wise role: two channels, E consecutive times
    const int pc = 2 * (tid % S::PAIRS), tg = tid / S::PAIRS;
    float w0[2], w1[2], w2[2], w3[2], conv_bias[2], dt_bias[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int d = d0 + min(pc + j, nd - 1);
        const float *w = p.in.conv_weight + (size_t)d * W;
        w3[j] = w[W - 1];
        w2[j] = w[W - 2];
        w1[j] = W > 2 ? w[W - 3] : 0.0f;
        w0[j] = W > 3 ? w[0] : 0.0f;
        conv_bias[j] = p.in.conv_bias ? p.in.conv_bias[d] : 0.0f;
        dt_bias[j] = p.in.dt_bias ? p.in.dt_bias[d] : 0.0f;
    }

    // recurrence role: one channel, NPT of its states
    const int rc = tid / LPC, part = tid % LPC;
    const int dr = d0 + min(rc, nd - 1), n0 = part * NPT;
    const float skip = !LOCAL && p.in.skip ? p.in.skip[dr] : 0.0f;
    f32x2 a2[NPT / 2], h[NPT / 2];
    {
        const float *hs = LOCAL ? nullptr
                        : p.splits > 1 ? p.split_state + (((size_t)b * p.splits + split) * D + dr) * N + n0
                        : p.in.ssm_state ? p.in.ssm_state + ((size_t)b * D + dr) * N + n0 : nullptr;
#pragma unroll
        for (int i = 0; i < NPT / 2; ++i) {
            float a[2], was[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int n = 2 * i + j;
                const bool in = n0 + n < N;
                a[j] = in ? log2_rate(p.in.a[(size_t)dr * N + n0 + n]) : 0.0f;
                was[j] = in && hs ? hs[n] : 0.0f;
            }
            a2[i] = pack2(a[0], a[1]);
            h[i] = pack2(was[0], was[1]);
        }
    }
    float step_sum = 0.0f;
    auto put_states = [&](float *to) {
        if (N % 4 == 0 && ((uintptr_t)to & 15u) == 0) {
#pragma unroll
            for (int i = 0; i < NPT / 4; ++i)
                if (n0 + 4 * i < N) {
                    float4 v;
                    unpack2(h[2 * i], v.x, v.y);
                    unpack2(h[2 * i + 1], v.z, v.w);
                    reinterpret_cast<float4 *>(to)[i] = v;
                }
        } else {
#pragma unroll
            for (int i = 0; i < NPT / 2; ++i) {
                float lo, hi;
                unpack2(h[i], lo, hi);
                if (n0 + 2 * i < N) to[2 * i] = lo;
                if (n0 + 2 * i + 1 < N) to[2 * i + 1] = hi;
            }
        }
    };

    // times t0 .. of a sequence into shared memory, zeros where there are none
    const RowCopy<T, CT, TT + 3, kThreads> copy_x(xp, p.pr.x_time, nd, tid);
    const RowCopy<T, CT, TT, kThreads> copy_dt(dtp, p.pr.dt_time, nd, tid), copy_z(zp, p.pr.z_time, nd, tid);
    const RowCopy<T, NP, TT, kThreads> copy_b(bp, p.pr.b_time, N, tid), copy_c(cp, p.pr.c_time, N, tid);
    auto fetch = [&](int t0) {
        auto &r = s.raw[(t0 - t_begin) / TT & 1];
        copy_x.run(&r.x[0][0], t0 - 3, t_live, tid);
        copy_dt.run(&r.dt[0][0], t0, t_live, tid);
        copy_b.run(&r.b[0][0], t0, t_live, tid);
        if (!LOCAL) copy_c.run(&r.c[0][0], t0, t_live, tid);
        if (t0 < 3 && cs) {                              // x before time 0, over the zeros
            __syncthreads();
            for (int i = tid; i < 3 * CT; i += kThreads) {
                const int k = i / CT, ch = i % CT, from = t0 - 3 + k + W - 1;
                if (t0 - 3 + k < 0 && from >= 0 && ch < nd) r.x[k][ch] = cs[(size_t)from * D + ch];
            }
        }
        copy_commit();
    };

    if (N < NP) {                                        // the padded states' B and C stay 0
        for (int i = tid; i < 2 * TT * NP; i += kThreads) {
            auto &r = s.raw[i / (TT * NP)];
            (&r.b[0][0])[i % (TT * NP)] = from_f32<T>(0.0f);
            if (!LOCAL) (&r.c[0][0])[i % (TT * NP)] = from_f32<T>(0.0f);
        }
        __syncthreads();
    }
    fetch(t_begin);
    for (int t0 = t_begin; t0 < t_end; t0 += TT) {
        const int live = max(0, min(TT, t_live - t0));   // times of this tile that exist
        copy_wait<0>();
        __syncthreads();                                 // the tile is here; z and the other buffer are free
        if (!LOCAL) {
            if (zp) copy_z.run(&s.z[0][0], t0, t_live, tid);
            copy_commit();
        }
        if (t0 + TT < t_end) fetch(t0 + TT);
        else copy_commit();
        const auto &r = s.raw[(t0 - t_begin) / TT & 1];

        // element-wise: convolution, step
        {
            float x0[2], x1[2], x2[2];
            get_pair(&r.x[tg * E][pc], x0);
            get_pair(&r.x[tg * E + 1][pc], x1);
            get_pair(&r.x[tg * E + 2][pc], x2);
#pragma unroll 4
            for (int i = 0; i < E; ++i) {
                const int t = tg * E + i;
                float x3[2], dv[2], u[2], st[2];
                get_pair(&r.x[t + 3][pc], x3);
                get_pair(&r.dt[t][pc], dv);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float c = fmaf(w3[j], x3[j], conv_bias[j]);
                    c = fmaf(w2[j], x2[j], c);
                    if (W > 2) c = fmaf(w1[j], x1[j], c);
                    if (W > 3) c = fmaf(w0[j], x0[j], c);
                    // a time that does not exist changes nothing: its factors are 1
                    u[j] = t < live ? silu(c) : 0.0f;
                    st[j] = t < live ? softplus(dv[j] + dt_bias[j]) : 0.0f;
                    x0[j] = x1[j];
                    x1[j] = x2[j];
                    x2[j] = x3[j];
                }
                *reinterpret_cast<float4 *>(&s.su[t][pc]) = make_float4(st[0], u[0], st[1], u[1]);
            }
        }
        for (int i = tid; i < TT * NP / 2; i += kThreads) {
            const int t = i / (NP / 2), n = 2 * (i % (NP / 2));
            float v[2];
            get_pair(&r.b[t][n], v);
            *reinterpret_cast<float2 *>(&s.bc[t][n]) = make_float2(v[0], v[1]);
            if (!LOCAL) {
                get_pair(&r.c[t][n], v);
                *reinterpret_cast<float2 *>(&s.bc[t][NP + n]) = make_float2(v[0], v[1]);
            }
        }
        __syncthreads();

        // recurrence, kGroup times at once: nothing is stored between their loads, so that these and the
        // factors of later times need not wait for the chain through h
#pragma unroll 1
        for (int tb = 0; tb < (SAVE ? min(TT, t_end - t0) : live); tb += kGroup) {
            // state before this time, for the backward pass
            if (SAVE && (t0 + tb) % THEMIS_SSM_CHUNK == 0 && rc < nd)
                put_states(p.out.checkpoints + (((size_t)b * p.n_chunks + (t0 + tb) / THEMIS_SSM_CHUNK) * D + dr) * N + n0);
            if (SAVE && tb >= live) continue;
            float v[kGroup];
#pragma unroll
            for (int k = 0; k < kGroup; ++k) {
                const int t = tb + k;
                const float2 su = s.su[t][rc];
                const float st = su.x, u = su.y, du = st * u;
                const f32x2 ss = pack2(st, st), dd = pack2(du, du);
                const float4 *B = reinterpret_cast<const float4 *>(&s.bc[t][n0]);
                const float4 *C = reinterpret_cast<const float4 *>(&s.bc[t][NP + n0]);
                if (LOCAL) step_sum += st;
                f32x2 acc[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
#pragma unroll
                for (int i = 0; i < NPT / 4; ++i) {
                    const float4 bb = B[i];
                    float4 cc;
                    if (!LOCAL) cc = C[i];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        h[2 * i + j] = fma2(decay2(ss, a2[2 * i + j]), h[2 * i + j], mul2(dd, j ? pack2(bb.z, bb.w) : pack2(bb.x, bb.y)));
                        if (!LOCAL) acc[j] = fma2(h[2 * i + j], j ? pack2(cc.z, cc.w) : pack2(cc.x, cc.y), acc[j]);
                    }
                }
                if (!LOCAL) {
                    float lo, hi;
                    unpack2(add2(acc[0], acc[1]), lo, hi);
                    v[k] = lo + hi;
#pragma unroll
                    for (int o = LPC / 2; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
                    v[k] = fmaf(skip, u, v[k]);
                }
            }
            if (!LOCAL && part == 0) {
#pragma unroll
                for (int k = 0; k < kGroup; ++k) s.su[tb + k][rc].x = v[k];
            }
        }
        if (!LOCAL) copy_wait<1>();                      // z; the next tile may still be on its way
        __syncthreads();

        if (!LOCAL && pc < nd) {
            const bool two = pc + 1 < nd;
            T *yp = (T *)p.out.y + ((size_t)b * L + t0 + tg * E) * D + d0 + pc;
            const bool y_pair = pairs_ok(yp, D, two);
#pragma unroll 4
            for (int i = 0; i < E; ++i) {
                const int t = tg * E + i;
                if (t0 + t < t_end) {
                    float y[2] = {0.0f, 0.0f};
                    if (t < live) {
                        const float4 v = *reinterpret_cast<const float4 *>(&s.su[t][pc]);
                        y[0] = v.x;
                        y[1] = v.z;
                        if (zp) {
                            float z[2];
                            get_pair(&s.z[t][pc], z);
                            y[0] *= silu(z[0]);
                            y[1] *= silu(z[1]);
                        }
                    }
                    store_pair(yp, y, y_pair, two);
                }
                yp += D;
            }
        }
    }

    if (rc < nd) {
        if (LOCAL) {
            put_states(p.split_state + (((size_t)b * p.splits + split) * D + dr) * N + n0);
            if (part == 0) p.split_step[((size_t)b * p.splits + split) * D + dr] = step_sum;
        } else if (p.out.ssm_state && split == p.splits - 1) {
            put_states(p.out.ssm_state + ((size_t)b * D + dr) * N + n0);
        }
    }
    if (!LOCAL && p.out.conv_state && split == p.splits - 1) {
        T *to = (T *)p.out.conv_state + (size_t)b * (W - 1) * D + d0;
        for (int i = tid; i < (W - 1) * CT; i += kThreads) {
            const int k = i / CT, ch = i % CT, t = t_live - (W - 1) + k;
            if (ch >= nd) continue;
            T v = from_f32<T>(0.0f);
            if (t >= 0) v = xp[(size_t)t * p.pr.x_time + ch];
            else if (cs) v = cs[(size_t)(t + W - 1) * D + ch];
            to[(size_t)k * D + ch] = v;
        }
    }
}

// Joins the parts: split_state holds every part's state from zero and gets the state before it.
__global__ void ssm_join_kernel(const SsmParams p)
{
    const int DN = p.pr.channels * p.pr.state, N = p.pr.state, D = p.pr.channels;
    const int e = blockIdx.y * blockDim.x + threadIdx.x, b = blockIdx.x;
    if (e >= DN) return;
    const int d = e / N;
    const float a = log2_rate(p.in.a[e]);
    float h = p.in.ssm_state ? p.in.ssm_state[(size_t)b * DN + e] : 0.0f;
    float *st = p.split_state + (size_t)b * p.splits * DN + e;
    const float *sum = p.split_step + (size_t)b * p.splits * D + d;
    constexpr int U = 8;                // loads of eight parts in flight
    for (int s0 = 0; s0 < p.splits; s0 += U) {
        float end[U], step[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool in = s0 + i < p.splits - 1;
            end[i] = in ? st[(size_t)(s0 + i) * DN] : 0.0f;
            step[i] = in ? sum[(size_t)(s0 + i) * D] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (s0 + i >= p.splits) break;
            st[(size_t)(s0 + i) * DN] = h;
            h = fmaf(exp2f(a * step[i]), h, end[i]);
        }
    }
}

template <typename T, int NPT, int LPC> cudaError_t launch(const SsmParams &p, cudaStream_t st)
{
    constexpr size_t main_smem = sizeof(Tile<T, NPT, LPC, false>), local_smem = sizeof(Tile<T, NPT, LPC, true>);
    static std::atomic<uint64_t> main_done{0}, save_done{0}, local_done{0};
    cudaError_t e = allow_max_smem((const void *)ssm_scan_kernel<T, NPT, LPC, false, false>, main_done);
    if (e == cudaSuccess) e = allow_max_smem((const void *)ssm_scan_kernel<T, NPT, LPC, false, true>, save_done);
    if (e == cudaSuccess) e = allow_max_smem((const void *)ssm_scan_kernel<T, NPT, LPC, true, false>, local_done);
    if (e != cudaSuccess) return e;
    const dim3 grid(p.pr.batch, p.tiles_per_group * p.pr.groups, p.splits);
    if (p.splits > 1) {
        ssm_scan_kernel<T, NPT, LPC, true, false><<<dim3(grid.x, grid.y, p.splits - 1), kThreads, local_smem, st>>>(p);
        const int DN = p.pr.channels * p.pr.state;
        ssm_join_kernel<<<dim3(p.pr.batch, (DN + 127) / 128), 128, 0, st>>>(p);
    }
    if (p.out.checkpoints) ssm_scan_kernel<T, NPT, LPC, false, true><<<grid, kThreads, main_smem, st>>>(p);
    else ssm_scan_kernel<T, NPT, LPC, false, false><<<grid, kThreads, main_smem, st>>>(p);
    return cudaGetLastError();
}

template <typename T> cudaError_t launch_shape(const SsmParams &p, cudaStream_t st)
{
    switch (p.shape.npt * 8 + p.shape.lpc) {
        case 4 * 8 + 1: return launch<T, 4, 1>(p, st);
        case 8 * 8 + 1: return launch<T, 8, 1>(p, st);
        case 16 * 8 + 1: return launch<T, 16, 1>(p, st);
        case 4 * 8 + 2: return launch<T, 4, 2>(p, st);
        case 8 * 8 + 2: return launch<T, 8, 2>(p, st);
        case 4 * 8 + 4: return launch<T, 4, 4>(p, st);
        case 16 * 8 + 2: return launch<T, 16, 2>(p, st);
        case 8 * 8 + 4: return launch<T, 8, 4>(p, st);
        default: return launch<T, 16, 4>(p, st);
    }
}

}  // namespace

// Microseconds for one time of `blocks` blocks with npt states to a lane, `resident` of them on a
// multiprocessor at once.  Measured at 1, 2 and 4 blocks to a multiprocessor (channels x rows of 16 to
// 256 x 1024, bf16, 16 states): 0.28, 0.34, 0.52 us with 16 states to a lane, 0.19 and 0.28 us (2, 4) with
// 8, 0.12 and 0.17 us with 4.  So more lanes to a channel pay while blocks are few, at saturation one
// lane to a channel is fastest (16384 rows x 16 lanes: 904 us against 953 and 1171); the first pass over
// split parts adds 0.7 of the main pass.
static double scan_time(int npt, long long blocks, int resident)
{
    const double base = npt == 16 ? 0.22 : npt == 8 ? 0.12 : 0.075, each = npt == 16 ? 0.075 : npt == 8 ? 0.042 : 0.024;
    const long long places = (long long)resident * kSMs, rest = blocks % places;
    return blocks / places * (base + each * resident) + (rest ? base + each * ((rest + kSMs - 1) / kSMs) : 0.0);
}

void ssm_forward_plan(const themis_ssm_problem_t *pr, SsmParams *p)
{
    int np = 4;
    while (np < pr->state) np *= 2;
    p->n_chunks = (pr->length + THEMIS_SSM_CHUNK - 1) / THEMIS_SSM_CHUNK;
    const int per = pr->channels / pr->groups;
    const int resident = pr->dtype == THEMIS_DTYPE_F32 ? kPlaces<float> : kPlaces<__nv_bfloat16>;
    double least = 0.0;
    for (int lpc = np > 16 ? np / 16 : 1; lpc <= 4 && np / lpc >= 4; lpc *= 2) {
        const int npt = np / lpc, ct = kThreads / lpc, tiles = (per + ct - 1) / ct;
        const long long blocks = (long long)tiles * pr->groups * pr->batch;
        // More parts than fill the GPU twice only repeat the first pass in smaller pieces.
        const int most = (int)std::min<long long>(p->n_chunks, 2LL * resident * kSMs / blocks + 1);
        for (int s = 1; s <= most; s += s < 16 ? 1 : s / 8) {
            const int chunks = (p->n_chunks + s - 1) / s, splits = (p->n_chunks + chunks - 1) / chunks;
            const double t = scan_time(npt, blocks * splits, resident) * chunks * THEMIS_SSM_CHUNK * (splits > 1 ? 1.7 : 1.0) +
                             (splits > 1 ? 6.0 + 0.12 * splits : 0.0);
            if (least == 0.0 || t < least) {
                least = t;
                p->shape = SsmShape{npt, lpc};
                p->tiles_per_group = tiles;
                p->splits = splits;
                p->split_len = chunks * THEMIS_SSM_CHUNK;
            }
        }
    }
}

cudaError_t launch_ssm_forward(const SsmParams &p, cudaStream_t st)
{
    switch (p.pr.dtype) {
        case THEMIS_DTYPE_F32: return launch_shape<float>(p, st);
        case THEMIS_DTYPE_BF16: return launch_shape<__nv_bfloat16>(p, st);
        default: return launch_shape<__half>(p, st);
    }
}

}  // namespace themis
