// One time of the selective scan for every row (a tick of all pipelines).
//
// The state is what moves: 4 N bytes read and 4 N written per row and channel (N = 16: 128 of
// about 150 bytes), against N exponentials and 3 N multiply-adds, so the kernel is bound by
// memory.  Four states per lane (one 16-byte access each way where the rows allow it), the lanes
// of a channel next to each other in a warp: a warp's accesses to the state are one contiguous
// run.  With many rows a thread takes several, so that the parameters are read once for them and
// several rows' states are on their way at the same time; the values per channel and row (convolution,
// step, gate) are then computed by one of the channel's lanes each and handed round by shuffles.
// 16384 rows x 512 channels x 16 states: 227 us, 0.84 of the copy bandwidth (1.24 GB).
#include <algorithm>

#include "themis_ssm.cuh"

namespace themis {
namespace {

constexpr int kStepThreads = 256;

// four neighbouring values with one access, zeros if !in
template <typename T> __device__ __forceinline__ void raw4(const T *p, bool in, Pair<T> (&q)[2])
{
    q[0] = q[1] = zero_pair<T>();
    if (in) {
        if (sizeof(T) == 4) *reinterpret_cast<uint4 *>(q) = *reinterpret_cast<const uint4 *>(p);
        else *reinterpret_cast<uint2 *>(q) = *reinterpret_cast<const uint2 *>(p);
    }
}
template <typename T> __device__ __forceinline__ void unpack4(const Pair<T> (&q)[2], float (&v)[4])
{
    float a[2], b[2];
    Unpack<T>::run(q[0], a);
    Unpack<T>::run(q[1], b);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}
// four neighbouring values of a row as 32-bit floats, the first n of them
template <typename T, bool VEC> __device__ __forceinline__ void load4(const T *p, int n, float (&v)[4])
{
    if (VEC) {
        Pair<T> q[2];
        raw4(p, n > 0, q);
        unpack4<T>(q, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? to_f32(p[i]) : 0.0f;
    }
}

// FULL: every lane of the block has a channel, four states and all rows.
template <typename T, int LPC, int ROWS, bool VEC, bool FULL>
__device__ __forceinline__ void step_rows(const SsmParams &p, int l, int64_t b0)
{
    constexpr int OWN = ROWS > LPC ? ROWS / LPC : 1;        // rows whose channel values a lane computes
    constexpr int W4 = THEMIS_SSM_MAX_CONV;
    const int D = p.pr.channels, N = FULL ? 4 * LPC : p.pr.state, W = p.pr.conv_width;
    const int d = l / LPC, part = l % LPC, n0 = part * 4;
    // lanes beyond the channels shadow the last one, without storing (they take part in the shuffles)
    const bool live = FULL || d < D;
    const int dd = FULL ? d : min(d, D - 1), g = p.pr.groups == 1 ? 0 : dd / (D / p.pr.groups), nn = FULL ? 4 : min(4, N - n0);
    const int rows = FULL ? ROWS : (int)min((int64_t)ROWS, p.pr.batch - b0);

    // the states of all rows are on their way first
    float h[ROWS][4];
    const float *h_in = p.in.ssm_state + (b0 * D + dd) * N + n0;
    const size_t h_row = (size_t)D * N;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) load4<float, VEC>(h_in + r * h_row, FULL ? 4 : r < rows ? nn : 0, h[r]);
    float A[4];
    load4<float, VEC>(p.in.a + (size_t)dd * N + n0, nn, A);

    Pair<T> bq[ROWS][2], cq[ROWS][2];       // B and C of the rows, as they are
    if (VEC) {
        const T *bp = (const T *)p.in.b + b0 * p.pr.b_row + g * p.pr.b_group + n0;
        const T *cp = (const T *)p.in.c + b0 * p.pr.c_row + g * p.pr.c_group + n0;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool in = FULL || (r < rows && nn > 0);
            raw4(bp + r * p.pr.b_row, in, bq[r]);
            raw4(cp + r * p.pr.c_row, in, cq[r]);
        }
    }

    // channel values of this lane's rows: part, part + LPC, ...
    T tap[OWN][W4];
    float step[OWN], u[OWN], gate[OWN];
    bool on[OWN], own[OWN];
    {
        float w[W4];
#pragma unroll
        for (int k = 0; k < W4; ++k) w[k] = k < W ? p.in.conv_weight[(size_t)dd * W + k] : 0.0f;
        const float conv_bias = p.in.conv_bias ? p.in.conv_bias[dd] : 0.0f, dt_bias = p.in.dt_bias ? p.in.dt_bias[dd] : 0.0f;
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            const int r = k * LPC + part;
            const int64_t b = b0 + r;
            own[k] = (FULL && ROWS % LPC == 0) || r < rows;
            on[k] = own[k] && (!p.in.lengths || p.in.lengths[b] >= 1);
            step[k] = u[k] = gate[k] = 0.0f;
            if (own[k]) {
                const T *conv_in = (const T *)p.in.conv_state + b * (W - 1) * D + dd;
#pragma unroll
                for (int i = 0; i < W4 - 1; ++i) tap[k][i] = i < W - 1 ? conv_in[(size_t)i * D] : from_f32<T>(0.0f);
            }
            if (on[k]) {
                const T now = ((const T *)p.in.x)[b * p.pr.x_row + dd];
                const float raw = to_f32(((const T *)p.in.dt)[b * p.pr.dt_row + dd]) + dt_bias;
                gate[k] = p.in.z ? silu(to_f32(((const T *)p.in.z)[b * p.pr.z_row + dd])) : 1.0f;
                float c = conv_bias;
#pragma unroll
                for (int i = 0; i < W4 - 1; ++i)
                    if (i < W - 1) c = fmaf(w[i], to_f32(tap[k][i]), c);
                c = fmaf(W == 4 ? w[3] : W == 3 ? w[2] : w[1], to_f32(now), c);
                u[k] = silu(c);
                step[k] = softplus(raw);
#pragma unroll
                for (int i = 0; i < W4 - 1; ++i)
                    if (i < W - 1) tap[k][i] = i < W - 2 ? tap[k][i + 1] : now;
            }
        }
    }

    // (scaled only here: where A is loaded, the scaling waits for it before the other loads are on their way; 254 us
    // against 229, 16384 x 512 x 16)
#pragma unroll
    for (int i = 0; i < 4; ++i) A[i] = log2_rate(A[i]);

    // states; a row that is not on has a step of 0: factors of 1, nothing added
    float v[ROWS];
    unsigned active = 0;
    constexpr unsigned kAll = 0xffffffffu;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int from = (threadIdx.x & 31 & ~(LPC - 1)) | (r % LPC);
        const float s = __shfl_sync(kAll, step[r / LPC], from), su = s * __shfl_sync(kAll, u[r / LPC], from);
        if (__shfl_sync(kAll, (int)on[r / LPC], from)) active |= 1u << r;
        float B[4], C[4];
        if (VEC) {
            unpack4<T>(bq[r], B);
            unpack4<T>(cq[r], C);
        } else {
            const int have = active >> r & 1 ? nn : 0;
            load4<T, false>((const T *)p.in.b + (b0 + r) * p.pr.b_row + g * p.pr.b_group + n0, have, B);
            load4<T, false>((const T *)p.in.c + (b0 + r) * p.pr.c_row + g * p.pr.c_group + n0, have, C);
        }
        v[r] = 0.0f;
        if (active >> r & 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[r][i] = fmaf(decay(s, A[i]), h[r][i], su * B[i]);
                v[r] = fmaf(h[r][i], C[i], v[r]);
            }
        }
#pragma unroll
        for (int o = LPC / 2; o > 0; o >>= 1) v[r] += __shfl_xor_sync(kAll, v[r], o);
    }
    // (the shuffles: all lanes of a channel have read its old inputs before any is overwritten in place)
    if (!live) return;
    float *h_out = p.out.ssm_state + (b0 * D + d) * N + n0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (r >= rows) break;
        if (VEC) {
            if (nn > 0) *reinterpret_cast<float4 *>(h_out + r * h_row) = make_float4(h[r][0], h[r][1], h[r][2], h[r][3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < nn) h_out[r * h_row + i] = h[r][i];
        }
    }
    const float skip = p.in.skip ? p.in.skip[d] : 0.0f;
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        if (!own[k]) continue;
        const int64_t b = b0 + k * LPC + part;
        T *conv_out = (T *)p.out.conv_state + b * (W - 1) * D + d;
#pragma unroll
        for (int i = 0; i < W4 - 1; ++i)
            if (i < W - 1) conv_out[(size_t)i * D] = tap[k][i];
        float mine = v[0];
#pragma unroll
        for (int r = 1; r < ROWS; ++r)
            if (r == k * LPC + part) mine = v[r];
        ((T *)p.out.y)[b * D + d] = from_f32<T>(on[k] ? fmaf(skip, u[k], mine) * gate[k] : 0.0f);
    }
}

template <typename T, int LPC, int ROWS, bool VEC>
__global__ __launch_bounds__(kStepThreads, LPC >= 4 && ROWS == 4 ? 3 : 4) void ssm_step_kernel(const SsmParams p, int blocks_per_row)
{
    const unsigned group = blockIdx.x / blocks_per_row;
    const int l0 = (blockIdx.x - group * blocks_per_row) * kStepThreads;
    const int64_t b0 = (int64_t)group * ROWS;
    if (VEC && LPC <= 4 && p.pr.state == 4 * LPC && b0 + ROWS <= p.pr.batch && l0 + kStepThreads <= p.pr.channels * LPC)
        step_rows<T, LPC, ROWS, VEC, true>(p, l0 + threadIdx.x, b0);
    else
        step_rows<T, LPC, ROWS, VEC, false>(p, l0 + threadIdx.x, b0);
}

template <typename T, int LPC, int ROWS> cudaError_t launch_rows(const SsmParams &p, cudaStream_t st)
{
    const int blocks_per_row = (int)(((long long)p.pr.channels * LPC + kStepThreads - 1) / kStepThreads);
    const unsigned blocks = (unsigned)(((p.pr.batch + (long long)ROWS - 1) / ROWS) * blocks_per_row);
    const size_t four = 4 * sizeof(T);
    const bool vec = p.pr.state % 4 == 0 && (((uintptr_t)p.in.ssm_state | (uintptr_t)p.out.ssm_state | (uintptr_t)p.in.a) & 15u) == 0 &&
                     (((uintptr_t)p.in.b | (uintptr_t)p.in.c) & (four - 1)) == 0 &&
                     ((p.pr.b_row | p.pr.b_group | p.pr.c_row | p.pr.c_group) & 3) == 0;
    if (vec)
        ssm_step_kernel<T, LPC, ROWS, true><<<blocks, kStepThreads, 0, st>>>(p, blocks_per_row);
    else
        ssm_step_kernel<T, LPC, ROWS, false><<<blocks, kStepThreads, 0, st>>>(p, blocks_per_row);
    return cudaGetLastError();
}

template <typename T, int LPC> cudaError_t launch_lanes(const SsmParams &p, cudaStream_t st)
{
    // As many rows to a thread as a channel has lanes (up to four: each computes one row's channel values)
    // once they fill the GPU's threads a few times all the same.  16384 x 512, bf16, when all were built: 16 states
    // 254 us with four rows, 283 with two, 455 with one; 8 states 195, 144, 230; 4 states 164, 121, 111 (the kept ones
    // are 227, 143 and 111 now).
    const double lanes = (double)p.pr.batch * p.pr.channels * LPC;
    return lanes >= 2.0 * 4 * 2048 * kSMs ? launch_rows<T, LPC, (LPC < 4 ? LPC : 4)>(p, st) : launch_rows<T, LPC, 1>(p, st);
}

template <typename T> cudaError_t launch(const SsmParams &p, cudaStream_t st)
{
    if (p.pr.state <= 4) return launch_lanes<T, 1>(p, st);
    if (p.pr.state <= 8) return launch_lanes<T, 2>(p, st);
    if (p.pr.state <= 16) return launch_lanes<T, 4>(p, st);
    if (p.pr.state <= 32) return launch_lanes<T, 8>(p, st);
    return launch_lanes<T, 16>(p, st);
}

}  // namespace

cudaError_t launch_ssm_step(const SsmParams &p, cudaStream_t st)
{
    switch (p.pr.dtype) {
        case THEMIS_DTYPE_F32: return launch<float>(p, st);
        case THEMIS_DTYPE_BF16: return launch<__nv_bfloat16>(p, st);
        default: return launch<__half>(p, st);
    }
}

}  // namespace themis
