// Matrix product with bias, activation and residual, and its gradients: the passes around the
// tensor-core product, and the product for a few rows.
#include "themis_gemm.cuh"

namespace themis {
namespace {

// --- a few rows: the weights are what is read ----------------------------------------------------
//
// With at most 8 NT rows a 128-row tile would be mostly empty and the few tiles would leave most of
// the GPU idle, while the time is that of reading the weights once.  So the output features are
// spread over blocks of 16 and the depth over the block's 8 warps; the weights are the left operand
// of mma m16n8k16 and the rows of x its 8 columns.  Which depth index an operand register stands for
// is free as long as both operands agree, so a thread takes 8 neighbouring k with one 16-byte load
// and uses them for two products: weights and x go from memory to the product's registers directly.
constexpr int kFewWarps = 8;
constexpr int kFewRows = 32;          // most rows of this path

template <typename T> struct Mma;
template <> struct Mma<__nv_bfloat16> {
    __device__ __forceinline__ static void run(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <> struct Mma<__half> {
    __device__ __forceinline__ static void run(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

// 8 values of a row from k on, zeros beyond K (VEC: K, pitches and addresses allow one 16-byte load)
template <typename T, bool VEC>
__device__ __forceinline__ uint4 load8(const T *row, bool in, int k, int K)
{
    uint4 r = make_uint4(0, 0, 0, 0);
    if (!in || k >= K) return r;
    if (VEC) return *reinterpret_cast<const uint4 *>(row + k);
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? row[k + i] : from_f32<T>(0.0f);
    memcpy(&r, v, sizeof(r));
    return r;
}

template <typename T, int NT, bool VEC>
__global__ __launch_bounds__(32 * kFewWarps) void few_rows_kernel(const T *x, int64_t x_row, const T *w, int64_t w_row, int M, int N, int K,
                                                                  const GemmEpilogue e)
{
    __shared__ float s_sum[kFewWarps][8 * NT][16 + 1];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int f0 = blockIdx.x * 16;
    const T *w0 = w + (int64_t)min(f0 + g, N - 1) * w_row, *w1 = w + (int64_t)min(f0 + g + 8, N - 1) * w_row;
    float c[NT][4] = {};
#pragma unroll 4
    for (int k = warp * 32 + t * 8; k - t * 8 < K; k += kFewWarps * 32) {
        const uint4 a0 = load8<T, VEC>(w0, true, k, K), a1 = load8<T, VEC>(w1, true, k, K);
        const uint32_t lo[4] = {a0.x, a1.x, a0.y, a1.y}, hi[4] = {a0.z, a1.z, a0.w, a1.w};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int m = j * 8 + g;
            const uint4 b = load8<T, VEC>(x + (int64_t)min(m, M - 1) * x_row, m < M, k, K);
            Mma<T>::run(c[j], lo, b.x, b.y);
            Mma<T>::run(c[j], hi, b.z, b.w);
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        s_sum[warp][j * 8 + 2 * t][g] = c[j][0];
        s_sum[warp][j * 8 + 2 * t + 1][g] = c[j][1];
        s_sum[warp][j * 8 + 2 * t][g + 8] = c[j][2];
        s_sum[warp][j * 8 + 2 * t + 1][g + 8] = c[j][3];
    }
    __syncthreads();
    for (int at = threadIdx.x; at < 16 * 8 * NT; at += 32 * kFewWarps) {
        const int m = at / 16, n = f0 + at % 16;
        if (m >= M || n >= N) continue;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kFewWarps; ++k) v += s_sum[k][m][at % 16];
        if (e.bias) v += e.bias[n];
        const int64_t to = (int64_t)m * N + n;
        if (e.pre) ((T *)e.pre)[to] = from_f32<T>(v);
        v = activate(v, e.act);
        if (e.residual) v += to_f32(((const T *)e.residual)[m * e.residual_row + n]);
        ((T *)e.y)[to] = from_f32<T>(v);
    }
}

template <typename T, int NT>
cudaError_t launch_few(const LinearParams &p, const GemmEpilogue &e, cudaStream_t st)
{
    const int M = p.pr.rows, N = p.pr.out_features, K = p.pr.in_features;
    const bool vec = K % 8 == 0 && p.pr.x_row % 8 == 0 && p.pr.weight_row % 8 == 0 && (((uintptr_t)p.x | (uintptr_t)p.weight) & 15u) == 0;
    const int blocks = (N + 15) / 16;
    if (vec)
        few_rows_kernel<T, NT, true><<<blocks, 32 * kFewWarps, 0, st>>>((const T *)p.x, p.pr.x_row, (const T *)p.weight, p.pr.weight_row, M, N, K, e);
    else
        few_rows_kernel<T, NT, false><<<blocks, 32 * kFewWarps, 0, st>>>((const T *)p.x, p.pr.x_row, (const T *)p.weight, p.pr.weight_row, M, N, K, e);
    return cudaGetLastError();
}

// --- operands that TMA cannot read: rows copied to a pitch of a multiple of 16 bytes ---------------
// A block takes 512 columns of a row after the other, two columns to a thread; rows of the copy have an
// even pitch, so a pair is stored at once.
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(const T *from, int64_t from_row, T *to, int64_t to_row, int rows, int width)
{
    const int c = blockIdx.x * 512 + 2 * threadIdx.x;
    if (c >= width) return;
    const bool two = c + 1 < width;
    constexpr int U = 4;
    for (long long r0 = (long long)blockIdx.y * U; r0 < rows; r0 += (long long)gridDim.y * U) {
        uint32_t v[U];
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (r0 + k < rows) v[k] = load_two(from + (r0 + k) * from_row + c, two);
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (r0 + k < rows) *reinterpret_cast<uint32_t *>(to + (r0 + k) * to_row + c) = v[k];
    }
}

inline int64_t round8(int64_t v) { return (v + 7) / 8 * 8; }

struct Bump {
    char *base;
    size_t off;
    void *take(size_t bytes)
    {
        void *at = base ? base + off : nullptr;
        off += align256(bytes);
        return at;
    }
};

inline bool needs_copy(int64_t pitch, bool unaligned) { return unaligned || pitch % 8 != 0; }

template <typename T>
cudaError_t aligned_rows(const void *&ptr, int64_t &pitch, int rows, int width, void *copy, cudaStream_t st)
{
    const dim3 grid((width + 511) / 512, (unsigned)std::min(65535, (rows + 3) / 4));
    copy_rows_kernel<T><<<grid, 256, 0, st>>>((const T *)ptr, pitch, (T *)copy, round8(width), rows, width);
    ptr = copy;
    pitch = round8(width);
    return cudaGetLastError();
}

// --- q = dy act'(pre) and the bias gradient ----------------------------------------------------------
//
// Reads dy and pre once and writes q once.  A block takes 256 columns of some rows, 8 columns
// to a thread (VEC) and 8 threads to a column; the sums of q over the block's rows are added in
// shared memory and, over the blocks, by column_sum_kernel, always in the same order.
// q is rounded to the 16 bits of the other operand, because a tensor-core product takes both in that type; its
// low bits as a second product would double the time of both.  The relative error of dx and dweight against 64 bits
// grows by it from 0.0017 to 0.0023 in bf16 (32768 x 4096 x 1024) and from 0.00021 to 0.00029 in fp16 (777 x 328 x
// 200), of which the outputs' own rounding is the first number.  The bias gradient sums q unrounded, in 32 bits.
// rows of a block: 64, or 16 where those would be too few blocks to fill the GPU (777 x 328 with gelu: 16 us
// with 64, 5 us with 16)
inline int slope_rows(int M, int N) { return (long long)((N + 255) / 256) * ((M + 63) / 64) >= 2 * kSMs ? 64 : 16; }

// d *= act'(v), one branch for the eight values
__device__ __forceinline__ void slopes(float (&d)[8], const float (&v)[8], int act)
{
    if (act == THEMIS_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= act_slope(v[j], THEMIS_ACT_SILU);
    } else if (act == THEMIS_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= act_slope(v[j], THEMIS_ACT_GELU);
    } else if (act == THEMIS_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= act_slope(v[j], THEMIS_ACT_RELU);
    }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void slope_kernel(const T *dy, int64_t dy_row, const T *pre, int act, T *q, int64_t q_row, float *part,
                                                    int M, int N, int block_rows)
{
    __shared__ float s_sum[8][256 + 8];
    const int cg = threadIdx.x % 32, rl = threadIdx.x / 32;
    const int n0 = blockIdx.x * 256 + (VEC ? cg * 8 : cg);
    constexpr int STEP = VEC ? 1 : 32;                  // columns of a thread: neighbours, or 32 apart
    for (long long r0 = (long long)blockIdx.y * block_rows; r0 < M; r0 += (long long)gridDim.y * block_rows) {
        float s[8] = {};
        // four rows' values on their way at a time
#pragma unroll 1
        for (int i0 = 0; i0 < block_rows / 8; i0 += 4) {
            uint4 dq[4], pq[4];
            if (VEC) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const long long m = r0 + (i0 + k) * 8 + rl;
                    const bool in = m < M && n0 < N && (i0 + k) * 8 < block_rows;
                    dq[k] = in ? *reinterpret_cast<const uint4 *>(dy + m * dy_row + n0) : make_uint4(0, 0, 0, 0);
                    pq[k] = in && act != THEMIS_ACT_NONE ? *reinterpret_cast<const uint4 *>(pre + m * N + n0) : make_uint4(0, 0, 0, 0);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const long long m = r0 + (i0 + k) * 8 + rl;
                if (m >= M || n0 >= N || (i0 + k) * 8 >= block_rows) continue;
                float d[8], v[8];
                if (VEC) {
                    const T *t = reinterpret_cast<const T *>(&dq[k]), *u = reinterpret_cast<const T *>(&pq[k]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        d[j] = to_f32(t[j]);
                        v[j] = to_f32(u[j]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int n = n0 + j * STEP;
                        d[j] = n < N ? to_f32(dy[m * dy_row + n]) : 0.0f;
                        v[j] = n < N && act != THEMIS_ACT_NONE ? to_f32(pre[m * N + n]) : 0.0f;
                    }
                }
                slopes(d, v, act);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += d[j];
                if (q) {
                    if (VEC) {
                        T o[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = from_f32<T>(d[j]);
                        uint4 w;
                        memcpy(&w, o, sizeof(w));
                        *reinterpret_cast<uint4 *>(q + m * q_row + n0) = w;
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (n0 + j * STEP < N) q[m * q_row + n0 + j * STEP] = from_f32<T>(d[j]);
                    }
                }
            }
        }
        if (part) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) s_sum[rl][VEC ? cg * 8 + j : cg + j * 32] = s[j];
            __syncthreads();
            const int n = blockIdx.x * 256 + threadIdx.x;
            if (n < N) {
                float v = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) v += s_sum[k][threadIdx.x];
                part[(r0 / block_rows) * N + n] = v;
            }
        }
    }
}

__global__ __launch_bounds__(256) void column_sum_kernel(const float *part, float *out, int parts, int N)
{
    __shared__ float s_sum[8][32];
    const int n = blockIdx.x * 32 + threadIdx.x % 32, w = threadIdx.x / 32;
    float s = 0.0f;
    if (n < N)
        for (int k = w; k < parts; k += 8) s += part[(size_t)k * N + n];
    s_sum[w][threadIdx.x % 32] = s;
    __syncthreads();
    if (w > 0 || n >= N) return;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += s_sum[k][threadIdx.x];
    out[n] = s;
}

// --- workspaces -------------------------------------------------------------------------------------
struct ForwardSpace { void *x, *weight; size_t bytes; };
ForwardSpace forward_space(const themis_linear_problem_t &pr, bool unaligned, char *base)
{
    Bump b{base, 0};
    ForwardSpace s{};
    if (pr.rows > kFewRows) {
        if (needs_copy(pr.x_row, unaligned)) s.x = b.take((size_t)pr.rows * round8(pr.in_features) * 2);
        if (needs_copy(pr.weight_row, unaligned)) s.weight = b.take((size_t)pr.out_features * round8(pr.in_features) * 2);
    }
    s.bytes = b.off;
    return s;
}

struct BackwardSpace { void *q, *x, *weight; float *sums, *partial; GemmPlan dx, dw; size_t bytes; };
BackwardSpace backward_space(const themis_linear_problem_t &pr, bool unaligned, char *base)
{
    Bump b{base, 0};
    BackwardSpace s{};
    const int M = pr.rows, N = pr.out_features, K = pr.in_features;
    if (pr.activation != THEMIS_ACT_NONE || needs_copy(pr.dy_row, unaligned)) s.q = b.take((size_t)M * round8(N) * 2);
    if (needs_copy(pr.x_row, unaligned)) s.x = b.take((size_t)M * round8(K) * 2);
    if (needs_copy(pr.weight_row, unaligned)) s.weight = b.take((size_t)N * round8(K) * 2);
    const int block_rows = slope_rows(M, N);
    s.sums = (float *)b.take((size_t)((M + block_rows - 1) / block_rows) * N * sizeof(float));
    s.dx = gemm_plan(M, K, N, true);
    s.dw = gemm_plan(N, K, M, true);
    s.partial = (float *)b.take(std::max(gemm_partial_bytes(s.dx, M, K), gemm_partial_bytes(s.dw, N, K)));
    s.bytes = b.off;
    return s;
}

template <typename T> cudaError_t forward(const LinearParams &p, cudaStream_t st)
{
    const int M = p.pr.rows, N = p.pr.out_features, K = p.pr.in_features;
    GemmEpilogue e{};
    e.bias = p.bias;
    e.residual = p.residual;
    e.residual_row = p.pr.residual_row;
    e.act = p.pr.activation;
    e.y = p.y;
    e.pre = p.pre_out;
    e.status = p.status;
    if (M <= kFewRows) {
        if (M <= 8) return launch_few<T, 1>(p, e, st);
        if (M <= 16) return launch_few<T, 2>(p, e, st);
        return launch_few<T, 4>(p, e, st);
    }
    const bool unaligned = (((uintptr_t)p.x | (uintptr_t)p.weight) & 15u) != 0;
    const ForwardSpace s = forward_space(p.pr, unaligned, p.ws);
    GemmOperand a{p.x, p.pr.x_row, false}, b{p.weight, p.pr.weight_row, false};
    cudaError_t err = cudaSuccess;
    if (s.x) err = aligned_rows<T>(a.ptr, a.pitch, M, K, s.x, st);
    if (err == cudaSuccess && s.weight) err = aligned_rows<T>(b.ptr, b.pitch, N, K, s.weight, st);
    if (err != cudaSuccess) return err;
    return launch_gemm<T>(gemm_plan(M, N, K, false), M, N, K, a, b, e, nullptr, st);
}

template <typename T> cudaError_t backward(const LinearParams &p, cudaStream_t st)
{
    const int M = p.pr.rows, N = p.pr.out_features, K = p.pr.in_features, act = p.pr.activation;
    const bool unaligned = (((uintptr_t)p.dy | (uintptr_t)p.x | (uintptr_t)p.weight) & 15u) != 0;
    const BackwardSpace s = backward_space(p.pr, unaligned, p.ws);
    GemmOperand q{p.dy, p.pr.dy_row, false};
    cudaError_t err = cudaSuccess;
    const bool want_q = s.q && (p.dx || p.dweight);
    if (want_q || p.dbias) {
        const int block_rows = slope_rows(M, N), parts = (M + block_rows - 1) / block_rows;
        const dim3 grid((N + 255) / 256, std::min(parts, 65535));
        const bool vec = N % 8 == 0 && p.pr.dy_row % 8 == 0 && (((uintptr_t)p.dy | (uintptr_t)p.pre_in) & 15u) == 0;
        T *to = want_q ? (T *)s.q : nullptr;
        float *sums = p.dbias ? s.sums : nullptr;
        if (vec) slope_kernel<T, true><<<grid, 256, 0, st>>>((const T *)p.dy, p.pr.dy_row, (const T *)p.pre_in, act, to, round8(N), sums, M, N, block_rows);
        else slope_kernel<T, false><<<grid, 256, 0, st>>>((const T *)p.dy, p.pr.dy_row, (const T *)p.pre_in, act, to, round8(N), sums, M, N, block_rows);
        if (p.dbias) column_sum_kernel<<<(N + 31) / 32, 256, 0, st>>>(s.sums, p.dbias, parts, N);
        err = cudaGetLastError();
        if (want_q) q = GemmOperand{s.q, round8(N), false};
    }
    if (err == cudaSuccess && p.dx) {
        GemmOperand w{p.weight, p.pr.weight_row, true};
        if (s.weight) err = aligned_rows<T>(w.ptr, w.pitch, N, K, s.weight, st);
        GemmEpilogue e{};
        e.y = p.dx;
        e.status = p.status;
        if (err == cudaSuccess) err = launch_gemm<T>(s.dx, M, K, N, q, w, e, s.partial, st);
    }
    if (err == cudaSuccess && p.dweight) {
        GemmOperand x{p.x, p.pr.x_row, true};
        if (s.x) err = aligned_rows<T>(x.ptr, x.pitch, M, K, s.x, st);
        q.mn_major = true;
        GemmEpilogue e{};
        e.y = p.dweight;
        e.status = p.status;
        if (err == cudaSuccess) err = launch_gemm<T>(s.dw, N, K, M, q, x, e, s.partial, st);
    }
    return err;
}

}  // namespace

size_t linear_forward_workspace(const themis_linear_problem_t &pr, bool unaligned) { return forward_space(pr, unaligned, nullptr).bytes; }
size_t linear_backward_workspace(const themis_linear_problem_t &pr, bool unaligned) { return backward_space(pr, unaligned, nullptr).bytes; }

cudaError_t launch_linear_forward(const LinearParams &p, cudaStream_t st)
{
    return p.pr.dtype == THEMIS_DTYPE_BF16 ? forward<__nv_bfloat16>(p, st) : forward<__half>(p, st);
}

cudaError_t launch_linear_backward(const LinearParams &p, cudaStream_t st)
{
    return p.pr.dtype == THEMIS_DTYPE_BF16 ? backward<__nv_bfloat16>(p, st) : backward<__half>(p, st);
}

}  // namespace themis
