// Addressing shared by the selective-scan kernels.
#pragma once

#include "themis_forecast_internal.h"
#include "themis_numeric.cuh"

namespace themis {

// the row's number of times, as the interface clamps it
__device__ __forceinline__ int row_length(const SsmParams &p, int b)
{
    if (!p.in.lengths) return p.pr.length;
    return min(max(p.in.lengths[b], 0), p.pr.length);
}

// Channel tiles do not cross a group: tile -> group, first channel, number of channels.
__device__ __forceinline__ void tile_of_block(const SsmParams &p, int tile, int ct, int &group, int &d0, int &nd)
{
    const int per = p.pr.channels / p.pr.groups;
    group = tile / p.tiles_per_group;
    const int first = (tile - group * p.tiles_per_group) * ct;
    d0 = group * per + first;
    nd = min(ct, per - first);
}

// --- asynchronous copies of rows into shared memory -----------------------------------------------
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// A block's copies of ROWS rows of `width` <= PITCH values, one row per time, into shared memory rows
// of PITCH values; times below 0 or from t_live on become zeros and are not read.  Columns from width
// on are not written, or written with zeros.  16 bytes a copy where addresses, pitch and width allow
// it, otherwise value by value.
template <typename T, int PITCH, int ROWS, int THREADS> struct RowCopy {
    static constexpr int V = 16 / sizeof(T) < PITCH ? 16 / sizeof(T) : PITCH;     // values of a copy
    static constexpr int PER = PITCH / V, ITEMS = ROWS * PER, K = (ITEMS + THREADS - 1) / THREADS;
    const T *src;
    int64_t stride;
    uint32_t off[K];        // bytes from the first row to this thread's values (~0: none)
    int width;
    bool vec, whole;

    __device__ __forceinline__ RowCopy(const T *from, int64_t row_stride, int w, int tid) : src(from), stride(row_stride), width(w)
    {
        vec = V * sizeof(T) == 16 && ((uintptr_t)from & 15u) == 0 && (row_stride * sizeof(T)) % 16 == 0;
        whole = vec && w % V == 0 && row_stride < (1ll << 31) / (ROWS * (int)sizeof(T));
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = tid + k * THREADS;
            off[k] = i < ITEMS && i % PER * V < w ? (uint32_t)(((int64_t)(i / PER) * row_stride + i % PER * V) * sizeof(T)) : ~0u;
        }
    }
    __device__ __forceinline__ static void async16(T *to, const char *from)
    {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
    }
    // rows of times t0 .. t0 + ROWS - 1
    __device__ __forceinline__ void run(T *dst, int t0, int t_live, int tid) const
    {
        if (whole && t0 >= 0 && t0 + ROWS <= t_live) {
            const char *base = reinterpret_cast<const char *>(src + t0 * stride);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (off[k] != ~0u) async16(dst + (tid + k * THREADS) * V, base + off[k]);
            return;
        }
        if (vec && width % V == 0) {                     // the row's ends
#pragma unroll 1
            for (int i = tid; i < ITEMS; i += THREADS) {
                const int c = i % PER * V, t = t0 + i / PER;
                if (c >= width) continue;
                if (t >= 0 && t < t_live) async16(dst + i * V, reinterpret_cast<const char *>(src + (int64_t)t * stride + c));
                else *reinterpret_cast<uint4 *>(dst + i * V) = make_uint4(0, 0, 0, 0);
            }
            return;
        }
        // value by value, neighbouring threads at neighbouring columns, eight on their way at a time
        constexpr int ALL = ROWS * PITCH, U = 8;
#pragma unroll 1
        for (int i0 = tid; i0 < ALL; i0 += U * THREADS) {
            T v[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * THREADS, c = i % PITCH, t = t0 + i / PITCH;
                v[k] = i < ALL && c < width && t >= 0 && t < t_live ? src[(int64_t)t * stride + c] : from_f32<T>(0.0f);
            }
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (i0 + k * THREADS < ALL) dst[i0 + k * THREADS] = v[k];
        }
    }
};

// two neighbouring values in shared memory
template <typename T> __device__ __forceinline__ void get_pair(const T *p, float (&v)[2])
{
    Unpack<T>::run(*reinterpret_cast<const Pair<T> *>(p), v);
}

}  // namespace themis
