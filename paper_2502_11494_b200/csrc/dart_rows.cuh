// Rows of queries, keys and values: the norm of each head and the position rotation in one pass, written densely or into the
// pages of a cache.
//
// For a row's head x of D values:  y = x * rsqrt(mean(x^2) + eps) * w;  with angle_i = pos * inv_freq[i], i < half:
//   halves:       z[i] = y[i] cos_i - y[i + half] sin_i,      z[i + half]  = y[i + half] cos_i + y[i] sin_i
//   interleaved:  the same with elements 2i and 2i + 1;  elements from 2 half on stay y.
// Everything is held in fp32 and rounded once, when it is stored.  An angle is a product in fp64, reduced to one turn there
// (rint of the number of turns), so that far positions lose little (two products' roundings, 3 2^-53 of all turns); what is left of it goes
// through sincospif in fp32.
//
// Bound by memory, with the SM's issue close behind (77 % of it): each value is read once and written once.  A thread owns both halves
// of eight rotated pairs (two 16-byte loads, two 16-byte stores) and needs nobody else's values but for the sum of squares (shuffles
// among the 4 to 16 threads of a head).  A row's cosines and sines are taken once per block, into shared memory, and serve all of its
// heads (per head they would be most of the kernel's instructions).  Both sides' weights kept in registers, 16 more: 5 % slower.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dart_common.cuh"

namespace dart {
namespace rows {

constexpr int kThreads = 128;
constexpr int kMaxRows = 8;      // rows per block
constexpr int kMaxHalf = 128;    // rotated pairs of a head (head_dim <= 256)

// One kind of row: queries, keys or values.
struct Side {
    const char *src;
    char *dst;             // dense: rows; paged: the cache
    const char *weight;    // [D] of the rows' type, or NULL: no norm
    long long src_stride, dst_stride; // bytes from row to row
    int heads;
    bool turn;             // rotate
};

struct Params {
    Side side[2];
    int n_rows, D, half, interleaved, n_axes, sec0, sec01; // pairs below sec0 turn by the first axis, below sec01 by the second
    float eps;
    const float *inv_freq;
    const int64_t *pos;    // [n_axes][pos_stride], or NULL: a paged row's position is its slot
    long long pos_stride;
    int rows_per_block, heads_per_block;
    // paged
    int n_seq, per_seq, S, table_stride, page_size, n_pages;
    const int32_t *cu, *idx, *table, *start;
    int32_t *status;
};

template <typename T>
__device__ __forceinline__ void widen(uint4 w, float *f);
template <>
__device__ __forceinline__ void widen<__nv_bfloat16>(uint4 w, float *f)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = bf16_lo(u[i]), f[2 * i + 1] = bf16_hi(u[i]);
}
template <>
__device__ __forceinline__ void widen<__half>(uint4 w, float *f)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
        f[2 * i] = v.x, f[2 * i + 1] = v.y;
    }
}
template <typename T>
__device__ __forceinline__ uint32_t narrow2(float a, float b);
template <>
__device__ __forceinline__ uint32_t narrow2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t narrow2<__half>(float a, float b)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <typename T>
__device__ __forceinline__ uint4 narrow8(const float *f)
{
    return make_uint4(narrow2<T>(f[0], f[1]), narrow2<T>(f[2], f[3]), narrow2<T>(f[4], f[5]), narrow2<T>(f[6], f[7]));
}

// Where a packed row comes from and goes to.
struct Place {
    long long src;  // source row; < 0: the row is not handled
    long long page; // paged: (page * heads) of the cache, to be completed by the head; dense: unused
    int at;         // paged: the place inside the page
    long long slot; // paged: the token's number in its sequence
};

__device__ __forceinline__ Place place_of(const Params &p, int n)
{
    Place r{-1, 0, 0, 0};
    int b, t;
    if (p.cu) {
        if (n < p.cu[0] || n >= p.cu[p.n_seq]) return r; // behind the last sequence: left alone
        int lo = 0, hi = p.n_seq; // the last b with cu[b] <= n
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.cu[mid] <= n)
                lo = mid;
            else
                hi = mid;
        }
        b = lo, t = n - p.cu[lo];
    } else {
        b = n / p.per_seq, t = n - b * p.per_seq;
    }
    const long long slot = (long long)(p.start ? p.start[b] : 0) + t;
    const long long col = slot / p.page_size;
    int page = -1;
    if (slot >= 0 && col < p.table_stride) page = p.table[(long long)b * p.table_stride + col];
    const long long src = p.idx ? (long long)p.idx[n] : n;
    if (page < 0 || page >= p.n_pages || (p.idx && (src < 0 || src >= p.S))) {
        report_check(p.status);
        return r;
    }
    r.src = p.idx ? (long long)b * p.S + src : src;
    r.page = page, r.at = (int)(slot - col * p.page_size), r.slot = slot;
    return r;
}

// kHead: threads of a head (the next power of two of D / 16, at least 4).
template <typename T, int kHead, bool kPaged>
__global__ void __launch_bounds__(kThreads) head_rows_kernel(const Params p)
{
    constexpr int kGroups = kThreads / kHead;
    __shared__ __align__(16) float s_cos[kMaxRows][kMaxHalf], s_sin[kMaxRows][kMaxHalf];
    __shared__ Place s_place[kMaxRows];
    const int tid = threadIdx.x, g = tid / kHead, lane = tid % kHead;
    const int row0 = blockIdx.x * p.rows_per_block, n_here = min(p.rows_per_block, p.n_rows - row0);
    const int H = p.side[0].heads + p.side[1].heads;
    const int h0 = blockIdx.y * p.heads_per_block, nh = min(p.heads_per_block, H - h0);
    const float inv_D = 1.0f / (float)p.D;
    wait_for_previous();
    if (kPaged) {
        if (tid < n_here) s_place[tid] = place_of(p, row0 + tid);
        __syncthreads();
    }

    // the thread's two pieces of eight values: both halves of eight pairs, or two pieces that do not turn
    const int turned = p.half >> 3, pieces = p.D >> 3; // slots that turn
    int c0, c1;
    if (lane < turned)
        c0 = p.interleaved ? 2 * lane : lane, c1 = p.interleaved ? 2 * lane + 1 : lane + turned;
    else
        c0 = 2 * lane, c1 = 2 * lane + 1;
    const bool has0 = c0 < pieces, has1 = c1 < pieces;

    const int total = n_here * nh, n_iter = (total + kGroups - 1) / kGroups;
    int row = 0, h = g; // of the item at hand, h relative to h0
    while (h >= nh) h -= nh, ++row;
    uint4 w0, w1;
    const auto fetch = [&](int r, int hh) {
        w0 = w1 = make_uint4(0, 0, 0, 0);
        if (r >= n_here) return;
        const bool second = h0 + hh >= p.side[0].heads;
        const Side &s = p.side[second];
        const long long src = kPaged ? s_place[r].src : row0 + r;
        if (src < 0) return;
        const uint4 *at = reinterpret_cast<const uint4 *>(s.src + src * s.src_stride) + (long long)(h0 + hh - (second ? p.side[0].heads : 0)) * pieces;
        if (has0) w0 = ld_stream<true>(at + c0);
        if (has1) w1 = ld_stream<true>(at + c1);
    };
    fetch(row, h);

    if (p.half) { // the rows' angles, behind the first loads
        for (int i = tid; i < n_here * p.half; i += kThreads) {
            const int r = i / p.half, j = i - r * p.half;
            const int axis = p.n_axes == 1 ? 0 : (j >= p.sec0) + (j >= p.sec01);
            long long where;
            if (kPaged)
                where = s_place[r].src < 0 ? 0 : (p.pos ? p.pos[axis * p.pos_stride + row0 + r] : s_place[r].slot);
            else
                where = p.pos[axis * p.pos_stride + row0 + r];
            double turns = (double)where * (double)p.inv_freq[j] * 0.15915494309189533577; // / 2 pi
            turns -= rint(turns);
            float sn, cs;
            sincospif(2.0f * (float)turns, &sn, &cs);
            s_cos[r][j] = cs, s_sin[r][j] = sn;
        }
        __syncthreads();
    }

    for (int it = 0; it < n_iter; ++it) {
        const int r = row, hh = h;
        const uint4 a = w0, b = w1;
        h += kGroups;
        while (h >= nh && row < n_here) h -= nh, ++row;
        if (it + 1 < n_iter) fetch(row, h);
        const bool here = r < n_here && (!kPaged || s_place[r].src >= 0);
        const bool second = h0 + hh >= p.side[0].heads;
        const Side &s = p.side[second];
        const bool norm = s.weight != nullptr, turn = s.turn && lane < turned;
        uint4 out0 = a, out1 = b;
        // (whether a side has a norm may differ inside a warp: the shuffles are taken by all)
        float x[8], y[8], ss = 0.0f;
        widen<T>(a, x), widen<T>(b, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
        if (p.side[0].weight || p.side[1].weight) {
#pragma unroll
            for (int o = kHead / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        }
        if (here && (norm || turn)) {
            if (norm) {
                const float scale = rsqrtf(ss * inv_D + p.eps);
                float u[8];
                const uint4 *w = reinterpret_cast<const uint4 *>(s.weight);
                if (has0) {
                    widen<T>(w[c0], u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = x[i] * scale * u[i];
                }
                if (has1) {
                    widen<T>(w[c1], u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = y[i] * scale * u[i];
                }
            }
            if (turn) {
                float cs[8], sn[8];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    *reinterpret_cast<float4 *>(cs + 4 * i) = *reinterpret_cast<const float4 *>(&s_cos[r][8 * lane + 4 * i]);
                    *reinterpret_cast<float4 *>(sn + 4 * i) = *reinterpret_cast<const float4 *>(&s_sin[r][8 * lane + 4 * i]);
                }
                if (!p.interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = x[i] * cs[i] - y[i] * sn[i];
                        y[i] = y[i] * cs[i] + x[i] * sn[i];
                        x[i] = u;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float u = x[2 * i] * cs[i] - x[2 * i + 1] * sn[i];
                        x[2 * i + 1] = x[2 * i + 1] * cs[i] + x[2 * i] * sn[i];
                        x[2 * i] = u;
                        u = y[2 * i] * cs[4 + i] - y[2 * i + 1] * sn[4 + i];
                        y[2 * i + 1] = y[2 * i + 1] * cs[4 + i] + y[2 * i] * sn[4 + i];
                        y[2 * i] = u;
                    }
                }
            }
            out0 = narrow8<T>(x), out1 = narrow8<T>(y);
        }
        if (here) {
            const int head = h0 + hh - (second ? p.side[0].heads : 0);
            char *at;
            if (kPaged)
                at = s.dst + (((s_place[r].page * s.heads + head) * p.page_size + s_place[r].at) * (long long)p.D) * 2;
            else
                at = s.dst + (row0 + r) * s.dst_stride + (long long)head * p.D * 2;
            if (has0) st_stream(reinterpret_cast<uint4 *>(at) + c0, out0);
            if (has1) st_stream(reinterpret_cast<uint4 *>(at) + c1, out1);
        }
    }
}

} // namespace rows
} // namespace dart
