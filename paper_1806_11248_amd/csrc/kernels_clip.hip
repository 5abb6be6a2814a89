// The global norm of many gradient tensors, and the gradients scaled down to a limit.
//
// Two launches over the same pieces: one adds up squares, the other scales (every workgroup adds up the few partial sums for itself,
// so no third launch stands between); few pieces take one.  Squares are summed in 64 bits: a square of any float is representable there, so neither large
// nor tiny gradients leave the range, and the order of the partial sums is fixed.  Bound: memory,
// of which the gradients are read twice, since the factor needs all of them.  220 tensors of 1000 to 5,000,000 elements, 310 MB: 79 us and 102, together
// 5.1 TB/s, the rate of a large copy (some of the second reading is met in the cache behind L2, and its dirty lines are written while the next norm is
// taken).
#include "gbt_internal.h"

namespace {

constexpr int kClipBlocks = 2048;   // workgroups of 256 threads, and doubles of workspace: what the compute units hold at once

template <typename E>
struct alignas(16) Vec {
    E x[16 / sizeof(E)];
};

// By kThreads threads, of which this one is number `thread`.
template <typename E, int kThreads>
__device__ __forceinline__ void add_squares(const ClipPiece &p, double (&sum)[4], int thread) {
    constexpr int kVec = 16 / sizeof(E);
    const E *src = (const E *)p.src;
    int i = 0;
    if (((uintptr_t)src & 15) == 0) {
        const int vecs = p.n / kVec;
        const Vec<E> *v = (const Vec<E> *)src;
        for (int at = thread; at < vecs; at += 4 * kThreads) {
            Vec<E> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (at + kThreads * u < vecs) x[u] = v[at + kThreads * u];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (at + kThreads * u < vecs)
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        const double w = (double)(float)x[u].x[e];
                        sum[e & 3] = fma(w, w, sum[e & 3]);
                    }
        }
        i = vecs * kVec;
    }
    for (i += thread; i < p.n; i += kThreads) {
        const double w = (double)(float)src[i];
        sum[0] = fma(w, w, sum[0]);
    }
}
template <int kThreads>
__device__ __forceinline__ void add_squares(const ClipPiece &p, double (&sum)[4], int thread) {
    if (p.dtype == GBT_F32) add_squares<float, kThreads>(p, sum, thread);
    else if (p.dtype == GBT_BF16) add_squares<__bf16, kThreads>(p, sum, thread);
    else add_squares<_Float16, kThreads>(p, sum, thread);
}

template <typename E, int kThreads>
__device__ __forceinline__ void scale_piece(const ClipPiece &p, float coef, int thread) {
    constexpr int kVec = 16 / sizeof(E);
    const E *src = (const E *)p.src;
    E *dst = (E *)p.dst;
    int i = 0;
    if ((((uintptr_t)src | (uintptr_t)dst) & 15) == 0) {
        const int vecs = p.n / kVec;
        for (int at = thread; at < vecs; at += 4 * kThreads) {
            Vec<E> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (at + kThreads * u < vecs) x[u] = ((const Vec<E> *)src)[at + kThreads * u];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (at + kThreads * u < vecs) {
#pragma unroll
                    for (int e = 0; e < kVec; ++e) x[u].x[e] = (E)((float)x[u].x[e] * coef);
                    ((Vec<E> *)dst)[at + kThreads * u] = x[u];
                }
        }
        i = vecs * kVec;
    }
    for (i += thread; i < p.n; i += kThreads) dst[i] = (E)((float)src[i] * coef);
}
template <int kThreads>
__device__ __forceinline__ void scale_piece(const ClipPiece &p, float coef, int thread) {
    if (coef == 1.0f && p.src == p.dst) return;
    if (p.dtype == GBT_F32) scale_piece<float, kThreads>(p, coef, thread);
    else if (p.dtype == GBT_BF16) scale_piece<__bf16, kThreads>(p, coef, thread);
    else scale_piece<_Float16, kThreads>(p, coef, thread);
}
// A norm that is no finite number says nothing about how to scale: the gradients stay as they are.
__device__ __forceinline__ float clip_factor(double norm, double max_norm) {
    return isfinite((float)norm) ? (float)fmin(1.0, max_norm / (norm + 1e-6)) : 1.0f;
}

__device__ __forceinline__ double block_sum(double x, double *part) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(256) void clip_norm_kernel(const ClipPiece *pieces, int n_pieces, double *sums) {
    __shared__ double part[4];
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    for (int i = blockIdx.x; i < n_pieces; i += gridDim.x) add_squares<256>(pieces[i], sum, threadIdx.x);
    const double all = block_sum((sum[0] + sum[1]) + (sum[2] + sum[3]), part);
    if (threadIdx.x == 0) sums[blockIdx.x] = all;
}

// Pieces in the opposite order: those read last are still in the cache behind L2.
__global__ __launch_bounds__(256) void clip_scale_kernel(const ClipPiece *pieces, int n_pieces, const double *sums, int n_sums, double max_norm,
                                                         float *norm_out) {
    __shared__ double part[4];
    double sum = 0.0;
    for (int i = threadIdx.x; i < n_sums; i += 256) sum += sums[i];
    const double norm = sqrt(block_sum(sum, part));
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const float coef = clip_factor(norm, max_norm);
    for (int i = n_pieces - 1 - (int)blockIdx.x; i >= 0; i -= gridDim.x) scale_piece<256>(pieces[i], coef, threadIdx.x);
}

// Few pieces: both in one launch, by one workgroup, a wave to a piece.  (us a call with two launches and with one: 16 pieces of 2048 float32 elements 9.3,
// 6.5; 24 9.3, 8.1; 32 9.2, 10.3; 64 9.3, 17.7.)
constexpr int kClipFew = 24;
__global__ __launch_bounds__(1024) void clip_few_kernel(const ClipPiece *pieces, int n_pieces, double max_norm, float *norm_out) {
    __shared__ double part[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    for (int i = wave; i < n_pieces; i += 16) add_squares<64>(pieces[i], sum, lane);
    double all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) all += __shfl_xor(all, s);
    if (lane == 0) part[wave] = all;
    __syncthreads();
    all = 0.0;
#pragma unroll
    for (int w = 0; w < 16; ++w) all += part[w];
    const double norm = sqrt(all);
    if (threadIdx.x == 0) *norm_out = (float)norm;
    const float coef = clip_factor(norm, max_norm);
    for (int i = wave; i < n_pieces; i += 16) scale_piece<64>(pieces[i], coef, lane);
}

}  // namespace

hipError_t gbt_launch_clip(hipStream_t stream, const ClipPiece *pieces, int n_pieces, double max_norm, float *norm_out, double *sums) {
    if (n_pieces <= kClipFew) {
        clip_few_kernel<<<1, 1024, 0, stream>>>(pieces, n_pieces, max_norm, norm_out);
        return hipGetLastError();
    }
    const int blocks = std::min(n_pieces, kClipBlocks);
    clip_norm_kernel<<<blocks, 256, 0, stream>>>(pieces, n_pieces, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    clip_scale_kernel<<<blocks, 256, 0, stream>>>(pieces, n_pieces, sums, blocks, max_norm, norm_out);
    return hipGetLastError();
}
