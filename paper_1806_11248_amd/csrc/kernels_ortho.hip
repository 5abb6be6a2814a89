// Updates of weight matrices, orthogonalised: X = G / |G|, then X <- (a I + b A + c A^2) X with A = X X^T, a few times, which takes all singular values
// towards one.
//
// Such steps multiply small singular values, and with them whatever rounding left there, by a^steps (some 500), so sixteen bits do not do for what lies
// between products, and matrix instructions on 32 bits run at a sixteenth of the rate.  Everything between products is held in two float16 parts, high
// and low, 22 bits in all, and a product is three on the matrix units: high * high + high * low + low * high, added up in 32 bits.  All values are held times
// 2^8: X's entries lie around 1 / sqrt(w), and so their low parts stay among float16's normal numbers.  The errors left are those of 32-bit products.
//
// All products have both operands' rows along the sum: A = X X^T, A^2 = A A^T, and B X = B (X^T)^T, for which X's transpose is kept beside it.  The first
// two are symmetric: their upper tiles are computed, and written twice.
#include "ortho.h"
#include "attention.h"

namespace {

constexpr float kUp = 256.0f, kDown = 1.0f / 256.0f;   // of what is held in two parts
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The matrix whose tiles tile number `tile` belongs to, the same in all lanes; list[i].*begin ascends.
__device__ __forceinline__ int matrix_of(const OrthoArgs &a, int64_t OrthoMatrix::*begin, int64_t tile) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.count;
    while (n > 1) {
        const int step = (n + 63) / 64, at = min(lo + lane * step, lo + n - 1);
        const int before = __popcll(__ballot(a.list[at].*begin <= tile && lane * step < n));
        const int from = max(before - 1, 0) * step;
        n = min(step, n - from);
        lo += from;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ float element(const OrthoMatrix &m, int64_t i) {
    return m.dtype == GBT_F32 ? ((const float *)m.src)[i] : m.dtype == GBT_BF16 ? (float)((const __bf16 *)m.src)[i] : (float)((const _Float16 *)m.src)[i];
}
__device__ __forceinline__ void put_element(const OrthoMatrix &m, int64_t i, float x) {
    if (m.dtype == GBT_F32) ((float *)m.dst)[i] = x;
    else if (m.dtype == GBT_BF16) ((__bf16 *)m.dst)[i] = (__bf16)x;
    else ((_Float16 *)m.dst)[i] = (_Float16)x;
}

__device__ __forceinline__ double block_sum(double x, double *part) {   // of 256 threads
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// Squares in 64 bits, where no float's leaves the range.
__global__ __launch_bounds__(256) void ortho_squares_kernel(OrthoArgs a) {
    __shared__ double part[4];
    const OrthoMatrix &m = a.list[matrix_of(a, &OrthoMatrix::piece_begin, blockIdx.x)];
    const int64_t from = (blockIdx.x - m.piece_begin) * kOrthoPiece, to = min(from + kOrthoPiece, (int64_t)m.p * m.w);
    double sum = 0.0;
#pragma unroll 4
    for (int64_t i = from + threadIdx.x; i < to; i += 256) {
        const double x = (double)element(m, i);
        sum = fma(x, x, sum);
    }
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) a.squares[blockIdx.x] = sum;
}

__device__ __forceinline__ void split(float x, _Float16 &high, _Float16 &low) {
    high = (_Float16)x;
    low = (_Float16)(x - (float)high);
}

// X and its transpose in two parts, 64 x 64 elements a workgroup, padding included.
__global__ __launch_bounds__(256) void ortho_fill_kernel(OrthoArgs a) {
    __shared__ double part[4];
    __shared__ float tile[64][65];
    const OrthoMatrix &m = a.list[matrix_of(a, &OrthoMatrix::fill_begin, blockIdx.x)];
    double sum = 0.0;
    for (int i = threadIdx.x; i < m.pieces; i += 256) sum += a.squares[m.piece_begin + i];
    const double norm = sqrt(block_sum(sum, part));
    // a norm of zero leaves zeros; one that is no finite number leaves none anywhere
    const double factor = norm == 0.0 ? 0.0 : isfinite(norm) ? (double)kUp / norm : (double)NAN;
    const int64_t at = blockIdx.x - m.fill_begin;
    const int across = m.ww / 64, i0 = (int)(at / across) * 64, j0 = (int)(at % across) * 64;   // of X
    const int col = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        // rows of memory
        const int i = m.tall ? i0 + col : i0 + r, j = m.tall ? j0 + r : j0 + col;
        float x = 0.0f;
        if (i < m.p && j < m.w) x = (float)((double)element(m, m.tall ? (int64_t)j * m.cols + i : (int64_t)i * m.cols + j) * factor);
        tile[m.tall ? col : r][m.tall ? r : col] = x;
    }
    __syncthreads();
    _Float16 *x = (_Float16 *)(a.workspace + m.x[0]), *xt = (_Float16 *)(a.workspace + m.xt[0]);
    const int64_t plane = (int64_t)m.pp * m.ww;
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        _Float16 high, low;
        split(tile[r][col], high, low);
        const int64_t to = (int64_t)(i0 + r) * m.ww + j0 + col;
        x[to] = high, x[plane + to] = low;
        split(tile[col][r], high, low);
        const int64_t tt = (int64_t)(j0 + r) * m.pp + i0 + col;
        xt[tt] = high, xt[plane + tt] = low;
    }
}

// ---------------------------------------------------------------- products --
// 128 x 128 of P Q^T by four waves of 64 x 64 each: rows of P and Q along the sum, `depth` of them, in two parts each.
typedef Tile<32> Step;   // 64 rows, 32 along the sum
struct Stage {
    alignas(256) char p[2][2][Step::kBytes], q[2][2][Step::kBytes];   // [part][half]
};

__device__ __forceinline__ void fetch_stage(Stage &s, const _Float16 *p, const _Float16 *q, int64_t p_plane, int64_t q_plane, int row, int k, int wave) {
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Step::fetch(s.p[part][half], (const char *)(p + part * p_plane + (int64_t)half * 64 * row + k), (uint32_t)row * 2, 64, 32, wave);
            Step::fetch(s.q[part][half], (const char *)(q + part * q_plane + (int64_t)half * 64 * row + k), (uint32_t)row * 2, 64, 32, wave);
        }
}

__device__ __forceinline__ void product(f32x16 (&acc)[2][2], Stage (&stage)[2], const _Float16 *p, const _Float16 *q, int64_t p_plane, int64_t q_plane,
                                        int row, int depth) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    fetch_stage(stage[0], p, q, p_plane, q_plane, row, 0, wave);
    for (int k = 0; k < depth; k += 32) {
        tiles_ready();
        const Stage &s = stage[(k >> 5) & 1];
        if (k + 32 < depth) fetch_stage(stage[((k >> 5) & 1) ^ 1], p, q, p_plane, q_plane, row, k + 32, wave);
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            f16x8 x[2][2], y[2][2];
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[part][i] = Step::rows<F16>(s.p[part][wave >> 1], 32 * i, step, lane);
                    y[part][i] = Step::rows<F16>(s.q[part][wave & 1], 32 * i, step, lane);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = F16::mma(x[1][i], y[0][j], acc[i][j]);
                    acc[i][j] = F16::mma(x[0][i], y[1][j], acc[i][j]);
                    acc[i][j] = F16::mma(x[0][i], y[0][j], acc[i][j]);
                }
        }
        done_reading();
    }
}

// Tile number `at` of the upper half of n x n tiles: the last column first would be as good; columns j, rows i <= j.
__device__ __forceinline__ void upper_tile(int64_t at, int &i, int &j) {
    j = (int)((sqrt(8.0 * (double)at + 1.0) - 1.0) * 0.5);
    while ((int64_t)(j + 1) * (j + 2) / 2 <= at) ++j;
    while ((int64_t)j * (j + 1) / 2 > at) --j;
    i = (int)(at - (int64_t)j * (j + 1) / 2);
}

// Four values of rows i .. i + 3 of column j, into a matrix in two parts and into its transpose.
__device__ __forceinline__ void put_four(_Float16 *m, int64_t plane, int row, _Float16 *t, int64_t t_plane, int t_row, int i, int j, const float (&v)[4],
                                         bool direct) {
    f16x4 high, low;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        _Float16 h, l;
        split(v[e], h, l);
        high[e] = h, low[e] = l;
        if (direct) {
            const int64_t at = (int64_t)(i + e) * row + j;
            m[at] = h, m[plane + at] = l;
        }
    }
    const int64_t at = (int64_t)j * t_row + i;
    *(f16x4 *)(t + at) = high;
    *(f16x4 *)(t + t_plane + at) = low;
}

__global__ __launch_bounds__(256, 2) void ortho_gram_kernel(OrthoArgs a) {
    __shared__ Stage stage[2];
    const OrthoMatrix &m = a.list[matrix_of(a, &OrthoMatrix::sym_begin, blockIdx.x)];
    int ti, tj;
    upper_tile(blockIdx.x - m.sym_begin, ti, tj);
    const _Float16 *x = (const _Float16 *)(a.workspace + m.x[a.from]);
    const int64_t plane = (int64_t)m.pp * m.ww, to_plane = (int64_t)m.pp * m.pp;
    f32x16 acc[2][2];
    product(acc, stage, x + (int64_t)ti * kOrthoTile * m.ww, x + (int64_t)tj * kOrthoTile * m.ww, plane, plane, m.ww, m.ww);
    _Float16 *to = (_Float16 *)(a.workspace + m.a);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int row = ti * kOrthoTile + (wave >> 1) * 64 + 32 * i + result_row(r, lane >> 5), col = tj * kOrthoTile + (wave & 1) * 64 + 32 * j + (lane & 31);
                const float v[4] = {acc[i][j][r] * kDown, acc[i][j][r + 1] * kDown, acc[i][j][r + 2] * kDown, acc[i][j][r + 3] * kDown};
                put_four(to, to_plane, m.pp, to, to_plane, m.pp, row, col, v, ti != tj);
            }
}

__global__ __launch_bounds__(256, 2) void ortho_factor_kernel(OrthoArgs a) {
    __shared__ Stage stage[2];
    const OrthoMatrix &m = a.list[matrix_of(a, &OrthoMatrix::sym_begin, blockIdx.x)];
    int ti, tj;
    upper_tile(blockIdx.x - m.sym_begin, ti, tj);
    const _Float16 *from = (const _Float16 *)(a.workspace + m.a);
    const int64_t plane = (int64_t)m.pp * m.pp;
    f32x16 acc[2][2];
    product(acc, stage, from + (int64_t)ti * kOrthoTile * m.pp, from + (int64_t)tj * kOrthoTile * m.pp, plane, plane, m.pp, m.pp);
    _Float16 *to = (_Float16 *)(a.workspace + m.b);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int row = ti * kOrthoTile + (wave >> 1) * 64 + 32 * i + result_row(r, lane >> 5), col = tj * kOrthoTile + (wave & 1) * 64 + 32 * j + (lane & 31);
                // A is symmetric: its four values of this column lie side by side in the row of that number
                const f16x4 high = *(const f16x4 *)(from + (int64_t)col * m.pp + row), low = *(const f16x4 *)(from + plane + (int64_t)col * m.pp + row);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = fmaf(a.c * kDown, acc[i][j][r + e], a.b * ((float)high[e] + (float)low[e]));
                    if (row + e == col) v[e] = fmaf(a.a, kUp, v[e]);
                }
                put_four(to, plane, m.pp, to, plane, m.pp, row, col, v, ti != tj);
            }
}

__global__ __launch_bounds__(256, 2) void ortho_apply_kernel(OrthoArgs a) {
    __shared__ Stage stage[2];
    const OrthoMatrix &m = a.list[matrix_of(a, &OrthoMatrix::full_begin, blockIdx.x)];
    const int64_t at = blockIdx.x - m.full_begin;
    const int down = m.pp / kOrthoTile, ti = (int)(at % down), tj = (int)(at / down);
    const _Float16 *b = (const _Float16 *)(a.workspace + m.b), *xt = (const _Float16 *)(a.workspace + m.xt[a.from]);
    const int64_t plane = (int64_t)m.pp * m.ww;
    f32x16 acc[2][2];
    product(acc, stage, b + (int64_t)ti * kOrthoTile * m.pp, xt + (int64_t)tj * kOrthoTile * m.pp, (int64_t)m.pp * m.pp, plane, m.pp, m.pp);
    _Float16 *to = (_Float16 *)(a.workspace + m.x[a.from ^ 1]), *to_t = (_Float16 *)(a.workspace + m.xt[a.from ^ 1]);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float scale = m.scale * kDown;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int row = ti * kOrthoTile + (wave >> 1) * 64 + 32 * i + result_row(r, lane >> 5), col = tj * kOrthoTile + (wave & 1) * 64 + 32 * j + (lane & 31);
                float v[4] = {acc[i][j][r] * kDown, acc[i][j][r + 1] * kDown, acc[i][j][r + 2] * kDown, acc[i][j][r + 3] * kDown};
                if (!a.last) {
                    put_four(to, plane, m.ww, to_t, plane, m.pp, row, col, v, true);
                } else if (col < m.w) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row + e < m.p) put_element(m, m.tall ? (int64_t)col * m.cols + row + e : (int64_t)(row + e) * m.cols + col, v[e] * scale);
                }
            }
}

}  // namespace

hipError_t gbt_launch_ortho_begin(hipStream_t stream, const OrthoArgs &a, int64_t pieces, int64_t fill_tiles) {
    ortho_squares_kernel<<<(unsigned)pieces, 256, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ortho_fill_kernel<<<(unsigned)fill_tiles, 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t gbt_launch_ortho_step(hipStream_t stream, const OrthoArgs &a, int64_t sym_tiles, int64_t full_tiles) {
    ortho_gram_kernel<<<(unsigned)sym_tiles, 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ortho_factor_kernel<<<(unsigned)sym_tiles, 256, 0, stream>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    ortho_apply_kernel<<<(unsigned)full_tiles, 256, 0, stream>>>(a);
    return hipGetLastError();
}
