// Updates of weight matrices, orthogonalised: X = G / |G|, then X <- F X with F = a I + b A + c A^2, A = X X^T, a few times, which takes all singular
// values towards one.
//
// All F and A of one X commute: A after a step is F A F, so two steps can be taken on the p x p matrices alone, and X is multiplied once by the product
// of their factors.  That halves the work where X is wide, and costs nothing where it is square (a step on X is 1.5 w/p + 0.5 products of p x p x p, one on
// A is 2; symmetric ones count half).  But an error of A grows by a^2 with each such step where singular values are small, so X is multiplied and A taken
// anew after one step or two, as many as leave errors like those of 32-bit products (kind_of, gbt_tower.hip).
//
// Steps multiply small singular values, and with them whatever rounding left there, by a^steps (some 500), so sixteen bits do not do for what lies
// between products, and matrix instructions on 32 bits run at a sixteenth of the rate.  Everything between products is held in two float16 parts, high
// and low, 22 bits in all, and a product is three on the matrix units: high * high + high * low + low * high, added up in 32 bits.  Float16 has few exponents, so all
// is held times powers of two that the coefficients give: X has singular values, and so elements, up to a bound that the host knows for each step, and the scale
// takes that bound to 2^15.  Elements down to 2^-17 of it then have their 22 bits (X begins with some 1 / sqrt(p w), 2^-12.5 for 4096 x 8192), smaller
// ones are off by 2^-40 of it: rows and columns of very different size keep theirs.  (512 x 2048, rows of 1 to 1e-4, ten steps: all held times 2^8 3.6e-5 off, as it is 2.4e-6,
// and 32-bit products 7.5e-6; of rows of 1 to 1e-6 the smallest one 1.4e-2 and 1.2e-4 of its length, and 3e-5 to 2e-4.)
//
// All products have both operands' rows along the sum: X X^T, products of symmetric matrices, and F X = F (X^T)^T, for which X's transpose is kept beside it.
// Of symmetric results the upper tiles are computed, and written twice.
#include "ortho.h"
#include "attention.h"

namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A matrix in two parts lies in blocks of 64 rows by 32 columns, a row of blocks after the other, each block's high parts and then its low ones, 4 KB each: a
// tile's step along the sum is then whole 8 KB of memory, copied to LDS as they are, with the places of a row's sixteen-byte pieces as they are read there
// (Tile<32>: piece c at place c ^ fold(row)).
typedef Tile<32> Step;
constexpr int kBlock = 64 * 32, kPair = 2 * kBlock;    // elements of a part, of both
__device__ __forceinline__ int64_t place(int row, int col, int cols) {   // of a high part; its low part is kBlock further
    return ((int64_t)(row >> 6) * (cols >> 5) + (col >> 5)) * kPair + (row & 63) * 32 + ((((col >> 3) & 3) ^ Step::fold(row & 63)) << 3) + (col & 7);
}

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
__device__ __forceinline__ double block_sum(double x, double *part) {   // of 256 threads
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

template <typename E>
struct alignas(16) Vec {
    E x[16 / sizeof(E)];
};
template <typename E>
__device__ __forceinline__ double add_squares(const E *src, int n) {   // by 256 threads, each its own
    constexpr int kVec = 16 / sizeof(E);
    double sum[2] = {0.0, 0.0};
    int i = 0;
    if (((uintptr_t)src & 15) == 0) {
#pragma unroll 4
        for (int at = threadIdx.x; at < n / kVec; at += 256) {
            const Vec<E> v = ((const Vec<E> *)src)[at];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const double x = (double)(float)v.x[e];
                sum[e & 1] = fma(x, x, sum[e & 1]);
            }
        }
        i = n / kVec * kVec;
    }
    for (i += threadIdx.x; i < n; i += 256) {
        const double x = (double)(float)src[i];
        sum[0] = fma(x, x, sum[0]);
    }
    return sum[0] + sum[1];
}

// Squares in 64 bits, where no float's leaves the range.
__global__ __launch_bounds__(256) void ortho_squares_kernel(OrthoArgs a) {
    __shared__ double part[4];
    const OrthoMatrix &m = a.list[matrix_of(a, &OrthoMatrix::piece_begin, blockIdx.x)];
    const int64_t from = (blockIdx.x - m.piece_begin) * kOrthoPiece;
    const int n = (int)min((int64_t)kOrthoPiece, (int64_t)m.p * m.w - from);
    double sum;
    if (m.dtype == GBT_F32) sum = add_squares((const float *)m.src + from, n);
    else if (m.dtype == GBT_BF16) sum = add_squares((const __bf16 *)m.src + from, n);
    else sum = add_squares((const _Float16 *)m.src + from, n);
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) a.squares[blockIdx.x] = sum;
}

__device__ __forceinline__ void split(float x, _Float16 &high, _Float16 &low) {
    high = (_Float16)x;
    low = (_Float16)(x - (float)high);
}

// 64 x 64 elements of G from row r0 and column c0 on, zeros outside, times the factor.
template <typename E>
__device__ __forceinline__ void read_tile(float (&tile)[64][65], const OrthoMatrix &m, int r0, int c0, double factor) {
    const int rows = (m.tall ? m.w : m.p) - r0, cols = (int)m.cols - c0;
    const E *src = (const E *)m.src + (int64_t)r0 * m.cols + c0;
    if (cols >= 64 && m.cols % 8 == 0 && ((uintptr_t)m.src & 15) == 0) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int row = (threadIdx.x >> 3) + 32 * n, piece = (threadIdx.x & 7) * 8;
            Vec<E> v[sizeof(E) / 2] = {};
            if (row < rows)
#pragma unroll
                for (int u = 0; u < (int)sizeof(E) / 2; ++u) v[u] = ((const Vec<E> *)(src + (int64_t)row * m.cols + piece))[u];
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[row][piece + e] = (float)((double)(float)v[e / (16 / sizeof(E))].x[e % (16 / sizeof(E))] * factor);
        }
        return;
    }
    const int col = threadIdx.x & 63;
#pragma unroll 4
    for (int row = threadIdx.x >> 6; row < 64; row += 4)
        tile[row][col] = row < rows && col < cols ? (float)((double)(float)src[(int64_t)row * m.cols + col] * factor) : 0.0f;
}

// X and its transpose in two parts, padding included: 64 rows and 128 columns of X a workgroup.
__global__ __launch_bounds__(256) void ortho_fill_kernel(OrthoArgs a) {
    __shared__ double part[4];
    __shared__ float tile[2][64][65];
    const OrthoMatrix &m = a.list[matrix_of(a, &OrthoMatrix::fill_begin, blockIdx.x)];
    double sum = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < m.pieces; i += 256) sum += a.squares[m.piece_begin + i];
    const double norm = sqrt(block_sum(sum, part));
    // a norm of zero leaves zeros; one that is no finite number leaves none anywhere
    const double factor = norm == 0.0 ? 0.0 : isfinite(norm) ? (double)a.up_x / norm : (double)NAN;
    const int64_t at = blockIdx.x - m.fill_begin;
    const int across = m.ww / 128, i0 = (int)(at / across) * 64, j0 = (int)(at % across) * 128;   // of X
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int j = j0 + 64 * t, r = m.tall ? j : i0, c = m.tall ? i0 : j;
        if (m.dtype == GBT_F32) read_tile<float>(tile[t], m, r, c, factor);
        else if (m.dtype == GBT_BF16) read_tile<__bf16>(tile[t], m, r, c, factor);
        else read_tile<_Float16>(tile[t], m, r, c, factor);
    }
    __syncthreads();
    _Float16 *x = (_Float16 *)(a.workspace + m.x), *xt = (_Float16 *)(a.workspace + m.xt[0]);
#pragma unroll
    for (int n = 0; n < 8; ++n) {   // sixteen-byte pieces of G's tile as it lies, then of its transpose
        const int t = n >> 2, row = (threadIdx.x >> 3) + 32 * (n & 1), piece = (threadIdx.x & 7) * 8;
        const bool along = (n >> 1) & 1;
        f16x8 high, low;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(along ? tile[t][piece + e][row] : tile[t][row][piece + e], h, l);
            high[e] = h, low[e] = l;
        }
        const int j = j0 + 64 * t;
        _Float16 *to = along != (m.tall != 0) ? xt + place(j + row, i0 + piece, m.pp) : x + place(i0 + row, j + piece, m.ww);
        *(f16x8 *)to = high;
        *(f16x8 *)(to + kBlock) = low;
    }
}

// ---------------------------------------------------------------- products --
// 128 x 128 of P Q^T: two rows of blocks of P and of Q, 32 along the sum at a time, in kStages stages of 32 KB of LDS, of which all but one are being loaded.
// Four waves take 64 x 64 each, eight 64 x 32.
struct Stage {
    alignas(256) char p[2][2][Step::kBytes], q[2][2][Step::kBytes];   // [row of blocks][part]
};

// p, q: this wave's part of a pair of blocks; rows of blocks are `row` bytes apart.
template <int kWaves>
__device__ __forceinline__ void fetch_stage(Stage &s, const char *p, const char *q, int64_t row, int wave, uint32_t lane_bytes) {
    const uint32_t to = lds_address(&s) + wave * (8192 / kWaves);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int n = 0; n < 8 / kWaves; ++n) {
            load_to_lds(to + half * 8192 + n * 1024, p + half * row + n * 1024, lane_bytes);
            load_to_lds(to + 16384 + half * 8192 + n * 1024, q + half * row + n * 1024, lane_bytes);
        }
}

// Sums of many products are added up in pieces of 128, so that roundings are those of few and small sums: an instruction's own is off by 0.4 units of its sum's last place (root
// mean square; one to the nearest by 0.29), and there are three for every 16 products.  (777 x 1001 in float32: pieces of 512 3.2e-6 off, of 128 2.2e-6, of 64 1.9e-6, and
// 32-bit products 2.4e-6; 4096 x 4096 5.2e-6, 3.4e-6, 3.4e-6 and 8.4e-6.  4096 x 4096, 4096 x 8192 and two of 1024 x 4096 take 10.6, 10.8 and 11.0 ms.)
constexpr int kPiece = 4;   // steps

// A wave's operands of sixteen steps along the sum: [part][row or column of 32].
template <int kWaves>
struct Operands {
    static constexpr int kAcross = 8 / kWaves;
    f16x8 x[2][2], y[2][kAcross];
    __device__ __forceinline__ void read(const Stage &s, int step, int wave, int lane) {
        const int down = kWaves == 4 ? wave >> 1 : wave >> 2, across = kWaves == 4 ? wave & 1 : (wave & 3) >> 1, first = kWaves == 4 ? 0 : 32 * (wave & 1);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
#pragma unroll
            for (int i = 0; i < 2; ++i) x[part][i] = Step::rows<F16>(s.p[down][part], 32 * i, step, lane);
#pragma unroll
            for (int j = 0; j < kAcross; ++j) y[part][j] = Step::rows<F16>(s.q[across][part], first + 32 * j, step, lane);
        }
    }
    // low * low where that is wanted, low * high, high * low, high * high: the sums in turn, so that none waits for itself
    template <bool kLow>
    __device__ __forceinline__ void add(f32x16 (&acc)[2][kAcross]) const {
#pragma unroll
        for (int of = kLow ? -1 : 0; of < 3; ++of)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < kAcross; ++j) acc[i][j] = F16::mma(x[of <= 0][i], y[of == 1 || of < 0][j], acc[i][j]);
    }
};
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }   // what is before it is issued before what is behind it

// While the matrix units work on one half of a step, the operands of the next half are read, also from the next step, behind the barrier.
template <bool kLow, int kWaves, int kStages>
__device__ __forceinline__ void product(f32x16 (&sum)[2][8 / kWaves], Stage *stages, const char *p, const char *q, int64_t row, int steps, int wave, int lane) {
    constexpr int kAcross = 8 / kWaves, kLoads = 4 * (8 / kWaves);   // of a stage, by each wave
    f32x16 acc[2][kAcross] = {};
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        if (s < steps) fetch_stage<kWaves>(stages[s], p + s * (kPair * 2), q + s * (kPair * 2), row, wave, lane * 16);
    Operands<kWaves> even, odd;
    int now = 0;
    for (int k = 0; k < steps; ++k) {
        // this step's loads are done, those of the steps behind it under way; and all waves are done with the step before
        if (k + kStages - 1 <= steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads * (kStages - 2)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const int next = k + kStages - 1, at = now == 0 ? kStages - 1 : now - 1;
        even.read(stages[now], 0, wave, lane);
        in_order();
        if (next < steps) fetch_stage<kWaves>(stages[at], p + (int64_t)next * (kPair * 2), q + (int64_t)next * (kPair * 2), row, wave, lane * 16);
        if (k > 0) {
            odd.template add<kLow>(acc);
            if ((k & (kPiece - 1)) == 0) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < kAcross; ++j) {
                        sum[i][j] += acc[i][j];
                        acc[i][j] = f32x16{};
                    }
            }
        }
        in_order();
        odd.read(stages[now], 1, wave, lane);
        in_order();
        even.template add<kLow>(acc);
        in_order();
        now = now + 1 == kStages ? 0 : now + 1;
    }
    odd.template add<kLow>(acc);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < kAcross; ++j) sum[i][j] += acc[i][j];
}

// Sixteen-bit values of four rows in the column of each of four lanes, and back: the lane's own row's values of the four columns.
struct Exchange {
    int quad;
    uint32_t sel0, sel1, keep, give;
    __device__ Exchange(int lane) {
        quad = lane & 3;
        // bytes 0 to 3 are of what the lane keeps (its column, and that of two lanes on), 4 to 7 of what it is given
        const bool odd = quad & 1, high = quad & 2;
        sel0 = odd ? (high ? 0x03020706u : 0x01000504u) : (high ? 0x07060302u : 0x05040100u);
        sel1 = odd ? (high ? 0x01000504u : 0x03020706u) : (high ? 0x05040100u : 0x07060302u);
        keep = odd ? 0x07060302u : 0x05040100u;   // of (other, mine): both high halves, or both low ones
        give = odd ? 0x05040100u : 0x07060302u;
    }
    __device__ f16x4 operator()(f16x4 v) const {
        const uint64_t both = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)both, hi = (uint32_t)(both >> 32), mine = quad & 2 ? hi : lo, theirs = quad & 2 ? lo : hi;
        const uint32_t other = __builtin_amdgcn_mov_dpp(theirs, 0x4e, 0xf, 0xf, true);   // of the lane two on
        const uint32_t kept = __builtin_amdgcn_perm(other, mine, keep);
        const uint32_t given = __builtin_amdgcn_mov_dpp(__builtin_amdgcn_perm(other, mine, give), 0xb1, 0xf, 0xf, true);   // of the neighbour
        return __builtin_bit_cast(f16x4, (uint64_t)__builtin_amdgcn_perm(given, kept, sel1) << 32 | __builtin_amdgcn_perm(given, kept, sel0));
    }
};

// Four values of rows i .. i + 3 of column j into a matrix's transpose and, if `direct`, into the matrix.
__device__ __forceinline__ void put_four(_Float16 *m, int cols, _Float16 *t, int t_cols, int i, int j, const float (&v)[4], bool direct, const Exchange &swap) {
    f16x4 high, low;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        _Float16 h, l;
        split(v[e], h, l);
        high[e] = h, low[e] = l;
    }
    _Float16 *to = t + place(j, i, t_cols);
    *(f16x4 *)to = high;
    *(f16x4 *)(to + kBlock) = low;
    if (direct) {
        to = m + place(i + swap.quad, j & ~3, cols);
        *(f16x4 *)to = swap(high);
        *(f16x4 *)(to + kBlock) = swap(low);
    }
}

// A wave's sums, rows of 32 from `row0` and columns of 32 from `col0` on, times `less` and the matrix's scale into G's place.  Four rows' values of a column lie side by side in a G with more
// rows; in another one they are exchanged where they have sixteen bits, so that a lane writes four columns of its row.  (One element at a time, its type looked up for
// each: 157 us in place of 82 for the last product of 6 x 512 x 512, 6 x 1536, 12 x 2048 and 2 x 777 x 1001.)
template <typename E, int kAcross>
__device__ __forceinline__ void put_result(const OrthoMatrix &m, const f32x16 (&acc)[2][kAcross], int row0, int col0, float less, int lane, const Exchange &swap) {
    struct alignas(4 * sizeof(E)) Quad {
        E x[4];
    };
    E *dst = (E *)m.dst;
    const float scale = m.scale;
    const int64_t cols = m.cols;
    const int p = m.p, w = m.w;
    const bool tall = m.tall, quads = cols % 4 == 0 && ((uintptr_t)dst & (4 * sizeof(E) - 1)) == 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < kAcross; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int row = row0 + 32 * i + result_row(r, lane >> 5), col = col0 + 32 * j + (lane & 31);
                Quad v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v.x[e] = (E)(acc[i][j][r + e] * less * scale);
                if (tall) {
                    E *to = dst + (int64_t)col * cols + row;
                    if (col < w && quads) {
                        if (row < p) *(Quad *)to = v;   // p is a multiple of four too
                    } else if (col < w) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (row + e < p) to[e] = v.x[e];
                    }
                } else if (sizeof(E) == 2 && quads) {   // so is w, and four lanes lie inside or outside together
                    if constexpr (sizeof(E) == 2) {
                        const f16x4 x = swap(__builtin_bit_cast(f16x4, v));
                        if (row + swap.quad < p && col < w) *(f16x4 *)(dst + (int64_t)(row + swap.quad) * cols + (col & ~3)) = x;
                    }
                } else if (col < w) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row + e < p) dst[(int64_t)(row + e) * cols + col] = v.x[e];
                }
            }
}

template <int kProduct, int kWaves, int kStages>
__global__ __launch_bounds__(64 * kWaves, 2) void ortho_product_kernel(OrthoArgs a) {
    extern __shared__ __attribute__((aligned(256))) char lds[];
    constexpr bool kApply = kProduct == kOrthoApply;
    const OrthoTile tile = a.tiles[blockIdx.x];
    if (tile.matrix < 0) return;
    const OrthoMatrix &m = a.list[tile.matrix];
    const int ti = tile.i, tj = tile.j;
    auto at = [&](int64_t offset) { return (_Float16 *)(a.workspace + offset); };
    const _Float16 *p = at(kProduct == kOrthoGram ? m.x : kProduct == kOrthoFactor ? m.gram : kProduct == kOrthoBetween ? m.factor[0] : kProduct == kOrthoNext ? m.between
                           : kProduct == kOrthoTotal ? m.factor[1] : a.step == 0 ? m.factor[0] : m.total);
    const _Float16 *q = at(kProduct == kOrthoGram ? m.x : kProduct == kOrthoFactor || kProduct == kOrthoBetween ? m.gram : kApply ? m.xt[a.xt] : m.factor[0]);
    _Float16 *to = at(kProduct == kOrthoGram || kProduct == kOrthoNext ? m.gram : kProduct == kOrthoFactor ? m.factor[a.step] : kProduct == kOrthoBetween ? m.between
                      : kProduct == kOrthoTotal ? m.total : m.x);
    _Float16 *to_t = kApply ? at(m.xt[a.xt ^ 1]) : to;
    const int depth = kProduct == kOrthoGram ? m.ww : m.pp, cols = kApply ? m.ww : m.pp;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), steps = depth / 32;
    const int64_t row_bytes = (int64_t)steps * kPair * 2;
    f32x16 acc[2][8 / kWaves] = {};
    const char *p_rows = (const char *)p + (int64_t)ti * 2 * row_bytes + wave * (8192 / kWaves);
    const char *q_rows = (const char *)q + (int64_t)tj * 2 * row_bytes + wave * (8192 / kWaves);
    // What is left out of X X^T and A A with low * low is never negative on their diagonals, 2^-24.4 of them, and the factor's elements there are small differences of larger ones.  Of a
    // few long rows, which are nearly orthogonal, that is most of the error; where there are more it is not seen.  (2000 x 30 1.8e-6 off without, 1.4e-6 with, 32-bit products
    // 1.2e-6; 689 x 15 1.7e-6, 1.25e-6, 1.24e-6; 300 x 300 1.4e-6 either way.  With it in all products, 4096 x 4096, 4096 x 8192 and two of 1024 x 4096 take 12.4 in place of 10.6 ms.)
    if ((kProduct == kOrthoFactor || kProduct == kOrthoGram) && m.pp == kOrthoTile) product<true, kWaves, kStages>(acc, (Stage *)lds, p_rows, q_rows, row_bytes, steps, wave, lane);
    else product<false, kWaves, kStages>(acc, (Stage *)lds, p_rows, q_rows, row_bytes, steps, wave, lane);
    const int first_row = ti * kOrthoTile + (kWaves == 4 ? wave >> 1 : wave >> 2) * 64, first_col = tj * kOrthoTile + (kWaves == 4 ? (wave & 1) * 64 : (wave & 3) * 32);
    const Exchange swap(lane);
    if (kApply && a.last) {
        if (m.dtype == GBT_F32) put_result<float>(m, acc, first_row, first_col, a.less, lane, swap);
        else if (m.dtype == GBT_BF16) put_result<__bf16>(m, acc, first_row, first_col, a.less, lane, swap);
        else put_result<_Float16>(m, acc, first_row, first_col, a.less, lane, swap);
        return;
    }
    const float less = a.less, to_factor = a.up_factor / a.up_gram;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        // A is symmetric: its four values of a lane's column lie side by side in the row of that number.  All are read before anything is written.
        f16x4 high[8 / kWaves][4], low[8 / kWaves][4];
        if (kProduct == kOrthoFactor)
#pragma unroll
            for (int j = 0; j < 8 / kWaves; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const _Float16 *from = p + place(first_col + 32 * j + (lane & 31), first_row + 32 * i + result_row(4 * r, lane >> 5), m.pp);
                    high[j][r] = *(const f16x4 *)from, low[j][r] = *(const f16x4 *)(from + kBlock);
                }
#pragma unroll
        for (int j = 0; j < 8 / kWaves; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int row = first_row + 32 * i + result_row(r, lane >> 5), col = first_col + 32 * j + (lane & 31);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][r + e] * less;
                if (kProduct == kOrthoFactor) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float with_a = row + e == col ? a.a * a.up_gram : 0.0f;
                        v[e] = fmaf(a.c, v[e], fmaf(a.b, (float)high[j][r / 4][e] + (float)low[j][r / 4][e], with_a)) * to_factor;
                    }
                }
                put_four(to, cols, to_t, m.pp, row, col, v, kApply || ti != tj, swap);
            }
    }
}

// ------------------------------------------------------------------- small --
// A small matrix by one workgroup, all of it in LDS: X in blocks of 64 rows by 32 columns, and three p x p matrices of two blocks each, four waves a quarter
// of a product each.  A result goes back over an operand once all waves have it.  B operands that run along columns of X are read transposed, in the order
// of the sum that such reads give (attention.h), and those they meet in the same order.  What bounds it is how steps wait for one another, and the fetching of
// code that runs but once: all products of p x p are one loop (40 KB of code 52 us for 64 x 256 in five steps, the loop 34).
struct Small {
    char *gram, *factor, *total, *x;
    int wave, lane;
};
// One wave has nothing but this to do, so its three kinds of products are three sums, that none waits for another.  `low`: low * low too, for A A.
__device__ __forceinline__ void small_product(f32x16 &acc, const Small &s, const char *p, const char *q, int blocks, bool low) {
    f32x16 sum[3] = {};
    for (int b = 0; b < blocks; b += 2) {
        f16x8 x[4][2], y[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const int at = min(b + (k >> 1), blocks - 1) * 8192 + part * 4096;
                x[k][part] = Step::rows<F16>(p + at, 32 * (s.wave >> 1), k & 1, s.lane);
                y[k][part] = Step::rows<F16>(q + at, 32 * (s.wave & 1), k & 1, s.lane);
            }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (b + (k >> 1) < blocks) {
                if (low) sum[2] = F16::mma(x[k][1], y[k][1], sum[2]);
                sum[0] = F16::mma(x[k][1], y[k][0], sum[0]);
                sum[1] = F16::mma(x[k][0], y[k][1], sum[1]);
                sum[2] = F16::mma(x[k][0], y[k][0], sum[2]);
            }
    }
    acc = (sum[0] + sum[1]) + sum[2];
}
// Byte offset of row `col`, elements row .. row + 3 of a symmetric p x p matrix: where a lane's four values belong.
__device__ __forceinline__ int small_four(const Small &s, int r) {
    const int row = 32 * (s.wave >> 1) + result_row(r, s.lane >> 5), col = 32 * (s.wave & 1) + (s.lane & 31);
    return (int)place(col, row, 64) * 2;
}
__device__ __forceinline__ void small_put(char *to, const float (&v)[4]) {
    f16x4 high, low;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        _Float16 h, l;
        split(v[e], h, l);
        high[e] = h, low[e] = l;
    }
    *(f16x4 *)to = high;
    *(f16x4 *)(to + kBlock * 2) = low;
}
// X into its blocks, divided by its norm, by pieces of eight elements, neighbours in memory by neighbouring lanes.  All of G is under way at once and in
// registers until the norm is known.
template <typename E>
__device__ __forceinline__ void small_read(const Small &s, const OrthoMatrix &m, int blocks, float up, double *part) {
    constexpr int kPieces = 64 * kOrthoSmallW / 8 / 256;
    const E *src = (const E *)m.src;
    const int cols = (int)m.cols, across = blocks * 4, pieces = 64 * across;
    const bool wide = !m.tall && cols % 8 == 0 && ((uintptr_t)src & 15) == 0;
    float x[kPieces][8];
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
        const int at = threadIdx.x + 256 * n, i = m.tall ? at & 63 : at / across, j = (m.tall ? at >> 6 : at - at / across * across) * 8;
        if (at >= pieces || i >= m.p) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[n][e] = 0.0f;
        } else if (wide) {
            Vec<E> v[sizeof(E) / 2] = {};
            if (j < cols)
#pragma unroll
                for (int u = 0; u < (int)sizeof(E) / 2; ++u) v[u] = ((const Vec<E> *)(src + i * cols + j))[u];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[n][e] = (float)v[e / (16 / sizeof(E))].x[e % (16 / sizeof(E))];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[n][e] = j + e < m.w ? (float)src[m.tall ? (j + e) * cols + i : i * cols + j + e] : 0.0f;
        }
    }
    double sum[2] = {0.0, 0.0};
#pragma unroll
    for (int n = 0; n < kPieces; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e & 1] = fma((double)x[n][e], (double)x[n][e], sum[e & 1]);
    const double norm = sqrt(block_sum(sum[0] + sum[1], part));
    // a norm of zero leaves zeros; one that is no finite number leaves none anywhere
    const double factor = norm == 0.0 ? 0.0 : isfinite(norm) ? (double)up / norm : (double)NAN;
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
        const int at = threadIdx.x + 256 * n, i = m.tall ? at & 63 : at / across, j = (m.tall ? at >> 6 : at - at / across * across) * 8;
        if (at >= pieces) break;
        f16x8 high, low;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split((float)((double)x[n][e] * factor), h, l);
            high[e] = h, low[e] = l;
        }
        char *to = s.x + place(i, j, blocks * 32) * 2;
        *(f16x8 *)to = high;
        *(f16x8 *)(to + kBlock * 2) = low;
    }
}
// A block's half of the result, rows 32 * i on, to G's place.
template <typename E>
__device__ __forceinline__ void small_result(const Small &s, const OrthoMatrix &m, const f32x16 &z, int i, int col, float less) {
    E *dst = (E *)m.dst;
    const float scale = m.scale;
    const int across = m.tall ? 1 : (int)m.cols, along = m.tall ? (int)m.cols : 1, first = 32 * i + 4 * (s.lane >> 5);
    if (col >= m.w) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = first + result_row(r, 0);
        if (row < m.p) dst[row * across + col * along] = (E)(z[r] * less * scale);
    }
}

__global__ __launch_bounds__(256) void ortho_small_kernel(OrthoArgs a, OrthoSmallScales scales, int steps, int together) {
    extern __shared__ __attribute__((aligned(256))) char lds[];
    __shared__ double part[4];
    __shared__ OrthoSmallScales up;   // arguments lie in the host's memory: read once, while G is under way
    static_assert(sizeof up.step == 1024, "");
    ((float *)up.step)[threadIdx.x] = ((const float *)scales.step)[threadIdx.x];
    const OrthoMatrix &m = a.list[blockIdx.x];
    const int blocks = (m.w + 31) / 32;
    Small s;
    s.gram = lds, s.factor = lds + 16384, s.total = lds + 32768, s.x = lds + 49152;
    s.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), s.lane = threadIdx.x & 63;
    if (m.dtype == GBT_F32) small_read<float>(s, m, blocks, scales.x, part);
    else if (m.dtype == GBT_BF16) small_read<__bf16>(s, m, blocks, scales.x, part);
    else small_read<_Float16>(s, m, blocks, scales.x, part);
    __syncthreads();
    const Exchange swap(s.lane);
    for (int done = 0; done < steps; done += together) {
        const int now = min(together, steps - done);
        // A; then for every step its factor F (the first begins their product), the product of the factors, F A, and A of the next step, (F A) F
#pragma unroll 1
        for (int op = -1; op < 4 * now; ++op) {
            const int i = op >> 2, kind = op < 0 ? -1 : op & 3;
            if ((kind == 1 && i == 0) || (kind > 1 && i == now - 1)) continue;
            char *f = i == 0 ? s.total : s.factor;
            const char *p = kind < 0 ? s.x : kind == 0 || kind == 3 ? s.gram : f, *q = kind < 0 ? s.x : kind == 1 ? s.total : kind == 3 ? f : s.gram;
            char *to = kind == 0 ? f : kind == 1 ? s.total : s.gram;
            f32x16 acc;
            small_product(acc, s, p, q, kind < 0 ? blocks : 2, kind == 0);
            const OrthoSmallScales::Step &scale = up.step[done + max(i, 0)];
            const float up_gram = scale.gram, to_factor = scale.factor, less = kind < 0 ? kScaleDown : scale.less[max(kind, 0)];
            if (kind > 0) __syncthreads();   // it goes over an operand
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int at = small_four(s, r), row = 32 * (s.wave >> 1) + result_row(r, s.lane >> 5), col = 32 * (s.wave & 1) + (s.lane & 31);
                float v[4] = {acc[r] * less, acc[r + 1] * less, acc[r + 2] * less, acc[r + 3] * less};
                if (kind == 0) {
                    const f16x4 high = *(const f16x4 *)(s.gram + at), low = *(const f16x4 *)(s.gram + at + kBlock * 2);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float with_a = row + e == col ? a.a * up_gram : 0.0f;
                        v[e] = fmaf(a.c, v[e], fmaf(a.b, (float)high[e] + (float)low[e], with_a)) * to_factor;
                    }
                }
                small_put(to + at, v);
            }
            __syncthreads();
        }
        // X, a block of 32 columns by a wave, in place
        const bool last = done + now == steps;
        const float less = up.step[done].apply;
        for (int b = s.wave; b < blocks; b += 4) {
            char *block = s.x + b * 8192;
            f16x8 y[2][4];
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int k = 0; k < 4; ++k) y[part][k] = Step::cols<F16>(block + part * 4096, 16 * k, 0, s.lane);
#pragma unroll 1
            for (int i = 0; i < 2; ++i) {
                const int of = s.lane & 31, half = s.lane >> 5;
                f32x16 z[3] = {};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    f16x8 x[2];
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const char *row = s.total + (k >> 1) * 8192 + part * 4096 + (32 * i + of) * 64 + 8 * half;
                        const f16x4 lo = *(const f16x4 *)(row + (((2 * (k & 1)) ^ Step::fold(of)) << 4)), hi = *(const f16x4 *)(row + (((2 * (k & 1) + 1) ^ Step::fold(of)) << 4));
                        x[part] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    }
                    z[0] = F16::mma(x[1], y[0][k], z[0]);
                    z[1] = F16::mma(x[0], y[1][k], z[1]);
                    z[2] = F16::mma(x[0], y[0][k], z[2]);
                }
                z[0] = (z[0] + z[1]) + z[2];
                if (last) {
                    if (m.dtype == GBT_F32) small_result<float>(s, m, z[0], i, 32 * b + of, less);
                    else if (m.dtype == GBT_BF16) small_result<__bf16>(s, m, z[0], i, 32 * b + of, less);
                    else small_result<_Float16>(s, m, z[0], i, 32 * b + of, less);
                    continue;
                }
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int row = 32 * i + result_row(r, half);
                    f16x4 high, low;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        _Float16 h, l;
                        split(z[0][r + e] * less, h, l);
                        high[e] = h, low[e] = l;
                    }
                    char *to = block + place(row + swap.quad, of & ~3, 32) * 2;
                    *(f16x4 *)to = swap(high);
                    *(f16x4 *)(to + kBlock * 2) = swap(low);
                }
            }
        }
        __syncthreads();
    }
}

template <int kProduct, int kWaves, int kStages>
hipError_t launch_form(hipStream_t stream, const OrthoArgs &a, int64_t tiles) {
    constexpr int kLds = kStages * (int)sizeof(Stage);
    static const hipError_t ready =
        hipFuncSetAttribute((const void *)ortho_product_kernel<kProduct, kWaves, kStages>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (ready != hipSuccess) return ready;
    ortho_product_kernel<kProduct, kWaves, kStages><<<(unsigned)tiles, 64 * kWaves, kLds, stream>>>(a);
    return hipGetLastError();
}
// Many tiles: two workgroups on a compute unit, with two stages each; few: one with all of the LDS, as the loads' latency is what counts.  (us of five steps on matrices of
// bfloat16, two workgroups everywhere and one: one of 512 x 512, 10 tiles of symmetric products and 16 of F X, 332 and 283; 24, 240 and 384, 478 and 465; 64, 640 and
// 1024, 1164 and 1201.  Between one and two tiles a compute unit it goes by how they lie: 32 of 512 x 512, 320 and 512, 616 and 693; 12 of 1024 x 1024, 432 and 768,
// 1178 and 1324; but with two from one tile a compute unit on, 26 matrices of seven sizes, 296 symmetric tiles, 889 in place of 845.)
template <int kProduct>
hipError_t launch(hipStream_t stream, const OrthoArgs &a, int64_t tiles, int num_cu) {
    return tiles <= 2 * num_cu ? launch_form<kProduct, 8, 5>(stream, a, tiles) : launch_form<kProduct, 4, 2>(stream, a, tiles);
}

}  // namespace

hipError_t gbt_launch_ortho_begin(hipStream_t stream, const OrthoArgs &a, int64_t pieces, int64_t fill_tiles) {
    ortho_squares_kernel<<<(unsigned)pieces, 256, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ortho_fill_kernel<<<(unsigned)fill_tiles, 256, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t gbt_launch_ortho_small(hipStream_t stream, const OrthoArgs &a, const OrthoSmallScales &up, int steps, int together) {
    static const hipError_t ready = hipFuncSetAttribute((const void *)ortho_small_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kOrthoSmallLds);
    if (ready != hipSuccess) return ready;
    ortho_small_kernel<<<a.count, 256, kOrthoSmallLds, stream>>>(a, up, steps, together);
    return hipGetLastError();
}

hipError_t gbt_launch_ortho_product(hipStream_t stream, const OrthoArgs &a, OrthoProduct product, int num_cu) {
    const int64_t tiles = a.count_tiles;
    switch (product) {
        case kOrthoGram: return launch<kOrthoGram>(stream, a, tiles, num_cu);
        case kOrthoFactor: return launch<kOrthoFactor>(stream, a, tiles, num_cu);
        case kOrthoBetween: return launch<kOrthoBetween>(stream, a, tiles, num_cu);
        case kOrthoTotal: return launch<kOrthoTotal>(stream, a, tiles, num_cu);
        case kOrthoNext: return launch<kOrthoNext>(stream, a, tiles, num_cu);
        default: return launch<kOrthoApply>(stream, a, tiles, num_cu);
    }
}
