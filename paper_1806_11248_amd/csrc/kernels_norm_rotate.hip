// The norm of every head's queries and keys, their rotation by position, and the way of keys and values into a store, in one pass; and the backward pass.
//
// x a head of dim elements: s = 1 / sqrt(mean x^2 + eps), y = x * s * weight, and each pair (a, b) of y's first `turned` elements is turned by
// position * turns revolutions.  Backward, of a gradient d: g is d turned back, u = g * weight, dx = s * (u - x * s^2 * mean(x * u)), and the weights'
// gradient is the sum of g * x * s over rows and heads.  A lane holds eight elements of a head, four pairs or both halves' four elements of them, so a
// pair never lies in two lanes; what lanes share is two sums.  Angles are taken in 64 bits, in revolutions, of which only the fraction goes on to the sine
// in 32.  Bound: memory.
#include "norm_rotate.h"

#include <type_traits>

namespace {

template <typename E>
struct alignas(8) Four {
    E x[4];
};

struct Place {
    int64_t store;       // the row of k_out and v_out, -1: none
    int64_t position;
    bool there;          // a row of a sequence
};

// Which sequence a row belongs to, for sequences in the order of their rows.  The whole wave looks for one row: 64 pointers at a time.
__device__ __forceinline__ int sequence_of(const int64_t *ptr, int n_seq, int64_t row) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = n_seq;   // the last of ptr[lo .. lo + n - 1] that is at most the row
    while (n > 1) {
        const int step = (n + 63) / 64, at = min(lo + lane * step, lo + n - 1);
        const int before = __popcll(__ballot(ptr[at] <= row && lane * step < n));
        const int from = max(before - 1, 0) * step;
        n = min(step, n - from);
        lo += from;
    }
    return lo;
}

__device__ __forceinline__ Place place_of(const RotateArgs &a, int64_t row, int seq) {
    Place p;
    int64_t q0, q1;
    if (a.n_seq == 0) {
        p.store = a.store ? -1 : row, p.position = 0, p.there = false;
        return p;
    }
    if (a.q_ptr) {
        q0 = a.q_ptr[seq], q1 = a.q_ptr[seq + 1];
    } else {
        const int64_t each = a.rows / a.n_seq;
        q0 = seq * each, q1 = q0 + each;
    }
    p.there = q0 >= 0 && q1 <= a.rows && row >= q0 && row < q1;
    int64_t at = row - q0, slot = 0, room = 0;
    if (a.slots) {
        int64_t k0, k1;
        if (a.k_ptr) {
            k0 = a.k_ptr[seq], k1 = a.k_ptr[seq + 1];
        } else {
            const int64_t each = a.store ? a.out_rows / a.n_seq : INT32_MAX;
            k0 = a.store ? seq * each : 0, k1 = k0 + each;
        }
        int64_t used = k1 - k0;
        if (a.k_len) used = min(used, (int64_t)a.k_len[seq]);
        if (k0 < 0 || used < 0 || (a.store && k0 + used > a.out_rows)) used = 0;
        at += used - (q1 - q0);
        slot = k0, room = used;
    }
    p.position = at;
    p.store = !a.store ? row : p.there && at >= 0 && at < room ? slot + at : -1;
    if (a.positions) p.position = a.position_bytes == 4 ? (int64_t)((const int32_t *)a.positions)[row] : ((const int64_t *)a.positions)[row];
    return p;
}

// Where a lane's two fours of a head begin, and whether they are turned: as four neighbouring pairs, or as the halves of four.
struct Part {
    int lo, hi;
    bool turned, works;
    int pair;   // of the first of the four pairs
    __device__ Part(const RotateArgs &a, int lane) {
        works = lane < a.dim / 8;
        turned = works && lane < a.turned / 8;
        pair = turned ? 4 * lane : 0;
        lo = a.halves && turned ? 4 * lane : 8 * lane;
        hi = a.halves && turned ? a.turned / 2 + 4 * lane : 8 * lane + 4;
    }
    __device__ int element(int e) const { return e < 4 ? lo + e : hi + e - 4; }   // of the lane's e-th
};

template <typename E>
struct Raw {   // a lane's eight elements as they lie in memory
    Four<E> lo, hi;
    __device__ void read(const char *row, const Part &p) { lo = *(const Four<E> *)(row + p.lo * 2), hi = *(const Four<E> *)(row + p.hi * 2); }
    __device__ void to(float (&x)[8], bool some) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = some ? (float)lo.x[e] : 0.0f, x[4 + e] = some ? (float)hi.x[e] : 0.0f;
    }
};
template <typename E>
__device__ __forceinline__ void write_parts(char *row, const float (&x)[8], const Part &p) {
    Four<E> lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) lo.x[e] = (E)x[e], hi.x[e] = (E)x[4 + e];
    *(Four<E> *)(row + p.lo * 2) = lo;
    *(Four<E> *)(row + p.hi * 2) = hi;
}

struct Turn {
    float cos[4], sin[4];
    __device__ void set(const RotateArgs &a, const Part &p, const double (&turns)[4], int64_t position) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double whole = (double)position * turns[i];
            const float part = (float)(whole - rint(whole));   // in -1/2 .. 1/2 revolutions
            cos[i] = p.turned ? __builtin_amdgcn_cosf(part) : 1.0f;
            sin[i] = p.turned ? __builtin_amdgcn_sinf(part) : 0.0f;
        }
    }
    // Pairs are (0, 4), (1, 5) .. of the eight as halves, (0, 1), (2, 3) .. as neighbours; sign -1: back.
    __device__ void apply(float (&x)[8], bool halves, float sign) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float &a = halves ? x[i] : x[2 * i], &b = halves ? x[4 + i] : x[2 * i + 1];
            const float s = sign * sin[i], was = a;
            a = fmaf(was, cos[i], -b * s);
            b = fmaf(was, s, b * cos[i]);
        }
    }
};

template <int LOG>
__device__ __forceinline__ float line_sum(float x) {
#pragma unroll
    for (int s = 0; s < LOG; ++s) x += __shfl_xor(x, 1 << s);
    return x;
}

// A wave's rows, and its lanes' places among them: lines of 1 << LOG lanes, of one row or of a few whole ones side by side.
template <int LOG>
struct Lines {
    static constexpr int kAtOnce = 64 >> LOG;
    int lane, sub, row_off, first;   // of the line; which of the wave's lines; its row; its line there in the first pass
    __device__ Lines(const RotateArgs &a) {
        lane = threadIdx.x & ((1 << LOG) - 1);
        sub = (threadIdx.x & 63) >> LOG;
        row_off = a.row_group > 1 ? sub / a.lines : 0;
        first = a.row_group > 1 ? (row_off < a.row_group ? sub % a.lines : a.lines) : sub;
    }
};

__device__ __forceinline__ Place my_place(const RotateArgs &a, int64_t row0, int row_off) {
    const int64_t row = min(row0 + row_off, a.rows - 1);
    int seq = 0;
    if (a.n_seq == 0) {
    } else if (a.q_ptr) {
        seq = sequence_of(a.q_ptr, a.n_seq, row0);
        if (a.row_group > 1)
            for (int n = a.n_seq - seq; n > 1;) {
                const bool behind = a.q_ptr[seq + n / 2] <= row;
                seq += behind ? n / 2 : 0;
                n = behind ? n - n / 2 : n / 2;
            }
    } else {
        seq = (int)min(row / max((int64_t)1, a.rows / a.n_seq), (int64_t)a.n_seq - 1);
    }
    return place_of(a, row, seq);
}

// What a lane keeps for all its rows.
template <int LOG>
struct Fixed {
    Lines<LOG> lines;
    Part part;
    double turns[4];
    float wq[8], wk[8];
    __device__ Fixed(const RotateArgs &a) : lines(a), part(a, lines.lane) {
#pragma unroll
        for (int i = 0; i < 4; ++i) turns[i] = part.turned ? a.turns[part.pair + i] : 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            wq[e] = part.works && a.q_weight ? a.q_weight[part.element(e)] : 1.0f;
            wk[e] = part.works && a.k_weight ? a.k_weight[part.element(e)] : 1.0f;
        }
    }
};
// Which head of what a line is.
struct Line {
    bool is_q, is_v;
    int head;
    __device__ Line(const RotateArgs &a, int line) {
        is_q = line < a.heads, is_v = line >= a.heads + a.kv_heads;
        head = line - (is_q ? 0 : is_v ? a.heads + a.kv_heads : a.heads);
    }
};
__device__ __forceinline__ int64_t bytes_to(const AttnView &x, int64_t row, int head) { return (row * x.row + head * x.head) * 2; }

template <typename E, bool kHalves, int LOG>
__global__ __launch_bounds__(256) void norm_rotate_kernel(RotateArgs a) {
    constexpr int kAhead = 4;   // lines under way
    const Fixed<LOG> f(a);
    const float each = 1.0f / a.dim;
    const int64_t items = (a.rows + a.row_group - 1) / a.row_group * a.parts;
    const int passes = (a.passes + a.parts - 1) / a.parts;
    for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
        const int64_t row0 = item / a.parts * a.row_group, row = row0 + f.lines.row_off;
        const bool mine = f.part.works && row < a.rows;
        const int from = (int)(item % a.parts) * passes, to = min(a.passes, from + passes);
        Place place;
        Turn turn;
        for (int pass0 = from; pass0 < to; pass0 += kAhead) {
            Raw<E> raw[kAhead];
#pragma unroll
            for (int b = 0; b < kAhead; ++b) {
                const int line = f.lines.first + (pass0 + b) * Lines<LOG>::kAtOnce;
                const Line l(a, line);
                if (mine && pass0 + b < to && line < a.lines) {
                    const AttnView &in = l.is_q ? a.q : l.is_v ? a.v : a.k;
                    raw[b].read(in.data + bytes_to(in, row, l.head), f.part);
                }
            }
            if (pass0 == from) {
                place = my_place(a, row0, f.lines.row_off);
                turn.set(a, f.part, f.turns, place.position);
            }
#pragma unroll
            for (int b = 0; b < kAhead; ++b) {
                if (pass0 + b >= to) break;
                const int line = f.lines.first + (pass0 + b) * Lines<LOG>::kAtOnce;
                const Line l(a, line);
                const bool live = mine && line < a.lines;
                float x[8], y[8], squares = 0.0f;
                raw[b].to(x, live && place.there);
#pragma unroll
                for (int e = 0; e < 8; ++e) squares = fmaf(x[e], x[e], squares);
                const float s = 1.0f / sqrtf(fmaf(line_sum<LOG>(squares), each, a.eps));
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[e] * s * (l.is_q ? f.wq[e] : f.wk[e]);
                turn.apply(y, kHalves, 1.0f);
                const int64_t to_row = l.is_q ? row : place.store;
                const AttnView &out = l.is_q ? a.q_out : l.is_v ? a.v_out : a.k_out;
                if (live && to_row >= 0) {
                    if (!place.there) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = 0.0f;
                    }
                    write_parts<E>(out.data + bytes_to(out, to_row, l.head), l.is_v ? x : y, f.part);
                }
            }
        }
    }
}

template <typename E, bool kHalves, int LOG>
__global__ __launch_bounds__(256) void norm_rotate_grad_kernel(RotateArgs a) {
    constexpr int kAhead = 2;
    __shared__ float shared[4][2][kRotateDim];
    const Fixed<LOG> f(a);
    float dwq[8] = {}, dwk[8] = {};
    const float each = 1.0f / a.dim;
    const int64_t items = (a.rows + a.row_group - 1) / a.row_group;
    for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
        const int64_t row0 = item * a.row_group, row = row0 + f.lines.row_off;
        const bool mine = f.part.works && row < a.rows;
        Place place;
        Turn turn;
        for (int pass0 = 0; pass0 < a.passes; pass0 += kAhead) {
            Raw<E> of_x[kAhead], of_g[kAhead];
#pragma unroll
            for (int b = 0; b < kAhead; ++b) {
                const int line = f.lines.first + (pass0 + b) * Lines<LOG>::kAtOnce;
                const Line l(a, line);
                if (mine && line < a.lines) {
                    const AttnView &in = l.is_q ? a.q : a.k, &back = l.is_q ? a.q_out : a.k_out;
                    of_x[b].read(in.data + bytes_to(in, row, l.head), f.part);
                    of_g[b].read(back.data + bytes_to(back, row, l.head), f.part);
                }
            }
            if (pass0 == 0) {
                place = my_place(a, row0, f.lines.row_off);
                turn.set(a, f.part, f.turns, place.position);
            }
#pragma unroll
            for (int b = 0; b < kAhead; ++b) {
                const int line = f.lines.first + (pass0 + b) * Lines<LOG>::kAtOnce;
                const Line l(a, line);
                const bool live = mine && line < a.lines;
                float x[8], g[8], u[8];
                of_x[b].to(x, live && place.there);
                of_g[b].to(g, live && place.there);
                turn.apply(g, kHalves, -1.0f);
                float squares = 0.0f, along = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    u[e] = g[e] * (l.is_q ? f.wq[e] : f.wk[e]);
                    squares = fmaf(x[e], x[e], squares);
                    along = fmaf(x[e], u[e], along);
                }
                // (of no row: zeros, also where eps is zero)
                squares = line_sum<LOG>(squares);
                along = line_sum<LOG>(along);
                const float s = live && place.there ? 1.0f / sqrtf(fmaf(squares, each, a.eps)) : 0.0f;
                const float less = along * each * s * s;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float of_weight = g[e] * (x[e] * s);
                    dwq[e] += l.is_q ? of_weight : 0.0f;
                    dwk[e] += l.is_q ? 0.0f : of_weight;
                    u[e] = s * fmaf(x[e], -less, u[e]);
                }
                const AttnView &out = l.is_q ? a.dq : a.dk;
                if (live) write_parts<E>(out.data + bytes_to(out, row, l.head), u, f.part);
            }
        }
    }
    // the weights' gradients: over the lines of a wave, then its workgroup's waves
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        for (int s = LOG; s < 6; ++s) {
            dwq[e] += __shfl_xor(dwq[e], 1 << s);
            dwk[e] += __shfl_xor(dwk[e], 1 << s);
        }
        if (f.part.works && f.lines.sub == 0) {
            shared[threadIdx.x >> 6][0][f.part.element(e)] = dwq[e];
            shared[threadIdx.x >> 6][1][f.part.element(e)] = dwk[e];
        }
    }
    __syncthreads();
    const int which = threadIdx.x / kRotateDim, at = threadIdx.x % kRotateDim;
    if (at < a.dim)
        a.part[(int64_t)blockIdx.x * 2 * kRotateDim + threadIdx.x] =
            (shared[0][which][at] + shared[1][which][at]) + (shared[2][which][at] + shared[3][which][at]);
}

// The workgroups' sums, eight elements of a weight by each workgroup, in 64 bits and a fixed order.
__global__ __launch_bounds__(256) void norm_rotate_weights_kernel(RotateArgs a) {
    __shared__ double shared[32][8];
    const int which = blockIdx.y, at = blockIdx.x * 8 + (threadIdx.x & 7), share = threadIdx.x >> 3;
    double sum = 0.0;
#pragma unroll 8
    for (int b = share; b < a.blocks; b += 32) sum += (double)a.part[((int64_t)b * 2 + which) * kRotateDim + at];
    shared[share][threadIdx.x & 7] = sum;
    __syncthreads();
    if (share == 0) {
        for (int i = 1; i < 32; ++i) sum += shared[i][threadIdx.x];
        (which ? a.dk_weight : a.dq_weight)[at] = (float)sum;
    }
}

template <typename Launch>
void by_lanes(int log_lanes, Launch launch) {
    switch (log_lanes) {
        case 0: return launch(std::integral_constant<int, 0>());
        case 1: return launch(std::integral_constant<int, 1>());
        case 2: return launch(std::integral_constant<int, 2>());
        case 3: return launch(std::integral_constant<int, 3>());
        default: return launch(std::integral_constant<int, 4>());
    }
}

}  // namespace

hipError_t gbt_launch_norm_rotate(hipStream_t stream, const RotateArgs &a, int dtype) {
    by_lanes(a.log_lanes, [&](auto log) {
        constexpr int L = decltype(log)::value;
        if (dtype == GBT_BF16 && a.halves) norm_rotate_kernel<__bf16, true, L><<<a.blocks, 256, 0, stream>>>(a);
        else if (dtype == GBT_BF16) norm_rotate_kernel<__bf16, false, L><<<a.blocks, 256, 0, stream>>>(a);
        else if (a.halves) norm_rotate_kernel<_Float16, true, L><<<a.blocks, 256, 0, stream>>>(a);
        else norm_rotate_kernel<_Float16, false, L><<<a.blocks, 256, 0, stream>>>(a);
    });
    return hipGetLastError();
}

hipError_t gbt_launch_norm_rotate_grad(hipStream_t stream, const RotateArgs &a, int dtype) {
    by_lanes(a.log_lanes, [&](auto log) {
        constexpr int L = decltype(log)::value;
        if (dtype == GBT_BF16 && a.halves) norm_rotate_grad_kernel<__bf16, true, L><<<a.blocks, 256, 0, stream>>>(a);
        else if (dtype == GBT_BF16) norm_rotate_grad_kernel<__bf16, false, L><<<a.blocks, 256, 0, stream>>>(a);
        else if (a.halves) norm_rotate_grad_kernel<_Float16, true, L><<<a.blocks, 256, 0, stream>>>(a);
        else norm_rotate_grad_kernel<_Float16, false, L><<<a.blocks, 256, 0, stream>>>(a);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    norm_rotate_weights_kernel<<<dim3(a.dim / 8, 2), 256, 0, stream>>>(a);
    return hipGetLastError();
}
