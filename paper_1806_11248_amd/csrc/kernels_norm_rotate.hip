// The norm of every head's queries and keys, their rotation by position, and the way of keys and values into a store, in one pass; and the backward pass.
//
// x a head of dim elements: s = 1 / sqrt(mean x^2 + eps), y = x * s * weight, and each pair (a, b) of y's first `turned` elements is turned by
// position * turns revolutions.  Backward, of a gradient d: g is d turned back, u = g * weight, dx = s * (u - x * s^2 * mean(x * u)), and the weights'
// gradient is the sum of g * x * s over rows and heads.  A lane holds eight elements of a head, four pairs or both halves' four elements of them, so a
// pair never lies in two lanes; what lanes share is two sums.  Angles are taken in 64 bits, in revolutions, of which only the fraction goes on to the sine
// in 32, and what rounding it leaves is made up for by the sine's slope (off by at most 1.2e-7, and by 1.5e-7 without).  Bound: memory.
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
    int64_t first, behind;   // the sequence's rows
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
        p.store = a.store ? -1 : row, p.position = p.first = p.behind = 0, p.there = false;
        return p;
    }
    if (a.q_ptr) {
        q0 = a.q_ptr[seq], q1 = a.q_ptr[seq + 1];
    } else {
        const int64_t each = a.rows / a.n_seq;
        q0 = seq * each, q1 = q0 + each;
    }
    p.there = q0 >= 0 && q1 <= a.rows && row >= q0 && row < q1;
    p.first = q0, p.behind = q1;
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
        if (k0 < 0 || k1 < k0 || used < 0 || (a.store && k0 + used > a.out_rows)) used = 0;   // (k1 < k0: their difference may have passed 64 bits)
        at += used - (q1 - q0);
        slot = k0, room = used;
    } else if (a.store) {   // slots of one length, in use from their first row on as far as there are rows
        room = a.out_rows / a.n_seq;
        slot = seq * room;
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
    __device__ void write(char *row, const Part &p) const { *(Four<E> *)(row + p.lo * 2) = lo, *(Four<E> *)(row + p.hi * 2) = hi; }
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

// Over the 1 << LOG lanes of a line: neighbours, pairs, then mirrored within eight and sixteen, where all lanes of a half hold the same.
template <int CTRL>
__device__ __forceinline__ float plus_lane(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int LOG>
__device__ __forceinline__ float line_sum(float x) {
    if (LOG > 0) x = plus_lane<0xb1>(x);    // quad_perm 1, 0, 3, 2
    if (LOG > 1) x = plus_lane<0x4e>(x);    // quad_perm 2, 3, 0, 1
    if (LOG > 2) x = plus_lane<0x141>(x);   // row_half_mirror
    if (LOG > 3) x = plus_lane<0x140>(x);   // row_mirror
    return x;
}

// 1 / sqrt(x).  The instruction takes a denormal number, a mean of squares below 2^-126 with no eps, for zero.
__device__ __forceinline__ float inverse_root(float x) {
    const bool small = x < 0x1p-96f;
    return __builtin_amdgcn_rsqf(small ? x * 0x1p96f : x) * (small ? 0x1p48f : 1.0f);
}

// The heads of one tensor by a wave: lines of 1 << LOG lanes, as many at once as a wave has, of one row; where a row has fewer, of a few whole rows side by
// side (kSide).  All but the lane's own offset is the same in all lanes, and so a scalar.
template <int LOG, bool kSide>
struct Stream {
    static constexpr int kAtOnce = 64 >> LOG;
    int heads, row_off, head;   // the lane's row among those side by side, and its head there, in the first pass
    bool works;
    __device__ Stream(int heads, int row_group, const Part &part) : heads(heads) {
        const int sub = (threadIdx.x & 63) >> LOG;
        row_off = kSide ? sub / heads : 0;
        head = kSide ? sub - row_off * heads : sub;
        works = part.works && row_off < row_group;
    }
    __device__ int passes() const { return kSide ? 1 : (heads + kAtOnce - 1) / kAtOnce; }
    __device__ int64_t offset(const AttnView &x) const { return (row_off * x.row + head * x.head) * 2; }
    __device__ bool live(const RotateArgs &a, int64_t row0, int pass) const {
        return works && (kSide ? row0 + row_off < a.rows : head + pass * kAtOnce < heads);
    }
};

template <bool kSide>
__device__ __forceinline__ Place place_for(const RotateArgs &a, int64_t row0, int row_off) {
    const int64_t row = kSide ? min(row0 + row_off, a.rows - 1) : row0;
    int seq = 0;
    if (a.n_seq == 0) {
    } else if (a.q_ptr) {
        seq = sequence_of(a.q_ptr, a.n_seq, row0);
        if (kSide)
            for (int n = a.n_seq - seq; n > 1;) {
                const bool behind = a.q_ptr[seq + n / 2] <= row;
                seq += behind ? n / 2 : 0;
                n = behind ? n - n / 2 : n / 2;
            }
        else seq = __builtin_amdgcn_readfirstlane(seq);
    } else {
        seq = (int)min(row / max((int64_t)1, a.rows / a.n_seq), (int64_t)a.n_seq - 1);
    }
    return place_of(a, row, seq);
}

// What a lane multiplies the two elements of each of its pairs by: the weight times the turn's cosine and sine.
struct Turn {
    float cos[4], sin[4];
    __device__ void set(const Part &p, const double (&turns)[4], int64_t position) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double whole = (double)position * turns[i];
            const double exact = whole - rint(whole);   // in -1/2 .. 1/2 revolutions
            const float part = (float)exact, rest = (float)(exact - (double)part) * 6.28318531f;   // up to 2^-26 of one, which the sine would be off by
            const float c = __builtin_amdgcn_cosf(part), s = __builtin_amdgcn_sinf(part);
            cos[i] = p.turned ? fmaf(-rest, s, c) : 1.0f;
            sin[i] = p.turned ? fmaf(rest, c, s) : 0.0f;
        }
    }
};
// Pairs are (0, 4), (1, 5) .. of a lane's eight as halves, (0, 1), (2, 3) .. as neighbours.
template <bool kHalves>
__device__ __forceinline__ constexpr int first_of(int pair) { return kHalves ? pair : 2 * pair; }
template <bool kHalves>
__device__ __forceinline__ constexpr int second_of(int pair) { return kHalves ? 4 + pair : 2 * pair + 1; }

__device__ __forceinline__ void read_weight(float (&w)[8], const float *weight, const Part &part) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = part.works && weight ? weight[part.element(e)] : 1.0f;
}
__device__ __forceinline__ void read_turns(double (&turns)[4], const RotateArgs &a, const Part &part) {
#pragma unroll
    for (int i = 0; i < 4; ++i) turns[i] = part.turned ? a.turns[part.pair + i] : 0.0;
}

// The heads of q or k of an item's rows.
template <typename E, bool kHalves, int LOG, bool kSide, bool kStore>
__device__ __forceinline__ void turn_heads(const RotateArgs &a, const Stream<LOG, kSide> &st, const Part &part, const AttnView &in, const AttnView &out,
                                           int64_t row0, const Place &place, const Turn &turn, const float (&w)[8], int from, int to) {
    constexpr int kAhead = 4;   // passes under way
    float ac[4], as[4], bc[4], bs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float wa = place.there ? w[first_of<kHalves>(i)] : 0.0f, wb = place.there ? w[second_of<kHalves>(i)] : 0.0f;
        ac[i] = wa * turn.cos[i], as[i] = wa * turn.sin[i], bc[i] = wb * turn.cos[i], bs[i] = wb * turn.sin[i];
    }
    const float each = 1.0f / a.dim;
    const char *src = in.data + row0 * in.row * 2;
    // where a row goes is its own affair in a store, and with rows side by side the lane's
    char *dst = out.data + (kStore ? (kSide ? max(place.store, (int64_t)0) : place.store) : row0) * out.row * 2;
    const int64_t src_lane = st.offset(in), dst_lane = kStore ? st.head * out.head * 2 : st.offset(out);
    for (int pass0 = from; pass0 < to; pass0 += kAhead) {
        Raw<E> raw[kAhead];
#pragma unroll
        for (int b = 0; b < kAhead; ++b)
            if (pass0 + b < to && st.live(a, row0, pass0 + b)) raw[b].read(src + (pass0 + b) * Stream<LOG, kSide>::kAtOnce * in.head * 2 + src_lane, part);
#pragma unroll
        for (int b = 0; b < kAhead; ++b) {
            if (pass0 + b >= to) break;
            const bool live = st.live(a, row0, pass0 + b);
            float x[8], squares = 0.0f;
            raw[b].to(x, live && place.there);
#pragma unroll
            for (int e = 0; e < 8; ++e) squares = fmaf(x[e], x[e], squares);
            const float mean = fmaf(line_sum<LOG>(squares), each, a.eps);
            const float s = place.there ? inverse_root(mean) : 0.0f;
            float y[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float xa = x[first_of<kHalves>(i)] * s, xb = x[second_of<kHalves>(i)] * s;
                y[first_of<kHalves>(i)] = fmaf(xa, ac[i], -xb * bs[i]);
                y[second_of<kHalves>(i)] = fmaf(xa, as[i], xb * bc[i]);
            }
            if (live && (!kStore || place.store >= 0)) write_parts<E>(dst + (pass0 + b) * Stream<LOG, kSide>::kAtOnce * out.head * 2 + dst_lane, y, part);
        }
    }
}
template <typename E, int LOG, bool kSide, bool kStore>
__device__ __forceinline__ void copy_heads(const RotateArgs &a, const Stream<LOG, kSide> &st, const Part &part, const AttnView &in, const AttnView &out,
                                           int64_t row0, const Place &place, int from, int to) {
    const char *src = in.data + row0 * in.row * 2;
    char *dst = out.data + (kStore ? (kSide ? max(place.store, (int64_t)0) : place.store) : row0) * out.row * 2;
    const int64_t src_lane = st.offset(in), dst_lane = kStore ? st.head * out.head * 2 : st.offset(out);
    constexpr int kAhead = 4;   // passes under way
    for (int pass0 = from; pass0 < to; pass0 += kAhead) {
        Raw<E> raw[kAhead] = {};
#pragma unroll
        for (int b = 0; b < kAhead; ++b)
            if (pass0 + b < to && place.there && st.live(a, row0, pass0 + b)) raw[b].read(src + (pass0 + b) * Stream<LOG, kSide>::kAtOnce * in.head * 2 + src_lane, part);
#pragma unroll
        for (int b = 0; b < kAhead; ++b)
            if (pass0 + b < to && st.live(a, row0, pass0 + b) && (!kStore || place.store >= 0))
                raw[b].write(dst + (pass0 + b) * Stream<LOG, kSide>::kAtOnce * out.head * 2 + dst_lane, part);
    }
}

template <typename E, bool kHalves, int LOG, bool kSide, bool kStore>
__global__ __launch_bounds__(256) void norm_rotate_kernel(RotateArgs a) {
    const Part part(a, threadIdx.x & ((1 << LOG) - 1));
    const Stream<LOG, kSide> of_q(a.heads, a.row_group, part), of_k(a.kv_heads, a.row_group, part);
    double turns[4];
    float wq[8], wk[8];
    read_turns(turns, a, part);
    read_weight(wq, a.q_weight, part);
    read_weight(wk, a.k_weight, part);
    const int64_t items = (a.rows + a.row_group - 1) / a.row_group * a.parts;
    const int q_passes = of_q.passes(), k_passes = of_k.passes(), all = q_passes + k_passes * (a.v.data ? 2 : 1);
    const int64_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    for (int64_t item = wave; item < items; item += (int64_t)gridDim.x * 4) {
        const int64_t row0 = item / a.parts * a.row_group;
        // one of `parts` stretches of the row's passes: those of q, of k, of v
        const int part_of = (int)(item % a.parts), first = (int)((int64_t)all * part_of / a.parts), last = (int)((int64_t)all * (part_of + 1) / a.parts);
        Place place = place_for<kSide>(a, row0, of_q.row_off);
        Turn turn;
        turn.set(part, turns, place.position);
        if (first < q_passes)
            turn_heads<E, kHalves, LOG, kSide, false>(a, of_q, part, a.q, a.q_out, row0, place, turn, wq, first, min(last, q_passes));
        if (last <= q_passes) continue;
        if (kSide) {   // a lane's key is not of its query's row
            place = place_for<kSide>(a, row0, of_k.row_off);
            turn.set(part, turns, place.position);
        }
        const int k_first = max(first - q_passes, 0), k_last = last - q_passes;
        if (k_first < k_passes)
            turn_heads<E, kHalves, LOG, kSide, kStore>(a, of_k, part, a.k, a.k_out, row0, place, turn, wk, k_first, min(k_last, k_passes));
        if (k_last > k_passes) copy_heads<E, LOG, kSide, kStore>(a, of_k, part, a.v, a.v_out, row0, place, max(k_first - k_passes, 0), k_last - k_passes);
    }
}

// The gradients of all rows' heads of q or of k by `blocks` workgroups, of which this one is number `block`, and what they add to the weight's.  A wave's rows lie side by
// side, so that it looks a sequence up once; while it works on a pass, the next one's elements are under way, across rows too.
// (30,141 rows of 32 and 8 heads of 128: 201 us, 4.6 TB/s; two passes at a time of rows far apart 221.)
template <typename E, bool kHalves, int LOG, bool kSide>
__device__ __forceinline__ void turn_all_back(const RotateArgs &a, int heads, int row_group, const AttnView &in, const AttnView &back, const AttnView &out,
                                              const float *weight, int block, int blocks, const Part &part, float (&dw)[8]) {
    constexpr int kAtOnce = Stream<LOG, kSide>::kAtOnce;
    const Stream<LOG, kSide> st(heads, row_group, part);
    double turns[4];
    float w[8];
    read_turns(turns, a, part);
    read_weight(w, weight, part);
    const float each = 1.0f / a.dim;
    const int64_t src_lane = st.offset(in), back_lane = st.offset(back), dst_lane = st.offset(out);
    const int passes = st.passes();
    const int64_t items = (a.rows + row_group - 1) / row_group, waves = (int64_t)blocks * 4;
    const int64_t wave = __builtin_amdgcn_readfirstlane(block * 4 + (threadIdx.x >> 6)), all = items / waves, more = items % waves;
    int64_t row0 = (wave * all + min(wave, more)) * row_group;
    const int64_t to = row0 + (all + (wave < more)) * row_group;
    Place place = {};
    Turn turn;
    float piece[8] = {};   // of the weight's gradient: at most kBehind terms behind one another (8400 equal ones were off by 1.1e-4)
    constexpr int kBehind = 256;
    struct Pass {
        int64_t row0;
        int pass;
        Raw<E> of_x, of_g;
    } even, odd;
    int pass = 0;
    auto fetch = [&](Pass &p) {   // the next one; there need not be one
        p.row0 = row0, p.pass = pass;
        if (row0 < to && st.live(a, row0, pass)) {
            p.of_x.read(in.data + row0 * in.row * 2 + (int64_t)pass * kAtOnce * in.head * 2 + src_lane, part);
            p.of_g.read(back.data + row0 * back.row * 2 + (int64_t)pass * kAtOnce * back.head * 2 + back_lane, part);
        }
        if (++pass == passes) pass = 0, row0 += row_group;
    };
    auto work = [&](const Pass &p) {
        if (p.row0 >= to) return;
        if (p.pass == 0) {
            if (!kSide && !a.positions && place.there && p.row0 < place.behind) ++place.position;   // the row behind the last one
            else place = place_for<kSide>(a, p.row0, st.row_off);
            turn.set(part, turns, place.position);
        }
        const bool live = st.live(a, p.row0, p.pass);
        float x[8], d[8], g[8], u[8], squares = 0.0f, along = 0.0f;
        p.of_x.to(x, live && place.there);
        p.of_g.to(d, live && place.there);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float da = d[first_of<kHalves>(i)], db = d[second_of<kHalves>(i)];
            g[first_of<kHalves>(i)] = fmaf(da, turn.cos[i], db * turn.sin[i]);
            g[second_of<kHalves>(i)] = fmaf(db, turn.cos[i], -da * turn.sin[i]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = g[e] * w[e];
            squares = fmaf(x[e], x[e], squares);
            along = fmaf(x[e], u[e], along);
        }
        squares = line_sum<LOG>(squares);
        along = line_sum<LOG>(along);
        // (of no row: zeros, also where eps is zero)
        const float s = live && place.there ? inverse_root(fmaf(squares, each, a.eps)) : 0.0f;
        const float less = along * each * s * s;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            piece[e] = fmaf(g[e], x[e] * s, piece[e]);
            u[e] = s * fmaf(x[e], -less, u[e]);
        }
        if (live) write_parts<E>(out.data + p.row0 * out.row * 2 + (int64_t)p.pass * kAtOnce * out.head * 2 + dst_lane, u, part);
    };
    fetch(even);
    int behind = 0;
    while (even.row0 < to) {
        fetch(odd);
        work(even);
        fetch(even);
        work(odd);
        if ((behind += 2) == kBehind) {
            behind = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) dw[e] += piece[e], piece[e] = 0.0f;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] += piece[e];
}

// The first blocks take q, the others k: a wave's registers hold one weight and its gradient.
template <typename E, bool kHalves, int LOG>
__global__ __launch_bounds__(256, 4) void norm_rotate_grad_kernel(RotateArgs a) {
    __shared__ float shared[4][kRotateDim];
    const Part part(a, threadIdx.x & ((1 << LOG) - 1));
    float dw[8] = {};
    const bool of_q = (int)blockIdx.x < a.q_blocks;
    const int block = of_q ? blockIdx.x : blockIdx.x - a.q_blocks, blocks = of_q ? a.q_blocks : a.blocks - a.q_blocks;
    const int heads = of_q ? a.heads : a.kv_heads, row_group = of_q ? a.row_group : a.k_row_group;
    const AttnView in = of_q ? a.q : a.k, back = of_q ? a.q_out : a.k_out, out = of_q ? a.dq : a.dk;
    const float *weight = of_q ? a.q_weight : a.k_weight;
    if (row_group > 1) turn_all_back<E, kHalves, LOG, true>(a, heads, row_group, in, back, out, weight, block, blocks, part, dw);
    else turn_all_back<E, kHalves, LOG, false>(a, heads, 1, in, back, out, weight, block, blocks, part, dw);
    // the weight's gradient: over the lines of a wave, then the workgroup's waves
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int s = LOG; s < 6; ++s) dw[e] += __shfl_xor(dw[e], 1 << s);
        if (part.works && (threadIdx.x & 63) >> LOG == 0) shared[threadIdx.x >> 6][part.element(e)] = dw[e];
    }
    __syncthreads();
    const int at = threadIdx.x;
    if (at < a.dim) a.part[(int64_t)blockIdx.x * kRotateDim + at] = (shared[0][at] + shared[1][at]) + (shared[2][at] + shared[3][at]);
}

// The workgroups' sums, eight elements of a weight by each workgroup, in 64 bits and a fixed order.
__global__ __launch_bounds__(256) void norm_rotate_weights_kernel(RotateArgs a) {
    __shared__ double shared[32][8];
    const int which = blockIdx.y, at = blockIdx.x * 8 + (threadIdx.x & 7), share = threadIdx.x >> 3;
    double sum = 0.0;
#pragma unroll 8
    for (int b = (which ? a.q_blocks : 0) + share; b < (which ? a.blocks : a.q_blocks); b += 32) sum += (double)a.part[(int64_t)b * kRotateDim + at];
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

template <typename Launch>
void by_flag(bool flag, Launch launch) {
    if (flag) launch(std::true_type());
    else launch(std::false_type());
}

}  // namespace

hipError_t gbt_launch_norm_rotate(hipStream_t stream, const RotateArgs &a, int dtype) {
    by_lanes(a.log_lanes, [&](auto log) {
        by_flag(a.halves, [&](auto halves) {
            by_flag(a.row_group > 1, [&](auto side) {
                by_flag(a.store, [&](auto store) {
                    constexpr int L = decltype(log)::value;
                    constexpr bool H = decltype(halves)::value, S = decltype(side)::value, T = decltype(store)::value;
                    if (dtype == GBT_BF16) norm_rotate_kernel<__bf16, H, L, S, T><<<a.blocks, 256, 0, stream>>>(a);
                    else norm_rotate_kernel<_Float16, H, L, S, T><<<a.blocks, 256, 0, stream>>>(a);
                });
            });
        });
    });
    return hipGetLastError();
}

hipError_t gbt_launch_norm_rotate_grad(hipStream_t stream, const RotateArgs &a, int dtype) {
    by_lanes(a.log_lanes, [&](auto log) {
        by_flag(a.halves, [&](auto halves) {
            constexpr int L = decltype(log)::value;
            constexpr bool H = decltype(halves)::value;
            if (dtype == GBT_BF16) norm_rotate_grad_kernel<__bf16, H, L><<<a.blocks, 256, 0, stream>>>(a);
            else norm_rotate_grad_kernel<_Float16, H, L><<<a.blocks, 256, 0, stream>>>(a);
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    norm_rotate_weights_kernel<<<dim3(a.dim / 8, 2), 256, 0, stream>>>(a);
    return hipGetLastError();
}
