// Attention over ragged rows, with a bias for each bucket of distance.
//
//   S_ij = scale * q_i . k_j + bias[b(t)][h],  t = j - (i + nk - nq);   out_i = sum_j softmax_j(S_ij) v_j
//
// One pass over the keys with a running maximum and sum: out is kept as sum_j 2^(s_ij - m) v_j.  m follows the row's maximum only when
// that has grown by more than kSlack: some row of a wave meets a new maximum in most tiles, but seldom one that much larger, and a factor of
// 2^kSlack more or less matters to no 32-bit sum and to no rounding of a probability.  float16 has few exponents: there m is kept
// P::kAbove below the maximum, so that probabilities reach up to 2^15 and those of 2^-21 are still normal numbers.  (One key and 131,000 others at 2^-26
// of its weight, without: 1.7% off, since the others are in the sum but not in the product.)
// Sums, maxima and out are held in 32 bits; the probabilities are rounded to the inputs' type for the second product, while their
// sum is taken of the unrounded ones (the rounding errors of a row then average out in out, whose own last place is of that size).
// Rows of out are divided by the sum at the end; a row without keys has none and is zeros.
#include "attention.h"

#include <type_traits>

namespace {

constexpr float kSlack = 8.0f;   // kSlack + P::kAbove < 16: float16 ends before 2^16

// ------------------------------------------------------------------------------------------------ blocks of queries --
// A wave takes 32 queries of one head (its columns), a workgroup 128 or 64 (attn_form); keys and values pass through LDS, 64 at a time.  Of two groups
// of waves each takes every other tile for the same queries, and they are joined at the end: half the steps one after the other.
//
// Bound: the matrix units together with the exponentials and the arithmetic around them, which take turns more than they overlap: 64 keys against 32
// queries are 32 matrix instructions at 128 elements a head, 16 at 64, and either way some 130 others, 32 of them exponentials of four times an
// addition's time.  So large heads come nearer the rate of a large library product (1198 TFLOP/s in bfloat16 here): 8192 causal rows, 16 heads of 128
// elements 304 us, 904 TFLOP/s of the pairs that count; not causal 128 queries a head against 16384 keys 1024 without a bias, 946 with one; heads of 64
// 676 and 621; the matrix units are busy 39% of the time, LDS 24%, without bank conflicts (two causal histories of 4096).  Ragged short histories are
// bound by how their blocks fall on the compute units: 24 of 100 to 1000 rows, 8 heads of 64 40 us, where blocks enough would take 27.
//
// kParts: probabilities as operands, whole or in two parts.  The rounding errors of few probabilities do not average out, and what is wrong in out is wrong
// in the backward pass's delta: of histories of 5 to 60 rows, 4 heads of 32, out was 1.12 times as far from the 64-bit result as rounding it alone makes it, and
// dq 1.48 times.  Calls of at most one tile of keys a sequence take two parts, 1.00 and 1.43: 32 such histories 11.5 us as before, 2000 of 64 rows, heads of 64
// 145, 150; 20,000 of 0 to 60 416, 461.  Longer ones are nearer anyhow (dq 1.43 to 1.45 times) and would pay as much.
constexpr int kFewKeys = 64;
template <typename P, int DP, int kQWaves, int kGroups, int kParts>
__global__ __launch_bounds__(64 * kQWaves * kGroups, 2) void attention_kernel(AttnArgs a, AttnCuts c) {
    typedef typename P::elem E;
    typedef typename P::vec8 V8;
    typedef Tile<DP> T;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32, kStride = 64 * kGroups, kQueries = 32 * kQWaves, kWaves = kQWaves * kGroups;
    __shared__ __align__(16) char k_tile[2][kGroups * T::kBytes];
    __shared__ __align__(16) char v_tile[2][kGroups * T::kBytes];
    __shared__ DistanceRing<256 * kGroups> ring;

    if (blockIdx.x >= a.work) return zero_gaps(a, a.out, false);
    const AttnItem item = attn_item(a);
    if (item.seq < 0) return;
    // the blocks that see the most keys first
    const int block = a.order.blocks - 1 - item.block, head = item.unit, seq = item.seq;
    const AttnSeq rows = attn_seq(a, seq);
    const int first = block * kQueries;
    if (first >= rows.nq) return;
    const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int wave = kGroups == 2 ? any_wave % kQWaves : any_wave, group = kGroups == 2 ? any_wave / kQWaves : 0;
    const int off = rows.nk - rows.nq;
    const int query = first + wave * 32 + (lane & 31);
    const bool bias = a.n_buckets > 0;
    // keys 0 .. last are seen by this lane's query; `end` by any of the workgroup's
    const int last = a.causal ? min(rows.nk - 1, query + off) : rows.nk - 1;
    const int end = a.causal ? min(rows.nk, min(first + kQueries, rows.nq) + off) : rows.nk;
    const int wave_first = first + wave * 32;                                               // the wave's keys end before
    const int wave_end = a.causal ? min(rows.nk, min(wave_first + 32, rows.nq) + off) : rows.nk;
    const int wave_all = a.causal ? min(rows.nk, wave_first + off + 1) : rows.nk;           // and all of its queries see those before

    const int kv_head = head / a.group;
    const char *k_base = a.k.data + (rows.k0 * a.k.row + (int64_t)kv_head * a.k.head) * 2;
    const char *v_base = a.v.data + (rows.k0 * a.v.row + (int64_t)kv_head * a.v.head) * 2;

    auto fetch = [&](int which, int kb) {
        T::template fetch<true, kQWaves>(k_tile[which] + group * T::kBytes, k_base + (int64_t)kb * a.k.row * 2, (uint32_t)a.k.row * 2, end - kb, a.dim, wave);
        T::template fetch<true, kQWaves>(v_tile[which] + group * T::kBytes, v_base + (int64_t)kb * a.v.row * 2, (uint32_t)a.v.row * 2, end - kb, a.dim, wave);
    };
    if (64 * group < end) fetch(0, 64 * group);
    V8 qf[kSteps];
    load_row(qf, a.q.data + ((rows.q0 + min(query, rows.nq - 1)) * a.q.row + (int64_t)head * a.q.head) * 2, half, a.dim);
    if (bias) {
        ring_cuts(ring, a, c);
        ring_head(ring, a, head);
    }
    f32x16 o[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;
    float top = -INFINITY, sum = 0.0f;
    arrived(qf);
    __syncthreads();
    if (bias && any_wave < kQWaves / 2 + kGroups) ring_put(ring, 64 * any_wave - (first + kQueries - 1 + off), any_wave, lane);

    // one tile; which of the two copies it lies in is known at compile time, so that LDS addresses are constants of the lane
    auto step = [&](auto which, int k0) {
        constexpr int kNow = decltype(which)::value;
        const char *k_now = k_tile[kNow] + group * T::kBytes, *v_now = v_tile[kNow] + group * T::kBytes;
        const int kb = k0 + 64 * group;
        tiles_ready();
        if (kb + kStride < end) fetch(1 - kNow, kb + kStride);
        const int lowest = k0 - (first + kQueries - 1 + off);   // distance
        const int turn = (any_wave - (k0 >> 6)) & (kWaves - 1);
        if (bias && turn < kGroups) ring_put(ring, lowest + kQueries - 1 + kStride + 64 * turn, any_wave, lane);
        if (kb >= wave_end) return;

        __builtin_amdgcn_s_setprio(1);   // products before the other waves' arithmetic
        f32x16 s[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[0][r] = s[1][r] = 0.0f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) s[b] = P::mma(T::template rows<P>(k_now, 32 * b, i, lane), qf[i], s[b]);
        // reads a few products ahead
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < kSteps - 2; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        __builtin_amdgcn_s_setprio(0);
        // scores in powers of two are s * factor + add
        const int at = (lowest & ring.kMask) + 64 * group + kQueries - 32 - 32 * wave;   // of the wave's lowest distance, of 95
        const int b0 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at]) : 0, b1 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at + 94]) : 0;
        float factor = a.scale2, add = 0.0f;
        if (b0 != b1) {
            const float *value = ring.value + at + 31 - (lane & 31);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] = fmaf(s[b][r], a.scale2, value[32 * b + result_row(r, half)]);
            factor = 1.0f;
        } else if (bias) {
            add = ring.of_bucket[b0];
        }
        if (kb + 64 > wave_all) {
            const int past = last - kb - 4 * half;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] = 32 * b + result_row(r, 0) <= past ? s[b][r] : -INFINITY;
        }
        float now = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) now = fmaxf(now, s[b][r]);
        now = fmaxf(top, column_max(fmaf(now, factor, add - P::kAbove)));
        if (__any(now > top + kSlack)) {
            const float shrink = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.0f : now));
            sum *= shrink;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= shrink;
            top = now;
        }
        add -= top == -INFINITY ? 0.0f : top;   // a row that has seen nothing yet
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], factor, add));
                sum += s[b][r];
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const V8 p = operand<P>(s[i / 2], i % 2);
            V8 rest;
            if constexpr (kParts == 2) rest = operand_rest<P>(s[i / 2], i % 2, p);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const V8 values = T::template cols<P>(v_now, 16 * i, b, lane);
                o[b] = P::mma(values, p, o[b]);
                if constexpr (kParts == 2) o[b] = P::mma(values, rest, o[b]);
            }
        }
    };
    for (int k0 = 0; k0 < end; k0 += 2 * kStride) {
        step(std::integral_constant<int, 0>{}, k0);
        if (k0 + kStride < end) step(std::integral_constant<int, 1>{}, k0 + kStride);
    }

    sum = column_sum(sum);
    if constexpr (kGroups == 2) {   // the second group's rows to the first, through LDS
        float *theirs = (float *)(wave < 2 ? &k_tile[0][0] : &v_tile[0][0]) + (wave & 1) * (16 * kBlocks + 2) * 64 + lane;
        static_assert(2 * (16 * kBlocks + 2) * 256 <= (int)sizeof k_tile, "two waves' sums fit where the keys were");
        __syncthreads();
        if (group == 1) {
#pragma unroll
            for (int i = 0; i < 16 * kBlocks; ++i) theirs[64 * i] = o[i / 16][i % 16];
            theirs[64 * 16 * kBlocks] = top;
            theirs[64 * (16 * kBlocks + 1)] = sum;
        }
        __syncthreads();
        if (group == 1) return;
        const float their_top = theirs[64 * 16 * kBlocks], all = fmaxf(top, their_top), base = all == -INFINITY ? 0.0f : all;
        const float mine_by = __builtin_amdgcn_exp2f(top - base), theirs_by = __builtin_amdgcn_exp2f(their_top - base);
        sum = sum * mine_by + theirs[64 * (16 * kBlocks + 1)] * theirs_by;
        top = all;
#pragma unroll
        for (int i = 0; i < 16 * kBlocks; ++i) o[i / 16][i % 16] = o[i / 16][i % 16] * mine_by + theirs[64 * i] * theirs_by;
    }
    if (query >= rows.nq) return;
    const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;   // no key: zeros; a sum that is no number stays none
    if (a.lse && half == 0) a.lse[(int64_t)head * a.q_rows + rows.q0 + query] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * GBT_LN2;
    E *out = (E *)a.out.data + (rows.q0 + query) * a.out.row + (int64_t)head * a.out.head;
    E *rest = (E *)a.rest + ((rows.q0 + query) * a.heads + head) * a.dim;
    typedef E E4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * b + 8 * g + 4 * half;
            if (d < a.dim) {
                E4 x, y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = o[b][4 * g + e] * inv;
                    x[e] = (E)w;
                    y[e] = (E)(w - (float)x[e]);
                }
                *(E4 *)(out + d) = x;
                if (a.rest) *(E4 *)(rest + d) = y;
            }
        }
}

// -------------------------------------------------------------------------------------------------------- few rows --
// Single new events against a long store: what there is to do is to read the store once.  The columns of a wave are the (query, head
// of the group) pairs of one key head, 32 of them at most, so that all heads that share keys read them together; the four waves of a
// workgroup take every fourth 32 keys of its piece of the key axis, each through its own part of LDS, so no wave waits for another.  The next
// keys are under way as soon as the products with the last have been made, the next values likewise.  The waves are joined at the
// end, the pieces by a second launch.
// Probabilities are operands in two parts, what rounding takes from the first being the second: a few rows are few numbers, in which one rounded probability
// shows (4 rows of 8 heads, an error of 1.3 to 1.8 times that of rounding the result alone), and the matrix units have the time.
// Bound: memory.  16 stores of 2000 to 30000 rows, 16 heads of 128 elements on 4 key heads, 557 MB: 111 us (5.0 TB/s, where a large copy moves 5.1) and
// 6 us for the joining; matrix units busy 11%, LDS 5%.  64 stores of 30 to 3000 rows, 220 MB: 45 + 5.  Four short ones: 10 us, the time of one step after
// the other.
template <typename P, int DP>
__global__ __launch_bounds__(256, 2) void attention_few_kernel(AttnArgs a, AttnCuts c) {
    typedef typename P::elem E;
    typedef typename P::vec8 V8;
    typedef Tile<DP> T;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32;
    constexpr int kJoin = 32 * 33;   // floats of a wave's 32 x 32 block, rows 33 places apart
    __shared__ __align__(16) char space[4 * T::kBytes >= 16 * kJoin ? 4 * T::kBytes : 16 * kJoin];   // keys and values of the waves; at the end such blocks
    __shared__ uint8_t is_cut[4][64], near_bucket[4][64];
    __shared__ float join_top[4][32], join_sum[4][32];
    extern __shared__ float table[];   // [n_buckets][32 columns]: the bias, times log2(e)

    if (blockIdx.x >= a.work) return zero_gaps(a, a.out, false);
    const int columns = a.group * a.max_q;
    // the first pieces of all sequences before the second ones, and each time one further: side by side the later pieces, of which there are fewer, would
    // all go to some of the XCDs, and without the shift all of a long sequence's to one (128 stores of 30 to 3000 rows, 8 key heads of 64, 115 and 98 us, so 94; 16
    // of 2000 to 30000, 4 of 128, 113 and 128, so 114)
    const unsigned units = a.work / a.pieces, turn = blockIdx.x / units, unit = (blockIdx.x + turn) % units;
    const int piece = (int)turn, kv_head = (int)(unit % a.kv_heads), seq = (int)(unit / a.kv_heads);
    const AttnSeq rows = attn_seq(a, seq);
    const int begin = piece * a.piece_len;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int query = col / a.group, head = kv_head * a.group + col % a.group;
    if (rows.nq == 0) return;
    if (begin > 0 && begin >= rows.nk) return;   // the first piece writes the rows without keys
    const int off = rows.nk - rows.nq;
    const bool there = query < rows.nq;
    const bool bias = a.n_buckets > 0;

    const int q_high = rows.nq - 1;
    const int last = a.causal ? min(rows.nk - 1, query + off) : rows.nk - 1;
    const int end = min(min(rows.nk, begin + a.piece_len), a.causal ? q_high + off + 1 : rows.nk);
    const int all = a.causal ? min(end, off + 1) : end;   // every query sees the keys before
    const char *k_base = a.k.data + (rows.k0 * a.k.row + (int64_t)kv_head * a.k.head) * 2;
    const char *v_base = a.v.data + (rows.k0 * a.v.row + (int64_t)kv_head * a.v.head) * 2;
    char *k_tile = space + wave * (T::kBytes / 2), *v_tile = k_tile + 2 * T::kBytes;
    auto fetch_k = [&](int kb) { T::fetch_half(k_tile, k_base + (int64_t)kb * a.k.row * 2, (uint32_t)a.k.row * 2, end - kb, a.dim); };
    auto fetch_v = [&](int kb) { T::fetch_half(v_tile, v_base + (int64_t)kb * a.v.row * 2, (uint32_t)a.v.row * 2, end - kb, a.dim); };
    const int start = begin + 32 * wave;
    V8 qf[kSteps];
    load_row(qf, a.q.data + ((rows.q0 + min(query, rows.nq - 1)) * a.q.row + (int64_t)head * a.q.head) * 2, half, a.dim);
    const LaneCuts cuts{lane < a.n_buckets - 1 ? c.at[lane] : INT32_MAX, lane + 64 < a.n_buckets - 1 ? c.at[lane + 64] : INT32_MAX};
    if (bias) {
        const float *from = a.bias + (there ? head : 0);
        for (int i = 2 * wave + half; i < a.n_buckets; i += 8) table[32 * i + col] = bias_value(from[(int64_t)i * a.heads]);
    }
    arrived(qf);
    if (start < end) {
        fetch_k(start);
        fetch_v(start);
    }
    __syncthreads();   // the table

    f32x16 o[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;
    float top = -INFINITY, sum = 0.0f;

    for (int kb = start; kb < end; kb += 128) {
        T::half_ready();   // the keys; the values after them are still under way
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) s = P::mma(T::template rows<P>(k_tile, 0, i, lane), qf[i], s);
        done_reading();
        fetch_k(min(kb + 128, end - 1));   // after the last step some key again, so that the count of loads under way stays the same
        const int lowest = kb - (q_high + off), span = 31 + q_high;   // distances lowest .. lowest + span, 63 at most
        const int mine = bias ? lane_bucket(is_cut[wave], cuts, lowest, lane) : 0;
        const int b0 = __builtin_amdgcn_readfirstlane(mine), b1 = __builtin_amdgcn_readlane(mine, span);
        float factor = a.scale2, add = 0.0f;
        if (b0 != b1) {
            near_bucket[wave][lane] = (uint8_t)mine;
            __builtin_amdgcn_wave_barrier();
            const uint8_t *at = near_bucket[wave] + (there ? q_high - query : 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], a.scale2, table[32 * at[result_row(r, half)] + col]);
            factor = 1.0f;
        } else if (bias) {
            add = table[32 * b0 + col];
        }
        if (kb + 32 > all) {
            const int past = min(last, end - 1) - kb - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = result_row(r, 0) <= past ? s[r] : -INFINITY;
        }
        float now = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) now = fmaxf(now, s[r]);
        now = fmaxf(top, column_max(fmaf(now, factor, add - P::kAbove)));
        if (__any(now > top + kSlack)) {
            const float shrink = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.0f : now));
            sum *= shrink;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= shrink;
            top = now;
        }
        add -= top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], factor, add));
            sum += s[r];
        }
        T::half_ready();   // the values; the next keys are under way
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const V8 p = operand<P>(s, i), rest = operand_rest<P>(s, i, p);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const V8 values = T::template cols<P>(v_tile, 16 * i, b, lane);
                o[b] = P::mma(values, p, o[b]);
                o[b] = P::mma(values, rest, o[b]);
            }
        }
        done_reading();
        fetch_v(min(kb + 128, end - 1));
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    // the four waves' rows together
    sum = column_sum(sum);
    if (half == 0) {
        join_top[wave][lane] = top;
        join_sum[wave][lane] = sum;
    }
    __syncthreads();
    float all_top = -INFINITY, all_sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) all_top = fmaxf(all_top, join_top[w][col]);
    const float base = all_top == -INFINITY ? 0.0f : all_top;
#pragma unroll
    for (int w = 0; w < 4; ++w) all_sum += join_sum[w][col] * __builtin_amdgcn_exp2f(join_top[w][col] - base);
    const bool whole = rows.nk <= a.piece_len;   // a sequence of one piece needs no joining
    const float factor = __builtin_amdgcn_exp2f(top - base) * (whole ? all_sum > 0.0f ? 1.0f / all_sum : all_sum == 0.0f ? 0.0f : all_sum : 1.0f);
    const int64_t part = ((((int64_t)seq * a.kv_heads + kv_head) * columns + col) * a.pieces + piece) * (a.dim + 2);
    if (wave == 0 && half == 0 && there) {
        if (whole) {
            if (a.lse) a.lse[(int64_t)head * a.q_rows + rows.q0 + query] = all_sum == 0.0f ? -INFINITY : (all_top + __builtin_amdgcn_logf(all_sum)) * GBT_LN2;
        } else {
            a.part[part + a.dim] = all_top;
            a.part[part + a.dim + 1] = all_sum;
        }
    }
    // a block of 32 elements after the other
    float *join_o = (float *)space;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        if (b) __syncthreads();
#pragma unroll
        for (int r = 0; r < 16; ++r) join_o[wave * kJoin + col * 33 + result_row(r, half)] = o[b][r] * factor;
        __syncthreads();
        for (int i = threadIdx.x; i < 32 * 32; i += 256) {
            const int cc = i >> 5, d = 32 * b + (i & 31), query2 = cc / a.group;
            if (query2 >= rows.nq || d >= a.dim) continue;
            const int x = cc * 33 + (i & 31);
            const float w = (join_o[x] + join_o[kJoin + x]) + (join_o[2 * kJoin + x] + join_o[3 * kJoin + x]);
            const int head2 = kv_head * a.group + cc % a.group;
            if (whole) {
                const E y = (E)w;
                ((E *)a.out.data)[(rows.q0 + query2) * a.out.row + (int64_t)head2 * a.out.head + d] = y;
                if (a.rest) ((E *)a.rest)[((rows.q0 + query2) * a.heads + head2) * a.dim + d] = (E)(w - (float)y);
            } else {
                a.part[((((int64_t)seq * a.kv_heads + kv_head) * columns + cc) * a.pieces + piece) * (a.dim + 2) + d] = w;
            }
        }
    }
}

// The pieces of the key axis together: a workgroup takes a (sequence, key head, column), a wave every fourth piece of it, its lanes the elements.
template <typename P>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a) {
    typedef typename P::elem E;
    __shared__ float join_top[4], join_sum[4], join_o[4][128];
    const int columns = a.group * a.max_q, at = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int column = at % columns, kv_head = at / columns % a.kv_heads, seq = at / columns / a.kv_heads;
    const int query = column / a.group, head = kv_head * a.group + column % a.group;
    const AttnSeq rows = attn_seq(a, seq);
    if (query >= rows.nq) return;
    const int n = (rows.nk + a.piece_len - 1) / a.piece_len, wide = a.dim + 2;
    if (n < 2) return;
    const float *part = a.part + (int64_t)at * a.pieces * wide;
    // a lane's piece of this wave's, 64 of them at most
    const int mine = wave + 4 * lane;
    const float top = mine < n ? part[(int64_t)mine * wide + a.dim] : -INFINITY, sum = mine < n ? part[(int64_t)mine * wide + a.dim + 1] : 0.0f;
    float most = top;
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    const float base = most == -INFINITY ? 0.0f : most, factor = __builtin_amdgcn_exp2f(top - base), total = wave_sum(sum * factor);
    float o0 = 0.0f, o1 = 0.0f;
    const int d0 = min(lane, a.dim - 1), d1 = min(lane + 64, a.dim - 1);
#pragma unroll 8
    for (int p = wave; p < n; p += 4) {
        const float f = __shfl(factor, p >> 2);
        o0 = fmaf(part[(int64_t)p * wide + d0], f, o0);
        o1 = fmaf(part[(int64_t)p * wide + d1], f, o1);
    }
    join_o[wave][lane] = o0;
    join_o[wave][lane + 64] = o1;
    if (lane == 0) {
        join_top[wave] = most;
        join_sum[wave] = total;
    }
    __syncthreads();
    const float all = fmaxf(fmaxf(join_top[0], join_top[1]), fmaxf(join_top[2], join_top[3])), all_base = all == -INFINITY ? 0.0f : all;
    float w[4], l = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = __builtin_amdgcn_exp2f(join_top[i] - all_base);
        l = fmaf(join_sum[i], w[i], l);
    }
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (a.lse && threadIdx.x == 0) a.lse[(int64_t)head * a.q_rows + rows.q0 + query] = l == 0.0f ? -INFINITY : (all + __builtin_amdgcn_logf(l)) * GBT_LN2;
    if ((int)threadIdx.x < a.dim) {
        const int d = threadIdx.x;
        const float x = ((join_o[0][d] * w[0] + join_o[1][d] * w[1]) + (join_o[2][d] * w[2] + join_o[3][d] * w[3])) * inv;
        const E y = (E)x;
        ((E *)a.out.data)[(rows.q0 + query) * a.out.row + (int64_t)head * a.out.head + d] = y;
        if (a.rest) ((E *)a.rest)[((rows.q0 + query) * a.heads + head) * a.dim + d] = (E)(x - (float)y);
    }
}

// The same for up to 16 pieces, a wave a column.  (500 stores of 30 to 1500 rows in two pieces, 8 columns each: kernel and joining 60 -> 54 us.)
constexpr int kFewJoined = 16;
template <typename P>
__global__ __launch_bounds__(256) void attention_join_few_kernel(AttnArgs a) {
    typedef typename P::elem E;
    const int columns = a.group * a.max_q, lane = threadIdx.x & 63, at = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int column = at % columns, kv_head = at / columns % a.kv_heads, seq = at / columns / a.kv_heads;
    if (seq >= a.n_seq) return;
    const int query = column / a.group, head = kv_head * a.group + column % a.group;
    const AttnSeq rows = attn_seq(a, seq);
    if (query >= rows.nq) return;
    const int n = (rows.nk + a.piece_len - 1) / a.piece_len, wide = a.dim + 2;
    if (n < 2) return;
    const float *part = a.part + (int64_t)at * a.pieces * wide;
    const float top = lane < n ? part[(int64_t)lane * wide + a.dim] : -INFINITY, sum = lane < n ? part[(int64_t)lane * wide + a.dim + 1] : 0.0f;
    float most = top;
#pragma unroll
    for (int s = 8; s >= 1; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    most = __shfl(most, 0);
    const float factor = __builtin_amdgcn_exp2f(top - (most == -INFINITY ? 0.0f : most)), l = wave_sum(sum * factor);
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    const int d0 = min(lane, a.dim - 1), d1 = min(lane + 64, a.dim - 1);
    float o0 = 0.0f, o1 = 0.0f;
#pragma unroll 4
    for (int p = 0; p < n; ++p) {
        const float f = __shfl(factor, p);
        o0 = fmaf(part[(int64_t)p * wide + d0], f, o0);
        o1 = fmaf(part[(int64_t)p * wide + d1], f, o1);
    }
    if (a.lse && lane == 0) a.lse[(int64_t)head * a.q_rows + rows.q0 + query] = l == 0.0f ? -INFINITY : (most + __builtin_amdgcn_logf(l)) * GBT_LN2;
    auto put = [&](int d, float x) {
        if (d >= a.dim) return;
        const E y = (E)x;
        ((E *)a.out.data)[(rows.q0 + query) * a.out.row + (int64_t)head * a.out.head + d] = y;
        if (a.rest) ((E *)a.rest)[((rows.q0 + query) * a.heads + head) * a.dim + d] = (E)(x - (float)y);
    };
    put(lane, o0 * inv);
    put(lane + 64, o1 * inv);
}

template <typename P, int DP>
hipError_t launch(hipStream_t stream, const AttnArgs &a, const AttnCuts &c) {
    const AttnForm form = attn_form(a, DP, false);
    const int64_t blocks = (a.max_q + form.queries - 1) / form.queries;
    AttnArgs b = a;
    b.order = attn_order(a, a.heads, blocks, true);
    b.work = attn_grid(b.order);
    const unsigned grid = b.work + attn_gap_workgroups(a, true, false);
    if (grid == 0) return hipSuccess;
    if (form.queries == 64) attention_kernel<P, DP, 2, 2, 1><<<grid, 256, 0, stream>>>(b, c);
    else if (a.max_k <= kFewKeys) attention_kernel<P, DP, 4, 1, 2><<<grid, 256, 0, stream>>>(b, c);   // which attn_form gives one group
    else if (form.groups == 1) attention_kernel<P, DP, 4, 1, 1><<<grid, 256, 0, stream>>>(b, c);
    else if constexpr (DP > 64) attention_kernel<P, DP, 4, 2, 1><<<grid, 512, 0, stream>>>(b, c);
    return hipGetLastError();
}

template <typename P, int DP>
hipError_t launch_few(hipStream_t stream, const AttnArgs &a, const AttnCuts &c) {
    const int64_t columns = (int64_t)a.group * a.max_q;
    AttnArgs b = a;
    b.work = (unsigned)((int64_t)a.pieces * a.kv_heads * a.n_seq);
    attention_few_kernel<P, DP><<<b.work + attn_gap_workgroups(a, true, false), 256, a.n_buckets * 32 * sizeof(float), stream>>>(b, c);
    if (a.pieces > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const unsigned all = (unsigned)(columns * a.kv_heads * a.n_seq);
        if (a.pieces <= kFewJoined) attention_join_few_kernel<P><<<(all + 3) / 4, 256, 0, stream>>>(a);
        else attention_join_kernel<P><<<all, 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}

template <typename P>
hipError_t by_dim(hipStream_t stream, const AttnArgs &a, const AttnCuts &c, bool few) {
    if (a.dim <= 32) return few ? launch_few<P, 32>(stream, a, c) : launch<P, 32>(stream, a, c);
    if (a.dim <= 64) return few ? launch_few<P, 64>(stream, a, c) : launch<P, 64>(stream, a, c);
    if (a.dim <= 96) return few ? launch_few<P, 96>(stream, a, c) : launch<P, 96>(stream, a, c);
    return few ? launch_few<P, 128>(stream, a, c) : launch<P, 128>(stream, a, c);
}

}  // namespace

hipError_t gbt_launch_attention(hipStream_t stream, const AttnArgs &a, const AttnCuts &c, int dtype) {
    return dtype == GBT_BF16 ? by_dim<Bf16>(stream, a, c, false) : by_dim<F16>(stream, a, c, false);
}
hipError_t gbt_launch_attention_few(hipStream_t stream, const AttnArgs &a, const AttnCuts &c, int dtype) {
    return dtype == GBT_BF16 ? by_dim<Bf16>(stream, a, c, true) : by_dim<F16>(stream, a, c, true);
}
