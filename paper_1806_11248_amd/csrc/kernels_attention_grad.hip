// Attention's backward pass.  Probabilities are recomputed from the rows' statistics, so nothing of size queries x keys is stored:
//
//   P_ij = exp(S_ij - lse_i)   delta_i = dout_i . out_i   dP_ij = dout_i . v_j   dS_ij = P_ij (dP_ij - delta_i)
//   dq_i = scale sum_j dS_ij k_j   dk_j = scale sum_i dS_ij q_i   dv_j = sum_i P_ij dout_i   dbias[b] = sum of dS over t in bucket b
//
// Two kernels, each owning what it sums: one the queries (dq, and delta), one the keys (dk and dv, over all heads that share them, and the
// bias gradient).  Recomputing S and dP twice costs seven products in place of five; it needs no atomics, so every result
// is the same on every run, and a wave keeps all of its sums in registers.
//
// delta.  With `rest`, what rounding took from out, dout . (out + rest) is off by the rounding of the probabilities in out alone: too
// little to show in dq, whose dS are rounded as much, but it would be the largest error by far of the bias gradient, which is a
// 32-bit result.  Since sum_j P_ij = 1, the row sums of the dS so computed are just that error: the first kernel adds them to its delta,
// and the second works with sums of P dP as exact as 32 bits allow.  (Relative error of the bias gradient in bfloat16 with delta of out
// and rest 7e-4, with the row sums 2e-7 .. 5e-7; of dq, rows of 5 .. 60 keys, without rest 2.8e-3, with it 2.35e-3.)
//
// Bound: as the forward kernel's, matrix units and the arithmetic between the products.  Two causal histories of 4096, 16 heads of 128 elements on 4 key
// heads: queries 245 us, 843 TFLOP/s of its three products, matrix units busy 45%; keys 414 us, 665 of its four, busy 35%: its waves keep 128 sums each and
// meet at a barrier every 64 queries, so they do the same at the same time; joining the parts 17 us (83 MB).  16 histories of 100 to 1000 rows, 8 heads of
// 64: 42 + 60 + 4.5 us.
#include "attention.h"

#include <type_traits>

namespace {

// One step of a sum over equal buckets of neighbouring lanes (a lane's bucket is never below that of the lane before): what the lane that CTRL
// names has summed, where it is of the same bucket.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ void run_step(float &v, int bucket) {
    const int w = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROW_MASK, 0xf, false);
    const int b = __builtin_amdgcn_update_dpp(-1, bucket, CTRL, ROW_MASK, 0xf, false);
    v += b == bucket ? __builtin_bit_cast(float, w) : 0.0f;
}
// Adds each run's sum to its bucket: shifts by 1, 2, 4, 8 inside each row of 16 lanes, lane 15 of rows 0 and 2 into rows 1 and 3, lane 31 into rows
// 2 and 3.  `next` is the bucket of the lane behind.
__device__ __forceinline__ void add_runs(float *sums, float v, int bucket, int next, int lane) {
    run_step<0x111, 0xf>(v, bucket);
    run_step<0x112, 0xf>(v, bucket);
    run_step<0x114, 0xf>(v, bucket);
    run_step<0x118, 0xf>(v, bucket);
    run_step<0x142, 0xa>(v, bucket);
    run_step<0x143, 0xc>(v, bucket);
    if (lane == 63 || next != bucket) sums[bucket] += v;
    __builtin_amdgcn_wave_barrier();
}

// The sums of lo and hi over all lanes, in lanes 31 and 63: halves first, so that each half of the wave has one of the two.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ void sum_step(float &v) {
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROW_MASK, 0xf, false));
}
__device__ __forceinline__ float pair_sum(float lo, float hi) {
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, lo), __builtin_bit_cast(int, hi), false, false);
    float v = __builtin_bit_cast(float, (int)both[0]) + __builtin_bit_cast(float, (int)both[1]);
    sum_step<0x111, 0xf>(v);
    sum_step<0x112, 0xf>(v);
    sum_step<0x114, 0xf>(v);
    sum_step<0x118, 0xf>(v);
    sum_step<0x142, 0xa>(v);
    return v;
}

// float16's normal numbers are 2^-14 to 2^16.  Probabilities of many keys, and dS of many keys or of a small dout, are below, dS of a large
// dout above, while what the products add up to is neither.  There probabilities, which are at most 1 but for rounding, are held times 2^kLift, which costs
// nothing in the exponent, and so are dS.  Where one of a column's dS would pass 2^15 as an operand, all of the column's
// are lowered by a power of two, so that this one is some 2^12, and the column's sums with them.  (Relative error of dq of 2048 keys, 64 elements a head,
// with a dout of size 2^-10: 2.8e-3 without, 5.3e-4 with it, of which rounding the result to float16 is 4.8e-4; without, any dS from 65520 on made
// infinities and NaN of finite gradients.  24 histories of 100 to 1000 rows, 8 heads of 64, the backward pass 178 and 177 us; 12 of 700, 6 heads of 80, 101
// and 105.)
template <typename P>
constexpr float kLift = P::kNarrow ? 10.0f : 0.0f;
template <typename P>
constexpr float kLiftDown = P::kNarrow ? 0x1p-10f : 1.0f;   // 2^-kLift
constexpr float kOperandMost = 0x1p15f;
__device__ __forceinline__ float column_most(const f32x16 &x) {
    float most = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(x[r]));
    return column_max(most);
}
// The exponent, as a float has it, of the power of two that brings what is too large down to 2^12 .. 2^13.
__device__ __forceinline__ int lower_by(float most) { return most > kOperandMost ? 266 - (__builtin_bit_cast(int, most) >> 23) : 127; }
template <int N>
__device__ __forceinline__ void scale_all(f32x16 (&x)[N], float by) {
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[b][r] *= by;
}

// ---------------------------------------------------------------------------------------------------------- queries --
// As the forward kernel: 128 or 64 queries of one head, 32 a wave, keys and values through LDS, one group of waves or two.
template <typename P, int DP, int kQWaves, int kGroups>
__global__ __launch_bounds__(64 * kQWaves * kGroups, 2) void grad_queries_kernel(AttnArgs a, AttnCuts c) {
    typedef typename P::elem E;
    typedef typename P::vec8 V8;
    typedef Tile<DP> T;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32, kStride = 64 * kGroups, kQueries = 32 * kQWaves, kWaves = kQWaves * kGroups;
    __shared__ __align__(16) char k_tile[2][kGroups * T::kBytes];
    __shared__ __align__(16) char v_tile[2][kGroups * T::kBytes];
    __shared__ DistanceRing<256 * kGroups> ring;

    if (blockIdx.x >= a.work) {
        zero_gaps(a, a.dq, false);
        zero_gaps(a, a.dk, true);
        return zero_gaps(a, a.dv, true);
    }
    const AttnItem item = attn_item(a);
    if (item.seq < 0) return;
    const int block = a.order.blocks - 1 - item.block, head = item.unit, seq = item.seq;
    const AttnSeq rows = attn_seq(a, seq);
    const int first = block * kQueries;
    const bool bias = a.n_buckets > 0;
    if (first >= rows.nq) return;
    const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int wave = kGroups == 2 ? any_wave % kQWaves : any_wave, group = kGroups == 2 ? any_wave / kQWaves : 0;
    const int off = rows.nk - rows.nq;
    const int query = first + wave * 32 + (lane & 31);
    const bool there = query < rows.nq;
    const int last = a.causal ? min(rows.nk - 1, query + off) : rows.nk - 1;
    const int end = a.causal ? min(rows.nk, min(first + kQueries, rows.nq) + off) : rows.nk;
    const int wave_first = first + wave * 32;
    const int wave_end = wave_first >= rows.nq ? 0 : a.causal ? min(rows.nk, min(wave_first + 32, rows.nq) + off) : rows.nk;
    const int wave_all = a.causal ? min(rows.nk, wave_first + off + 1) : rows.nk;

    const int kv_head = head / a.group;
    const char *k_base = a.k.data + (rows.k0 * a.k.row + (int64_t)kv_head * a.k.head) * 2;
    const char *v_base = a.v.data + (rows.k0 * a.v.row + (int64_t)kv_head * a.v.head) * 2;

    auto fetch = [&](int n, int kb) {
        T::template fetch<true, kQWaves>(k_tile[n] + group * T::kBytes, k_base + (int64_t)kb * a.k.row * 2, (uint32_t)a.k.row * 2, end - kb, a.dim, wave);
        T::template fetch<true, kQWaves>(v_tile[n] + group * T::kBytes, v_base + (int64_t)kb * a.v.row * 2, (uint32_t)a.v.row * 2, end - kb, a.dim, wave);
    };
    if (64 * group < end) fetch(0, 64 * group);
    const int64_t row = rows.q0 + min(query, rows.nq - 1);
    V8 qf[kSteps], gf[kSteps];
    float delta = 0.0f, lse = a.lse[(int64_t)head * a.q_rows + row] * GBT_LOG2E;
    load_row(qf, a.q.data + (row * a.q.row + (int64_t)head * a.q.head) * 2, half, a.dim);
    load_row(gf, a.dout.data + (row * a.dout.row + (int64_t)head * a.dout.head) * 2, half, a.dim);
    {
        V8 o[kSteps], r[kSteps];
        load_row(o, a.out.data + (row * a.out.row + (int64_t)head * a.out.head) * 2, half, a.dim);
        // without `rest`, out once more, with a factor of zero
        const bool rest = a.rest != nullptr;
        load_row(r, rest ? a.rest + (row * a.heads + head) * a.dim * 2 : a.out.data + (row * a.out.row + (int64_t)head * a.out.head) * 2, half, a.dim);
        if (bias) {
            ring_cuts(ring, a, c);
            ring_head(ring, a, head);
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[s][e], (float)o[s][e] + (rest ? (float)r[s][e] : 0.0f), delta);
    }
    delta = column_sum(delta);
    // a query that does not exist, or saw no key: its probabilities are 2^-inf
    const float minus = !there || lse == -INFINITY ? -INFINITY : -lse;
    f32x16 dq[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[b][r] = 0.0f;
    float row_sum = 0.0f;   // of dS: this lane's half of the column
    float lift = kLift<P>;  // dS, and the sums of them, are held times 2^lift
    arrived(qf);
    arrived(gf);
    __syncthreads();
    if (bias && any_wave < kQWaves / 2 + kGroups) ring_put(ring, 64 * any_wave - (first + kQueries - 1 + off), any_wave, lane);

    auto step = [&](auto which, int k0) {
        constexpr int kNow = decltype(which)::value;
        const char *k_now = k_tile[kNow] + group * T::kBytes, *v_now = v_tile[kNow] + group * T::kBytes;
        const int kb = k0 + 64 * group;
        tiles_ready();
        if (kb + kStride < end) fetch(1 - kNow, kb + kStride);
        const int lowest = k0 - (first + kQueries - 1 + off);
        const int turn = (any_wave - (k0 >> 6)) & (kWaves - 1);
        if (bias && turn < kGroups) ring_put(ring, lowest + kQueries - 1 + kStride + 64 * turn, any_wave, lane);
        if (kb >= wave_end) return;

#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int at = (lowest & ring.kMask) + 64 * group + kQueries - 32 - 32 * wave + 32 * b;   // of this 32 x 32 result's lowest distance, of 63
            const int b0 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at]) : 0, b1 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at + 62]) : 0;
            __builtin_amdgcn_s_setprio(1);   // products before the other waves' arithmetic
            f32x16 s, dp;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = 0.0f;
                dp[r] = -delta;
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                s = P::mma(T::template rows<P>(k_now, 32 * b, i, lane), qf[i], s);
                dp = P::mma(T::template rows<P>(v_now, 32 * b, i, lane), gf[i], dp);
            }
            // reads two products ahead
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int i = 0; i < kSteps - 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            const float lifted = P::kNarrow ? minus + lift : minus;
            if (b0 == b1) {
                const float add = (bias ? ring.of_bucket[b0] : 0.0f) + lifted;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, add));
            } else {
                const float *add = ring.value + at + 31 - (lane & 31);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, add[result_row(r, half)] + lifted));
            }
            if (kb + 32 * b + 32 > wave_all) {
                const int past = last - (kb + 32 * b) - 4 * half;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = result_row(r, 0) <= past ? s[r] : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] *= dp[r];
                row_sum += s[r];
            }
            if constexpr (P::kNarrow) {
                const float most = column_most(s);
                if (__any(most > kOperandMost)) {
                    const int to = lower_by(most);
                    const float by = __builtin_bit_cast(float, to << 23);
                    lift += (float)(to - 127);
                    row_sum *= by;
                    s *= by;
                    scale_all(dq, by);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const V8 ds = operand<P>(s, i);
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) dq[d] = P::mma(T::template cols<P>(k_now, 32 * b + 16 * i, d, lane), ds, dq[d]);
            }
        }
    };
    for (int k0 = 0; k0 < end; k0 += 2 * kStride) {
        step(std::integral_constant<int, 0>{}, k0);
        if (k0 + kStride < end) step(std::integral_constant<int, 1>{}, k0 + kStride);
    }
    if constexpr (P::kNarrow) {
        const float down = __builtin_ldexpf(1.0f, -(int)lift);
        row_sum *= down;
        scale_all(dq, down);
    }
    if constexpr (kGroups == 2) {   // the second group's sums to the first, through LDS
        float *theirs = (float *)(wave < 2 ? &k_tile[0][0] : &v_tile[0][0]) + (wave & 1) * (16 * kBlocks + 1) * 64 + lane;
        static_assert(2 * (16 * kBlocks + 1) * 256 <= (int)sizeof k_tile, "two waves' sums fit where the keys were");
        __syncthreads();
        if (group == 1) {
#pragma unroll
            for (int i = 0; i < 16 * kBlocks; ++i) theirs[64 * i] = dq[i / 16][i % 16];
            theirs[64 * 16 * kBlocks] = row_sum;
        }
        __syncthreads();
        if (group == 1) return;
        row_sum += theirs[64 * 16 * kBlocks];
#pragma unroll
        for (int i = 0; i < 16 * kBlocks; ++i) dq[i / 16][i % 16] += theirs[64 * i];
    }
    row_sum = column_sum(row_sum);
    if (!there) return;
    if (half == 0) {
        const int64_t at = (int64_t)head * a.q_rows + rows.q0 + query;
        a.row_less[at] = P::kNarrow ? minus + kLift<P> : minus;
        a.row_minus[at] = -(delta + row_sum);
    }
    E *out = (E *)a.dq.data + (rows.q0 + query) * a.dq.row + (int64_t)head * a.dq.head;
    typedef E E4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * b + 8 * g + 4 * half;
            if (d < a.dim) {
                E4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (E)(dq[b][4 * g + e] * a.scale);
                *(E4 *)(out + d) = x;
            }
        }
}

// ------------------------------------------------------------------------------------------------------------- keys --
// A workgroup takes 128 keys of one key head, a wave 32 of them (its columns); the queries of the heads that share them pass through LDS with
// their output gradients, 64 at a time.  Products of gradients with values start from -delta instead of zero.  (Products of scores that start from
// -lse / scale likewise save an addition each, but their sums are then some ten times as large and rounded as much more coarsely: the bias gradient
// was twice as far off.)  Where there are few blocks of keys, several workgroups share one, by heads and by
// queries, and their sums are added up by a kernel of its own.
//
// Bias gradient.  A 32 x 32 result all of whose distances are in one bucket adds to one running sum in each lane, one with a single cut among them to
// two, which are added up over the lanes.  Others are laid out by diagonals in LDS, eight rows at a time, and added up along them (63 distances, one a lane), and then over each run of lanes of one bucket.
template <typename P, int DP, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void grad_keys_kernel(AttnArgs a, AttnCuts c) {
    typedef typename P::elem E;
    typedef typename P::vec8 V8;
    typedef Tile<DP> T;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32, kThreads = 64 * kWaves;
    constexpr bool kValuesInLds = kWaves == 8 && DP == 128;
    __shared__ __align__(256) char tiles[2][2][T::kBytes];   // of queries and of output gradients, two of each in turn
    __shared__ __align__(256) char v_block[kValuesInLds ? 2 * T::kBytes : 16];
    __shared__ __align__(16) float row_less[2][64], row_minus[2][64];
    __shared__ DistanceRing<256> ring;
    __shared__ float sums[kWaves][kAttnBuckets];   // the head's bias gradient of this workgroup's keys, by wave
    __shared__ float skew[kWaves][8 * 64];         // [query][key - query + 31]: eight rows of a result by its diagonals

    const int k_blocks = a.order.blocks, parts = a.head_parts * a.q_parts;
    const AttnItem item = attn_item(a);
    if (item.seq < 0) return;
    const int part = item.unit % parts, kv_head = item.unit / parts, seq = item.seq;
    const int q_part = part % a.q_parts, head_part = part / a.q_parts;
    const int g_from = a.group * head_part / a.head_parts, g_to = a.group * (head_part + 1) / a.head_parts;
    const AttnSeq rows = attn_seq(a, seq);
    // a causal block of keys has as many queries to meet as lie behind it: counted from the sequence's end, the same for all of one turn
    int block = item.block;
    if (a.causal) {
        block -= k_blocks - (rows.nk + kAttnQueries - 1) / kAttnQueries;
        if (block < 0) block += k_blocks;
    }
    const int first = block * kAttnQueries;
    const bool bias = a.n_buckets > 0;
    auto strip = [&](int head) {
        return a.strips + (((int64_t)head * a.n_seq + seq) * k_blocks * a.q_parts + (int64_t)block * a.q_parts + q_part) * a.n_buckets;
    };
    if (first >= rows.nk) {
        for (int g = g_from; g < g_to; ++g)
            for (int i = threadIdx.x; i < a.n_buckets; i += kThreads) strip(kv_head * a.group + g)[i] = 0.0f;
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int key_wave = wave & 3;   // of eight waves, 4 .. 7 take the second half of each tile for the keys of 0 .. 3
    const int off = rows.nk - rows.nq;
    const int key = first + key_wave * 32 + (lane & 31);
    const bool there = key < rows.nk;
    if (bias) {
        ring_cuts(ring, a, c);
        for (int i = threadIdx.x; i < kWaves * 8 * 64; i += kThreads) (&skew[0][0])[i] = 0.0f;
    }

    V8 kf[kSteps], vf[kValuesInLds ? 1 : kSteps];
    {
        const int64_t row = rows.k0 + min(key, rows.nk - 1);
        load_row(kf, a.k.data + (row * a.k.row + (int64_t)kv_head * a.k.head) * 2, half, a.dim);
        if constexpr (!kValuesInLds) load_row(vf, a.v.data + (row * a.v.row + (int64_t)kv_head * a.v.head) * 2, half, a.dim);
        if constexpr (kValuesInLds) {
            const int row = first + 64 * (wave >> 2);
            if (row < rows.nk)
                T::fetch(v_block + (wave >> 2) * T::kBytes, a.v.data + ((rows.k0 + row) * a.v.row + (int64_t)kv_head * a.v.head) * 2, (uint32_t)a.v.row * 2,
                         rows.nk - row, a.dim, key_wave);
        }
    }
    arrived(kf);
    if constexpr (!kValuesInLds) {
        arrived(vf);
    } else if (a.dim < DP) {   // elements past the head's, which the other operand has copies of
        tiles_ready();
        for (int i = threadIdx.x; i < 128 * T::kPlaces; i += kThreads)
            if ((i % T::kPlaces ^ T::fold(i / T::kPlaces)) >= a.dim / 8) *(i32x4 *)(v_block + 16 * i) = i32x4{0, 0, 0, 0};
    }
    auto values = [&](uint32_t base, int i) {
        if constexpr (kValuesInLds) return T::template rows_at<P>(base, i, 0);
        else return vf[i];
    };
    f32x16 dk[kBlocks], dv[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.0f;
    float low = 1.0f;   // dk is of dS times this and 2^kLift; probabilities, dv and the bias gradient's sums are held times 2^kLift

    // queries from here on see one of the workgroup's keys; this workgroup takes its part of them, in whole tiles
    const int seen = a.causal ? max(0, first - off) & ~63 : 0, n_tiles = max(0, (rows.nq - seen + 63) >> 6);
    const int from = seen + 64 * (int)((int64_t)n_tiles * q_part / a.q_parts), to = min(rows.nq, seen + 64 * (int)((int64_t)n_tiles * (q_part + 1) / a.q_parts));
    const int sees = a.causal ? key - off : 0;                         // the first query that sees this lane's key
    const int wave_from = a.causal ? first + key_wave * 32 - off : 0;      // and one of the wave's,
    const int wave_all = a.causal ? first + key_wave * 32 + 31 - off : 0;  // and all of them
    const bool wave_last = first + key_wave * 32 + 32 > rows.nk;           // some of the wave's keys do not exist

    for (int g = g_from; g < g_to; ++g) {
        const int head = kv_head * a.group + g;
        const char *q_base = a.q.data + (rows.q0 * a.q.row + (int64_t)head * a.q.head) * 2;
        const char *g_base = a.dout.data + (rows.q0 * a.dout.row + (int64_t)head * a.dout.head) * 2;
        const int64_t at_row = (int64_t)head * a.q_rows + rows.q0;
        __syncthreads();   // the head before is done with the values, the ring and the sums
        float run = 0.0f;  // this lane's part of the sum over results of one bucket
        int run_bucket = 0;
        auto fetch = [&](int n, int qb) {
            if (kWaves == 4 || wave < 4) T::template fetch<DP <= 64>(tiles[n][0], q_base + (int64_t)qb * a.q.row * 2, (uint32_t)a.q.row * 2, rows.nq - qb, a.dim, key_wave);
            if (kWaves == 4 || wave >= 4) T::template fetch<DP <= 64>(tiles[n][1], g_base + (int64_t)qb * a.dout.row * 2, (uint32_t)a.dout.row * 2, rows.nq - qb, a.dim, key_wave);
            const uint32_t at = min(lane, rows.nq - qb - 1) * 4;
            if (wave == 0) load_word_to_lds(lds_address(row_less[n]), a.row_less + at_row + qb, at);
            if (wave == 1) load_word_to_lds(lds_address(row_minus[n]), a.row_minus + at_row + qb, at);
        };
        if (from < to) fetch(0, from);
        if (bias) {
            ring_head(ring, a, head);
            for (int i = threadIdx.x; i < kWaves * kAttnBuckets; i += kThreads) (&sums[0][0])[i] = 0.0f;
        }
        __syncthreads();
        if (bias && wave < 3) ring_put(ring, 64 * wave + first - (from + 63 + off), wave, lane);

        int now = 0;   // which of the two copies; not known at compile time as in the other kernels, which would cost registers
        for (int qb = from; qb < to; qb += 64, now ^= 1) {
            tiles_ready();
            if (qb + 64 < to) fetch(1 - now, qb + 64);
            const int lowest = first - (qb + 63 + off);
            if (bias && wave == ((qb >> 6) & (kWaves - 1))) ring_put(ring, lowest - 64, wave, lane);
#pragma unroll 1
            for (int turn = 0; turn < 8 / kWaves; ++turn) {
                const int b = kWaves == 8 ? wave >> 2 : turn;
                int here = lane;   // at large heads, LDS addresses are worked out each time: registers again
                if (DP > 64) asm volatile("" : "+v"(here));
                const int half = here >> 5;
                if (qb + 32 * b + 31 < wave_from || qb + 32 * b >= rows.nq) continue;
                const int at = (lowest & 255) + 32 * key_wave + 32 - 32 * b;   // of this result's lowest distance, of 63
                const int b0 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at]) : 0, b1 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at + 62]) : 0;
                const uint32_t rows_here = T::rows_base(tiles[now][0], 32 * b, here);
                const uint32_t values_here = kValuesInLds ? T::rows_base(v_block, 32 * key_wave, here) : 0;
                f32x16 s, dp;
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    const f32x4 d = *(const f32x4 *)(row_minus[now] + 32 * b + 8 * r4 + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[4 * r4 + e] = 0.0f;
                        dp[4 * r4 + e] = d[e];
                    }
                }
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    s = P::mma(T::template rows_at<P>(rows_here, i, 0), kf[i], s);
                    dp = P::mma(T::template rows_at<P>(rows_here, i, T::kBytes), values(values_here, i), dp);
                }
                // reads two products ahead, and no further: registers are what there is least of
                constexpr int kReads = kValuesInLds ? 3 : 2;
                __builtin_amdgcn_sched_group_barrier(0x100, 4 + 2 * kReads, 0);
#pragma unroll
                for (int i = 0; i < kSteps - 2; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
                __builtin_amdgcn_sched_barrier(0);
                const float *less = row_less[now] + 32 * b + 4 * half;
                if (b0 == b1) {
                    const float add = bias ? ring.of_bucket[b0] : 0.0f;
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4) {
                        const f32x4 l = *(const f32x4 *)(less + 8 * r4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[4 * r4 + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * r4 + e], a.scale2, add + l[e]));
                    }
                } else {
                    const float *add = ring.value + at + 31 + (here & 31);
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4) {
                        const f32x4 l = *(const f32x4 *)(less + 8 * r4);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[4 * r4 + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * r4 + e], a.scale2, add[-result_row(4 * r4 + e, half)] + l[e]));
                    }
                }
                if (qb + 32 * b < wave_all || qb + 32 * b + 32 > rows.nq) {   // rows past the last are the last one's copies
                    const int since = sees - (qb + 32 * b) - 4 * half, past = rows.nq - (qb + 32 * b) - 4 * half;
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = result_row(r, 0) >= since && result_row(r, 0) < past ? s[r] : 0.0f;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] *= s[r];
                // a key beyond the last has scores of its bias alone
                if (bias && wave_last) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) dp[r] = there ? dp[r] : 0.0f;
                }
                if (bias && b0 == b1) {
                    if (b0 != run_bucket) {
                        const float v = pair_sum(run, 0.0f);
                        if (lane == 31) sums[wave][run_bucket] += v;
                        __builtin_amdgcn_wave_barrier();
                        run = 0.0f;
                        run_bucket = b0;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) run += dp[r];
                } else if (bias && b1 == b0 + 1) {
                    // one cut among the result's 63 distances, of which a row's in this lane's column is the (31 + column - row)-th
                    const int distance = first + 32 * key_wave - (qb + 32 * b + 31 + off);   // the lowest
                    const int rows_above = 31 + (here & 31) - (ring.cut[b0] - distance) - 4 * half;
                    float lo = 0.0f, hi = 0.0f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool above = result_row(r, 0) <= rows_above;
                        hi += above ? dp[r] : 0.0f;
                        lo += above ? 0.0f : dp[r];
                    }
                    const float v = pair_sum(lo, hi);
                    if ((here & 31) == 31) sums[wave][b0 + half] += v;
                    __builtin_amdgcn_wave_barrier();
                } else if (bias) {
                    float *sk = skew[wave], v = 0.0f;
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) sk[result_row(r, half) * 63 + 31 + (here & 31)] = dp[4 * h + r];
                        __builtin_amdgcn_wave_barrier();
                        // eight rows further on, the same diagonal lies eight places further on; place 63 is never written
#pragma unroll
                        for (int i = 0; i < 8; ++i) v += sk[64 * i + min(here + 8 * h, 63)];
                        __builtin_amdgcn_wave_barrier();
                    }
                    add_runs(sums[wave], v, ring.bucket[at + min(here, 62)], ring.bucket[at + min(here + 1, 62)], here);
                }
                if constexpr (P::kNarrow) {
                    const float most = column_most(dp);
                    if (__any(most > kOperandMost || low != 1.0f)) {
                        const float by = __builtin_bit_cast(float, lower_by(most * low) << 23);
                        if (__any(by != 1.0f)) scale_all(dk, by);
                        low *= by;
                        dp *= low;
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                const uint32_t cols_here = T::cols_base(tiles[now][0], 32 * b, here);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const V8 p = operand<P>(s, i), ds = operand<P>(dp, i);
#pragma unroll
                    for (int d = 0; d < kBlocks; ++d) {
                        dv[d] = P::mma(T::template cols_at<P>(cols_here, 16 * i, d, T::kBytes), p, dv[d]);
                        dk[d] = P::mma(T::template cols_at<P>(cols_here, 16 * i, d, 0), ds, dk[d]);
                    }
                }
                __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                for (int i = 0; i < 4 * kBlocks - 2; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (bias) {
            const float v = pair_sum(run, 0.0f);
            if (lane == 31) sums[wave][run_bucket] += v;
            __syncthreads();
            for (int i = threadIdx.x; i < a.n_buckets; i += kThreads) {
                float v = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
                if (kWaves == 8) v += (sums[kWaves - 4][i] + sums[kWaves - 3][i]) + (sums[kWaves - 2][i] + sums[kWaves - 1][i]);
                strip(head)[i] = v * kLiftDown<P>;
            }
        }
    }
    if constexpr (kValuesInLds) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the values, if nobody has read them
    if constexpr (P::kNarrow) {
        scale_all(dk, kLiftDown<P> / low);
        scale_all(dv, kLiftDown<P>);
    }
    if constexpr (kWaves == 8) {   // the two halves' sums together, through LDS; 0 .. 3 hold them then
        float *mine = (float *)&tiles[0][0][0] + key_wave * kBlocks * 16 * 64 + lane;
        auto join = [&](f32x16 (&x)[kBlocks]) {
            __syncthreads();
            if (wave >= 4) {
#pragma unroll
                for (int i = 0; i < 16 * kBlocks; ++i) mine[64 * i] = x[i / 16][i % 16];
            }
            __syncthreads();
            if (wave < 4) {
#pragma unroll
                for (int i = 0; i < 16 * kBlocks; ++i) x[i / 16][i % 16] += mine[64 * i];
            }
        };
        join(dk);
        join(dv);
        if (wave >= 4) return;
    }
    if (!there) return;
    if (parts > 1) {
        const int64_t tensor = a.part_rows * a.kv_heads * a.dim;
        float *ko = a.part + 2 * part * tensor + ((attn_part_row(a, seq, rows) + key) * a.kv_heads + kv_head) * a.dim, *vo = ko + tensor;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const int d = 32 * b + 8 * r4 + 4 * half;
                if (d < a.dim) {
                    *(f32x4 *)(ko + d) = f32x4{dk[b][4 * r4], dk[b][4 * r4 + 1], dk[b][4 * r4 + 2], dk[b][4 * r4 + 3]};
                    *(f32x4 *)(vo + d) = f32x4{dv[b][4 * r4], dv[b][4 * r4 + 1], dv[b][4 * r4 + 2], dv[b][4 * r4 + 3]};
                }
            }
        return;
    }
    E *ko = (E *)a.dk.data + (rows.k0 + key) * a.dk.row + (int64_t)kv_head * a.dk.head;
    E *vo = (E *)a.dv.data + (rows.k0 + key) * a.dv.row + (int64_t)kv_head * a.dv.head;
    typedef E E4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const int d = 32 * b + 8 * r4 + 4 * half;
            if (d < a.dim) {
                E4 x, y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = (E)(dk[b][4 * r4 + e] * a.scale);
                    y[e] = (E)dv[b][4 * r4 + e];
                }
                *(E4 *)(ko + d) = x;
                *(E4 *)(vo + d) = y;
            }
        }
}

// The last launch: the parts of the keys' gradients together, a workgroup taking sixteen key rows of a sequence and a thread four elements of
// one; and behind those workgroups, one for each head, the strips of the bias gradient, in a fixed order: 2^k threads a bucket, which are then added
// up in pairs.  (One launch in place of two: 4 us of some 90 for five histories of 300 to 800 rows.)
constexpr int kJoinRows = 16;
__device__ __forceinline__ void add_strips(const AttnArgs &a, int head) {
    __shared__ double part[1024];
    const int n = a.n_buckets, lanes = 1 << (31 - __clz(1024 / n));
    const int64_t strips = (int64_t)a.n_seq * ((a.max_k + kAttnQueries - 1) / kAttnQueries) * a.q_parts;
    const float *from = a.strips + (int64_t)head * strips * n;
    const int b = threadIdx.x % n, l = threadIdx.x / n;
    double sum = 0.0;
    if (l < lanes) {
#pragma unroll 8
        for (int64_t s = l; s < strips; s += lanes) sum += from[s * n + b];
    }
    part[threadIdx.x] = sum;
    for (int w = lanes / 2; w > 0; w /= 2) {
        __syncthreads();
        if (l < w) part[threadIdx.x] += part[threadIdx.x + w * n];
    }
    if (l == 0) a.dbias[(int64_t)b * a.heads + head] = (float)part[threadIdx.x];
}
template <typename P>
__global__ __launch_bounds__(1024) void grad_join_kernel(AttnArgs a) {
    typedef typename P::elem E;
    typedef E E4 __attribute__((ext_vector_type(4)));
    if (blockIdx.x >= a.work) return add_strips(a, blockIdx.x - a.work);
    const int row_blocks = (a.max_k + kJoinRows - 1) / kJoinRows, seq = blockIdx.x / row_blocks, first = blockIdx.x % row_blocks * kJoinRows;
    const AttnSeq rows = attn_seq(a, seq);
    if (first >= rows.nk) return;
    const int wide = a.kv_heads * a.dim / 4, parts = a.head_parts * a.q_parts;
    const int64_t tensor = a.part_rows * a.kv_heads * a.dim, part_row = attn_part_row(a, seq, rows) + first;
    for (int i = threadIdx.x; i < min(kJoinRows, rows.nk - first) * wide; i += 1024) {
        const int64_t row = rows.k0 + first + i / wide;
        const int e = i % wide * 4, kv_head = e / a.dim, d = e % a.dim;
        const float *from = a.part + (part_row + i / wide) * a.kv_heads * a.dim + e;
        f32x4 k = {0.0f, 0.0f, 0.0f, 0.0f}, v = k;
#pragma unroll 4
        for (int p = 0; p < parts; ++p) {
            k += *(const f32x4 *)(from + 2 * p * tensor);
            v += *(const f32x4 *)(from + (2 * p + 1) * tensor);
        }
        E4 x, y;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = (E)(k[j] * a.scale);
            y[j] = (E)v[j];
        }
        *(E4 *)((E *)a.dk.data + row * a.dk.row + (int64_t)kv_head * a.dk.head + d) = x;
        *(E4 *)((E *)a.dv.data + row * a.dv.row + (int64_t)kv_head * a.dv.head + d) = y;
    }
}

template <typename P, int DP>
hipError_t launch(hipStream_t stream, const AttnArgs &a, const AttnCuts &c) {
    const AttnForm form = attn_form(a, DP, true);
    const int64_t q_blocks = (a.max_q + form.queries - 1) / form.queries, k_blocks = (a.max_k + kAttnQueries - 1) / kAttnQueries;
    hipError_t e = hipSuccess;
    {
        AttnArgs b = a;
        b.order = attn_order(a, a.heads, q_blocks, true);
        b.work = attn_grid(b.order);
        const unsigned grid = b.work + attn_gap_workgroups(a, true, true);
        if (grid == 0) {
        } else if (form.queries == 64) grad_queries_kernel<P, DP, 2, 2><<<grid, 256, 0, stream>>>(b, c);
        else if (form.groups == 1) grad_queries_kernel<P, DP, 4, 1><<<grid, 256, 0, stream>>>(b, c);
        else if constexpr (DP == 96) grad_queries_kernel<P, DP, 4, 2><<<grid, 512, 0, stream>>>(b, c);
        e = hipGetLastError();
    }
    if (e == hipSuccess && k_blocks > 0 && a.n_seq > 0) {
        constexpr int kWaves = DP == 128 ? 8 : 4;
        const int64_t units = (int64_t)a.kv_heads * a.head_parts * a.q_parts;
        AttnArgs b = a;
        b.order = attn_order(a, units, k_blocks, false);
        grad_keys_kernel<P, DP, kWaves><<<attn_grid(b.order), 64 * kWaves, 0, stream>>>(b, c);
        e = hipGetLastError();
    }
    AttnArgs b = a;
    b.work = a.head_parts * a.q_parts > 1 ? (unsigned)((int64_t)(a.max_k + kJoinRows - 1) / kJoinRows * a.n_seq) : 0;
    const unsigned grid = b.work + (a.n_buckets > 0 ? a.heads : 0);
    if (e == hipSuccess && grid > 0) {
        grad_join_kernel<P><<<grid, 1024, 0, stream>>>(b);
        e = hipGetLastError();
    }
    return e;
}

template <typename P>
hipError_t by_dim(hipStream_t stream, const AttnArgs &a, const AttnCuts &c) {
    if (a.dim <= 32) return launch<P, 32>(stream, a, c);
    if (a.dim <= 64) return launch<P, 64>(stream, a, c);
    if (a.dim <= 96) return launch<P, 96>(stream, a, c);
    return launch<P, 128>(stream, a, c);
}

}  // namespace

hipError_t gbt_launch_attention_grad(hipStream_t stream, const AttnArgs &a, const AttnCuts &c, int dtype) {
    return dtype == GBT_BF16 ? by_dim<Bf16>(stream, a, c) : by_dim<F16>(stream, a, c);
}
