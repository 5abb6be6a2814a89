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
// and rest 7e-4, with the row sums 2e-7 .. 5e-7; of dq, rows of 5 .. 60 keys, without rest 2.9e-3, with it 2.4e-3.)
#include "attention.h"

namespace {

// A head's bias gradient of one workgroup's keys, by wave.
struct BucketSums {
    float at[4][kAttnBuckets];
};

// Sums over equal buckets of neighbouring lanes (a lane's bucket is never below that of the lane before); the last lane of each run
// adds its sum.
__device__ __forceinline__ void add_runs(float *sums, float v, int bucket, int lane) {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const float w = __shfl_up(v, s);
        const int b = __shfl_up(bucket, s);
        if (lane >= s && b == bucket) v += w;
    }
    const int next = __shfl_down(bucket, 1);
    if (lane == 63 || next != bucket) sums[bucket] += v;
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------------------------------------------- queries --
// As the forward kernel: 128 queries of one head, 32 a wave, keys and values through LDS.
template <typename P, int DP>
__global__ __launch_bounds__(256, 2) void grad_queries_kernel(AttnArgs a, AttnCuts c) {
    typedef typename P::elem E;
    typedef typename P::vec8 V8;
    typedef Tile<DP> T;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32;
    __shared__ __align__(16) char k_tile[2][T::kBytes];
    __shared__ __align__(16) char v_tile[2][T::kBytes];
    __shared__ Buckets buckets;
    __shared__ DistanceRing ring;

    const int q_blocks = (a.max_q + kAttnQueries - 1) / kAttnQueries;
    const int64_t items = (int64_t)q_blocks * a.heads * a.n_seq, item = attn_item(items);
    if (item >= items) return;
    const int block = q_blocks - 1 - (int)(item % q_blocks), head = (int)(item / q_blocks % a.heads), seq = (int)(item / q_blocks / a.heads);
    const AttnSeq rows = attn_seq(a, seq);
    const int first = block * kAttnQueries;
    const bool bias = a.n_buckets > 0;
    if (first >= rows.nq) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int off = rows.nk - rows.nq;
    const int query = first + wave * 32 + (lane & 31);
    const bool there = query < rows.nq;
    if (bias) {
        buckets_load_cuts(buckets, a, c);
        buckets_load_values(buckets, a, head);
    }

    V8 qf[kSteps], gf[kSteps];
    float delta = 0.0f;
    {
        const char *qb = a.q.data + ((rows.q0 + query) * a.q.row + (int64_t)head * a.q.head) * 2;
        const char *gb = a.dout.data + ((rows.q0 + query) * a.dout.row + (int64_t)head * a.dout.head) * 2;
        const char *ob = a.out.data + ((rows.q0 + query) * a.out.row + (int64_t)head * a.out.head) * 2;
        const char *rb = a.rest + ((rows.q0 + query) * a.heads + head) * a.dim * 2;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 16 * s + 8 * half;
            const bool in = there && d < a.dim;
            qf[s] = as_vec<V8>(load16(qb, d * 2, in));
            gf[s] = as_vec<V8>(load16(gb, d * 2, in));
            const V8 o = as_vec<V8>(load16(ob, d * 2, in)), r = as_vec<V8>(load16(rb, d * 2, in && a.rest));
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[s][e], (float)o[e] + (float)r[e], delta);
        }
        delta = column_sum(delta);
    }
    // a query that does not exist, or saw no key: its probabilities are 2^-inf
    const float lse = there ? a.lse[(int64_t)head * a.q_rows + rows.q0 + query] * GBT_LOG2E : INFINITY;
    const float minus = lse == -INFINITY ? -INFINITY : -lse;
    const int last = a.causal ? min(rows.nk - 1, query + off) : rows.nk - 1;
    const int end = a.causal ? min(rows.nk, min(first + kAttnQueries, rows.nq) + off) : rows.nk;
    const int wave_first = first + wave * 32;
    const int wave_end = wave_first >= rows.nq ? 0 : a.causal ? min(rows.nk, min(wave_first + 32, rows.nq) + off) : rows.nk;
    const int wave_all = a.causal ? min(rows.nk, wave_first + off + 1) : rows.nk;

    const int kv_head = head / a.group;
    const char *k_base = a.k.data + (rows.k0 * a.k.row + (int64_t)kv_head * a.k.head) * 2;
    const char *v_base = a.v.data + (rows.k0 * a.v.row + (int64_t)kv_head * a.v.head) * 2;

    f32x16 dq[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[b][r] = 0.0f;
    float row_sum = 0.0f;   // of dS: this lane's half of the column

    auto fetch = [&](int kb) {
        T::fetch(k_tile[(kb >> 6) & 1], k_base + (int64_t)kb * a.k.row * 2, (uint32_t)a.k.row * 2, end - kb, a.dim);
        T::fetch(v_tile[(kb >> 6) & 1], v_base + (int64_t)kb * a.v.row * 2, (uint32_t)a.v.row * 2, end - kb, a.dim);
    };
    if (end > 0) fetch(0);
    arrived(qf);
    arrived(gf);
    __syncthreads();
    if (bias && threadIdx.x < 191) ring_put(ring, buckets, c.steps, (int)threadIdx.x - (first + 127 + off));

    for (int kb = 0; kb < end; kb += 64) {
        tiles_ready();
        if (kb + 64 < end) fetch(kb + 64);
        const char *k_now = k_tile[(kb >> 6) & 1], *v_now = v_tile[(kb >> 6) & 1];
        const int lowest = kb - (first + 127 + off);
        if (bias && wave == ((kb >> 6) & 3)) ring_put(ring, buckets, c.steps, lowest + 191 + lane);
        if (kb >= wave_end) continue;

#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int at = (lowest & 255) + 96 - 32 * wave + 32 * b;   // of this 32 x 32 result's lowest distance, of 63
            const int b0 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at]) : 0, b1 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at + 62]) : 0;
            f32x16 s, dp;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                s = P::mma(T::template rows<P>(k_now, 32 * b, i, lane), qf[i], s);
                dp = P::mma(T::template rows<P>(v_now, 32 * b, i, lane), gf[i], dp);
            }
            if (b0 == b1) {
                const float add = (bias ? buckets.value[b0] : 0.0f) + minus;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, add));
            } else {
                const float *add = ring.value + at + 31 - (lane & 31);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, add[result_row(r, half)] + minus));
            }
            if (kb + 32 * b + 32 > wave_all) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = kb + 32 * b + result_row(r, half) <= last ? s[r] : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] *= dp[r] - delta;
                row_sum += s[r];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const V8 ds = operand<P>(s, i);
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) dq[d] = P::mma(T::template cols<P>(k_now, 32 * b + 16 * i, d, lane), ds, dq[d]);
            }
        }
    }
    row_sum = column_sum(row_sum);
    if (!there) return;
    if (half == 0) a.delta[(int64_t)head * a.q_rows + rows.q0 + query] = delta + row_sum;
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
// A workgroup takes 128 keys of one key head, a wave 32 of them (its columns); the queries of every head that shares them pass through
// LDS with their output gradients, 64 at a time.
//
// Bias gradient.  A 32 x 32 result all of whose distances are in one bucket adds to one running sum in each lane.  Others are laid out by
// diagonals in LDS and added up along them (64 distances, one a lane), and then over each run of lanes of one bucket.
template <typename P, int DP>
__global__ __launch_bounds__(256, DP <= 64 ? 2 : 1) void grad_keys_kernel(AttnArgs a, AttnCuts c) {
    typedef typename P::elem E;
    typedef typename P::vec8 V8;
    typedef Tile<DP> T;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32;
    __shared__ __align__(16) char q_tile[2][T::kBytes];
    __shared__ __align__(16) char g_tile[2][T::kBytes];
    __shared__ __align__(16) float row_minus[2][64], row_delta[2][64];
    __shared__ Buckets buckets;
    __shared__ DistanceRing ring;
    __shared__ BucketSums sums;
    __shared__ float skew[4][32 * 64];   // [key][key - query + 31]: a 32 x 32 result by its diagonals

    const int k_blocks = (a.max_k + kAttnQueries - 1) / kAttnQueries;
    const int64_t items = (int64_t)k_blocks * a.kv_heads * a.n_seq, item = attn_item(items);
    if (item >= items) return;
    const int block = (int)(item % k_blocks), kv_head = (int)(item / k_blocks % a.kv_heads), seq = (int)(item / k_blocks / a.kv_heads);
    const AttnSeq rows = attn_seq(a, seq);
    const int first = block * kAttnQueries;
    const bool bias = a.n_buckets > 0;
    auto strip = [&](int head) { return a.strips + (((int64_t)head * a.n_seq + seq) * k_blocks + block) * a.n_buckets; };
    if (first >= rows.nk) {
        for (int g = 0; g < a.group; ++g)
            for (int i = threadIdx.x; i < a.n_buckets; i += 256) strip(kv_head * a.group + g)[i] = 0.0f;
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int off = rows.nk - rows.nq;
    const int key = first + wave * 32 + (lane & 31);
    const bool there = key < rows.nk;
    if (bias) {
        buckets_load_cuts(buckets, a, c);
        for (int i = threadIdx.x; i < 4 * 32 * 64; i += 256) (&skew[0][0])[i] = 0.0f;
    }

    V8 kf[kSteps], vf[kSteps];
    {
        const char *kb = a.k.data + ((rows.k0 + key) * a.k.row + (int64_t)kv_head * a.k.head) * 2;
        const char *vb = a.v.data + ((rows.k0 + key) * a.v.row + (int64_t)kv_head * a.v.head) * 2;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 16 * s + 8 * half;
            kf[s] = as_vec<V8>(load16(kb, d * 2, there && d < a.dim));
            vf[s] = as_vec<V8>(load16(vb, d * 2, there && d < a.dim));
        }
    }
    f32x16 dk[kBlocks], dv[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.0f;

    // queries from `start` on see one of the workgroup's keys
    const int start = a.causal ? max(0, first - off) & ~63 : 0;
    const int sees = a.causal ? key - off : 0;                         // the first query that sees this lane's key
    const int wave_from = a.causal ? first + wave * 32 - off : 0;      // and one of the wave's,
    const int wave_all = a.causal ? first + wave * 32 + 31 - off : 0;  // and all of them
    const bool wave_last = first + wave * 32 + 32 > rows.nk;           // some of the wave's keys do not exist

    for (int g = 0; g < a.group; ++g) {
        const int head = kv_head * a.group + g;
        const char *q_base = a.q.data + (rows.q0 * a.q.row + (int64_t)head * a.q.head) * 2;
        const char *g_base = a.dout.data + (rows.q0 * a.dout.row + (int64_t)head * a.dout.head) * 2;
        const float *lse = a.lse + (int64_t)head * a.q_rows + rows.q0, *delta = a.delta + (int64_t)head * a.q_rows + rows.q0;
        __syncthreads();   // the head before is done with the values, the ring and the sums
        float run = 0.0f;  // this lane's part of the sum over results of one bucket
        int run_bucket = 0;
        if (bias) {
            buckets_load_values(buckets, a, head);
            for (int i = threadIdx.x; i < 4 * kAttnBuckets; i += 256) (&sums.at[0][0])[i] = 0.0f;
        }
        auto fetch = [&](int qb) {
            const int n = (qb >> 6) & 1;
            T::fetch(q_tile[n], q_base + (int64_t)qb * a.q.row * 2, (uint32_t)a.q.row * 2, rows.nq - qb, a.dim);
            T::fetch(g_tile[n], g_base + (int64_t)qb * a.dout.row * 2, (uint32_t)a.dout.row * 2, rows.nq - qb, a.dim);
            if (threadIdx.x < 64) {
                const int q = qb + threadIdx.x;
                const float l = q < rows.nq ? lse[q] : -INFINITY;
                row_minus[n][threadIdx.x] = l == -INFINITY ? -INFINITY : -l * GBT_LOG2E;   // no query, or one that saw no key
                row_delta[n][threadIdx.x] = q < rows.nq ? delta[q] : 0.0f;
            }
        };
        if (start < rows.nq) fetch(start);
        arrived(kf);
        arrived(vf);
        __syncthreads();
        if (bias && threadIdx.x < 191) ring_put(ring, buckets, c.steps, (int)threadIdx.x + first - (start + 63 + off));
        for (int qb = start; qb < rows.nq; qb += 64) {
            tiles_ready();
            if (qb + 64 < rows.nq) fetch(qb + 64);
            const int now = (qb >> 6) & 1;
            const char *q_now = q_tile[now], *g_now = g_tile[now];
            const int lowest = first - (qb + 63 + off);
            if (bias && wave == ((qb >> 6) & 3)) ring_put(ring, buckets, c.steps, lowest - 64 + lane);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (qb + 32 * b + 31 < wave_from || qb + 32 * b >= rows.nq) continue;
                const int at = (lowest & 255) + 32 * wave + 32 - 32 * b;   // of this result's lowest distance, of 63
                const int b0 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at]) : 0, b1 = bias ? __builtin_amdgcn_readfirstlane(ring.bucket[at + 62]) : 0;
                f32x16 s, dp;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    s = P::mma(T::template rows<P>(q_now, 32 * b, i, lane), kf[i], s);
                    dp = P::mma(T::template rows<P>(g_now, 32 * b, i, lane), vf[i], dp);
                }
                f32x16 minus, del;
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    const f32x4 m = *(const f32x4 *)(row_minus[now] + 32 * b + 8 * r4 + 4 * half), d = *(const f32x4 *)(row_delta[now] + 32 * b + 8 * r4 + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        minus[4 * r4 + e] = m[e];
                        del[4 * r4 + e] = d[e];
                    }
                }
                if (b0 == b1) {
                    const float add = bias ? buckets.value[b0] : 0.0f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, add + minus[r]));
                } else {
                    const float *add = ring.value + at + 31 + (lane & 31);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, add[-result_row(r, half)] + minus[r]));
                }
                if (qb + 32 * b < wave_all) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = qb + 32 * b + result_row(r, half) >= sees ? s[r] : 0.0f;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] = s[r] * (dp[r] - del[r]);
                // a key beyond the last has scores of its bias alone
                if (bias && wave_last) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) dp[r] = there ? dp[r] : 0.0f;
                }
                if (bias && b0 == b1) {
                    if (b0 != run_bucket) {
                        const float v = wave_sum(run);
                        if (lane == 0) sums.at[wave][run_bucket] += v;
                        __builtin_amdgcn_wave_barrier();
                        run = 0.0f;
                        run_bucket = b0;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) run += dp[r];
                } else if (bias) {
                    float *sk = skew[wave];
#pragma unroll
                    for (int r = 0; r < 16; ++r) sk[(lane & 31) * 65 + 31 - result_row(r, half)] = dp[r];
                    __builtin_amdgcn_wave_barrier();
                    float v = 0.0f;
#pragma unroll
                    for (int i = 0; i < 32; ++i) v += sk[64 * i + lane];
                    add_runs(sums.at[wave], v, ring.bucket[at + min(lane, 62)], lane);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const V8 p = operand<P>(s, i), ds = operand<P>(dp, i);
#pragma unroll
                    for (int d = 0; d < kBlocks; ++d) {
                        dv[d] = P::mma(T::template cols<P>(g_now, 32 * b + 16 * i, d, lane), p, dv[d]);
                        dk[d] = P::mma(T::template cols<P>(q_now, 32 * b + 16 * i, d, lane), ds, dk[d]);
                    }
                }
            }
        }
        if (bias) {
            const float v = wave_sum(run);
            if (lane == 0) sums.at[wave][run_bucket] += v;
            __syncthreads();
            for (int i = threadIdx.x; i < a.n_buckets; i += 256)
                strip(head)[i] = (sums.at[0][i] + sums.at[1][i]) + (sums.at[2][i] + sums.at[3][i]);
        }
    }
    if (!there) return;
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

// The strips of every head together, in a fixed order: a workgroup takes a head, a thread every (256 / buckets)-th strip of a bucket.
__global__ __launch_bounds__(256) void grad_bias_kernel(AttnArgs a) {
    __shared__ double part[256];
    const int head = blockIdx.x, n = a.n_buckets, lanes = 256 / n;   // threads of a bucket
    const int64_t strips = (int64_t)a.n_seq * ((a.max_k + kAttnQueries - 1) / kAttnQueries);
    const float *from = a.strips + (int64_t)head * strips * n;
    const int b = threadIdx.x % n, l = threadIdx.x / n;
    double sum = 0.0;
    if (l < lanes)
        for (int64_t s = l; s < strips; s += lanes) sum += from[s * n + b];
    part[threadIdx.x] = sum;
    __syncthreads();
    if (l == 0) {
        for (int i = 1; i < lanes; ++i) sum += part[i * n + b];
        a.dbias[(int64_t)b * a.heads + head] = (float)sum;
    }
}

unsigned grid_of(int64_t items) { return (unsigned)((items + 7) / 8 * 8); }

template <typename P, int DP>
hipError_t launch(hipStream_t stream, const AttnArgs &a, const AttnCuts &c) {
    const int64_t q_blocks = (a.max_q + kAttnQueries - 1) / kAttnQueries, k_blocks = (a.max_k + kAttnQueries - 1) / kAttnQueries;
    hipError_t e = hipSuccess;
    if (q_blocks > 0 && a.n_seq > 0) {
        grad_queries_kernel<P, DP><<<grid_of(q_blocks * a.heads * a.n_seq), 256, 0, stream>>>(a, c);
        e = hipGetLastError();
    }
    if (e == hipSuccess && k_blocks > 0 && a.n_seq > 0) {
        grad_keys_kernel<P, DP><<<grid_of(k_blocks * a.kv_heads * a.n_seq), 256, 0, stream>>>(a, c);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.n_buckets > 0) {
        grad_bias_kernel<<<(unsigned)a.heads, 256, 0, stream>>>(a);
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
