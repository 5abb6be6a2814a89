// What the attention kernels share: arguments, the ragged rows, matrix instructions, tiles in LDS, buckets of distance.
//
// Everything is arranged around v_mfma_f32_32x32x16: a lane holds ONE column of the 32 x 32 result (column lane % 32) and
// sixteen of its rows (register r: row 8 * (r / 4) + 4 * (lane / 32) + r % 4).  The kernels take scores transposed where a wave
// owns queries (rows keys, columns queries), so a query's maximum and sum are sums over a lane's own registers and one exchange
// between the two halves of the wave.  Sixteen rows of such a result, as they lie in eight registers of the two halves, are the second
// operand of the next product without any move between lanes, as long as the first operand takes its rows in the same order:
// slot e of half hl is row 4 * hl + e for e < 4 and 8 + 4 * hl + e - 4 beyond.  That order is what two transposing LDS reads
// (ds_read_b64_tr_b16) of rows 4 * hl .. + 3 and 8 + 4 * hl .. + 3 give.
#pragma once

#include "gbt_internal.h"

constexpr int kAttnBuckets = GBT_MAX_BUCKETS;   // of distance; a power of two

struct AttnView {   // rows x heads x head_dim elements; strides in elements, the head's elements side by side
    char *data;
    int64_t row, head;
};

// How the workgroups of a launch go over the work: `blocks` blocks of each of `units` units (heads, or key heads and parts) of every sequence.
//
// Workgroups go to the eight XCDs in turn, and blocks of one unit share what they read, so an XCD takes whole units; sequences are as long as they
// are, so no XCD is to have more of one than another: an eighth of each where units divide so, else units in turn, single blocks where even
// those are few.  (24 histories of 100 to 1000 rows, 8 heads: an eighth of all units in a row for each XCD 58 us, an eighth of each history 48.)
// The blocks with the most to do come first.  Where causal blocks differ in that and all that is read fits the XCDs' L2, the first blocks of all units
// come before all second ones, so that the last workgroups are short ones (16 causal histories of 100 to 1000 rows, forward and the two gradient
// kernels unit by unit 32 + 44 + 73 us, block by block 31 + 41 + 63; two of 4096 211 + 263 + 431, 195 + 250 + 440; but 24 that are not causal 47, 56).
//
// Otherwise up to 64 sequences, or 32 causal ones, are taken by their length, the longest first, so that what is left at the end is short.  Lengths lie
// on the device, so every workgroup finds its sequence's place itself, in a few steps whatever the lengths.  (us forward and backward without and with, 8
// heads: 24 histories of 100 to 1000 rows, heads of 64, 47.6 + 166, 41.2 + 149; 64 114 + 436, 111 + 429; 6 of 500 to 3000 82.8 + 270, 64.4 + 216; 64 of 500
// 58.6 + 228, 59.8 + 232; causal, heads of 128, 24 54.0 + 198, 44.4 + 182; but 64 143 + 555, 148 + 614; and block by block, heads of 64, 16 26.1 + 80,
// 26.3 + 83.)
struct AttnOrder {
    int units, blocks, wide;    // wide: units of an XCD, or of all where single blocks go to XCDs
    int single, by_block;
    int sorted;                 // by the length of queries (1) or keys (2)
};
inline unsigned attn_grid(const AttnOrder &o) { return (unsigned)((int64_t)(o.single ? 1 : 8) * o.wide * o.blocks); }

struct AttnArgs {
    AttnView q, k, v, out;
    const int64_t *q_ptr, *k_ptr;   // NULL: sequence s has rows s * max .. (s + 1) * max
    const int32_t *k_len;           // NULL: all of a sequence's key rows are used
    int64_t q_rows, k_rows;
    int n_seq, heads, kv_heads, group, dim, max_q, max_k, causal, n_buckets;
    AttnOrder order;
    unsigned work;                  // workgroups of the launch; those behind them zero the rows of no sequence
    float scale, scale2;            // scale2 = scale * log2(e): probabilities are powers of two here
    const float *bias;              // [n_buckets][heads]
    float *lse;                     // [heads][q_rows], natural logarithm, or NULL
    char *rest;                     // what rounding took from out, [q_rows][heads][dim], or NULL
    // backward
    AttnView dout, dq, dk, dv;
    float *row_less;                // [heads][q_rows]: what a row's scores lose, kLift - lse * log2(e) (-inf: a row without keys)
    float *row_minus;               // [heads][q_rows]: and what its products of gradients with values are added to, -delta
    float *strips;                  // [heads][n_seq * k_blocks * q_parts][n_buckets]: the bias gradient of each block of keys
    float *dbias;                   // [n_buckets][heads]
    int head_parts, q_parts;        // a block of keys is shared by so many workgroups: by heads of the group, by queries
    // partial results: few rows' of the pieces of the key axis; keys' gradients [head_parts * q_parts][2][part_rows][kv_heads][dim]
    float *part;
    int64_t part_rows;              // of the k tensor, or max_k for each sequence where those are fewer: a store may be far larger than what is in use
    int pieces, piece_len;
};

inline AttnOrder attn_order(const AttnArgs &a, int64_t units, int64_t blocks, bool owns_queries) {
    const int64_t bytes = owns_queries ? 4 * a.k_rows * a.kv_heads * a.dim : 4 * a.q_rows * a.heads * a.dim;   // read by the blocks
    AttnOrder o;
    o.units = (int)units;
    o.blocks = (int)blocks;
    o.single = units % 8 != 0 && units * a.n_seq < 64;
    o.wide = (int)(o.single ? units * a.n_seq : (units * a.n_seq + 7) / 8);
    o.by_block = a.causal && bytes <= (int64_t)8 * (4 << 20);
    const int length = owns_queries == (a.causal != 0) ? 1 : 2;
    const bool ragged = length == 1 ? a.q_ptr != nullptr : a.k_ptr || a.k_len;
    o.sorted = ragged && !o.by_block && a.n_seq > 1 && a.n_seq <= (a.causal ? 32 : 64) && blocks > 2 ? length : 0;
    return o;
}

// How many queries a workgroup of the kernels that own queries takes, 32 a wave, and in how many groups of waves that take the tiles of keys in turn.
// Where there are fewer workgroups of 128 than compute units and keys are several tiles, how many steps follow one another is what counts: two groups
// halve them.  Two groups of 64 queries spread over twice as many compute units; with heads of more than 64 elements LDS has room for only one such
// workgroup on each, so they must all run at once.  Workgroups are counted as the rows give them, not as max_q would.
// us forward and backward, 128 queries and one group, 128 and two, 64 and two, causal: heads of 64 elements, 4 histories of 100 to 1000 rows, 8 heads
// 19.0 + 64, 16.2 + 61, 14.7 + 58; one of 4096, 4 heads 65 + 143, 48 + 122, 40 + 110; but 16 of 1000 35.7 + 132, 45.7 + 146, 47.4 + 141; heads of 80, 3 of
// 300 to 800, 6 heads 20.1 + 65, 17.8 + 61, 16.8 + 58; 5 20.1 + 68, 17.1 + 64, 20.0 + 65; not causal 20.9 + 71, 18.6 + 69, 27.0 + 77; 9 23.2 + 89,
// 25.0 + 91, 36.3 + 101; one of 2000, 16 heads 46.9 + 173, 38.5 + 165, 65.3 + 193; heads of 128, 3 21.9 + 68, 19.3 + 71, 18.1 + 63; 5 22.2 + 77, 19.9 + 79, 22.8 + 76 (two groups of the backward kernel at 128
// queries have too few registers, so there it has one).
struct AttnForm {
    int queries, groups;
};
inline AttnForm attn_form(const AttnArgs &a, int DP, bool backward) {
    const int64_t most = (a.max_q + 127) / 128 * (int64_t)a.n_seq, workgroups = a.heads * std::min(most, a.q_rows / 128 + (a.n_seq + 1) / 2);
    if (a.max_k < 256 || workgroups > 256 || a.heads * most > (1 << 20)) return AttnForm{128, 1};   // (the launch is as large as max_q says)
    const bool even = a.heads % 8 == 0 || a.n_seq == 1;   // over the XCDs
    if (DP <= 64 || workgroups <= (even ? 128 : 96)) return AttnForm{64, 2};
    return AttnForm{128, backward && DP == 128 ? 1 : 2};
}

struct AttnCuts {
    int32_t at[kAttnBuckets - 1];   // ascending
};

hipError_t gbt_launch_attention(hipStream_t stream, const AttnArgs &a, const AttnCuts &c, int dtype);
hipError_t gbt_launch_attention_few(hipStream_t stream, const AttnArgs &a, const AttnCuts &c, int dtype);
hipError_t gbt_launch_attention_grad(hipStream_t stream, const AttnArgs &a, const AttnCuts &c, int dtype);
constexpr int kAttnQueries = 128;   // of a workgroup of the block kernels (keys, where a workgroup owns keys)
constexpr int kAttnFewRows = 32;    // (query, head of the group) columns of a key head that the few-rows kernel takes at most

#define GBT_LOG2E 1.44269504088896340736f
#define GBT_LN2 0.69314718055994530942f

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

struct Bf16 {
    typedef __bf16 elem;
    typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
    static constexpr bool kNarrow = false;   // has too few exponents for what products are made of
    static constexpr float kAbove = 0.0f;   // while a row is summed, its largest probability is 2^kAbove at least
    static __device__ __forceinline__ f32x16 mma(vec8 a, vec8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
struct F16 {
    typedef _Float16 elem;
    typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
    static constexpr bool kNarrow = true;
    static constexpr float kAbove = 7.0f;
    static __device__ __forceinline__ f32x16 mma(vec8 a, vec8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};

struct AttnSeq {
    int64_t q0, k0;
    int nq, nk;
};
// The rows of sequence s.  Pointers that do not describe rows of the tensors describe none: no kernel reads past them.
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int s) {
    AttnSeq r;
    int64_t q1, k1;
    if (a.q_ptr) {
        r.q0 = a.q_ptr[s];
        q1 = a.q_ptr[s + 1];
    } else {
        r.q0 = (int64_t)s * a.max_q;
        q1 = r.q0 + a.max_q;
    }
    if (a.k_ptr) {
        r.k0 = a.k_ptr[s];
        k1 = a.k_ptr[s + 1];
    } else {
        r.k0 = (int64_t)s * a.max_k;
        k1 = r.k0 + a.max_k;
    }
    if (a.k_len) {
        const int64_t len = a.k_len[s];
        if (len < k1 - r.k0) k1 = r.k0 + len;
    }
    r.nq = r.q0 >= 0 && q1 <= a.q_rows && q1 > r.q0 ? (int)min(q1 - r.q0, (int64_t)a.max_q) : 0;
    r.nk = r.k0 >= 0 && k1 <= a.k_rows && k1 > r.k0 ? (int)min(k1 - r.k0, (int64_t)a.max_k) : 0;
    return r;
}

// The row of the partial results that sequence s begins at.
__device__ __forceinline__ int64_t attn_part_row(const AttnArgs &a, int s, const AttnSeq &rows) {
    return a.part_rows < a.k_rows ? (int64_t)s * a.max_k : rows.k0;
}

struct AttnItem {
    int seq, unit, block;   // seq < 0: none
};
// Which of up to 64 sequences is the place-th in length, counted from the longest; by blocks of 128 rows, in their own order where they have the same
// number of those.  Found bit by bit of that number, from the highest that a sequence can have: those with the bit come before those without.  So
// it takes no more steps than bits, however far the caller's maximum lies above the lengths (64 sequences of 100 to 300 rows, a maximum of 2^20, of half a
// million idle workgroups: 3.1 ms; 65 sequences, in no order, 1.8; counting down from the maximum 1435).
__device__ __forceinline__ int nth_longest(const AttnArgs &a, int place) {
    const int lane = threadIdx.x & 63;
    int blocks = 0;
    if (lane < a.n_seq) {
        const AttnSeq rows = attn_seq(a, lane);
        blocks = ((a.order.sorted == 1 ? rows.nq : rows.nk) + 127) >> 7;
    }
    const int most = (int)((a.order.sorted == 1 ? min((int64_t)a.max_q, a.q_rows) : min((int64_t)a.max_k, a.k_rows)) + 127) >> 7;
    uint64_t left = ~0ull >> (64 - a.n_seq);
    for (int bit = 31 - __clz(most); bit >= 0; --bit) {
        const uint64_t with = __ballot((blocks >> bit) & 1) & left;
        const int count = __popcll(with);
        if (place < count) {
            left = with;
        } else {
            place -= count;
            left &= ~with;
        }
    }
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(left >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)left, 0u));
    return __ffsll((unsigned long long)(__ballot(before == place) & left)) - 1;
}
__device__ __forceinline__ AttnItem attn_item(const AttnArgs &a) {
    const AttnOrder &o = a.order;
    AttnItem it;
    const int at = o.single ? blockIdx.x : blockIdx.x / 8, xcd = blockIdx.x % 8;
    int unit = o.by_block ? at % o.wide : at / o.blocks;
    it.block = o.by_block ? at / o.wide : at % o.blocks;
    if (o.units % 8 == 0) {
        const int eighth = o.units / 8;
        it.seq = unit / eighth;
        it.unit = xcd * eighth + unit % eighth;
    } else {
        if (!o.single) unit = unit * 8 + xcd;
        it.seq = unit / o.units;
        it.unit = unit % o.units;
    }
    if (it.seq >= a.n_seq) it.seq = -1;
    else if (o.sorted) it.seq = nth_longest(a, it.seq);
    return it;
}

// Rows of no sequence.  What follows attention, and what the gradients of its inputs go into, runs over whole tensors, so such rows are zeros and not
// whatever was in memory.  They lie before a sequence and behind the one before it; workgroups at the end of a launch look for them: all waves share
// those before the first sequence and behind the last, where padding is, others take a wave each.  Pointers that lie outside or do not ascend
// describe no sequences, and which of their rows are zeros is open.
constexpr unsigned kGapWorkgroups = 64;
inline unsigned attn_gap_workgroups(const AttnArgs &a, bool queries, bool keys) {
    return (queries && (a.q_ptr || (int64_t)a.n_seq * a.max_q < a.q_rows)) || (keys && (a.k_ptr || a.k_len || (int64_t)a.n_seq * a.max_k < a.k_rows))
               ? kGapWorkgroups : 0;
}
__device__ __forceinline__ void zero_gaps(const AttnArgs &a, const AttnView &x, bool keys) {
    const int lane = threadIdx.x & 63, waves = kGapWorkgroups * (blockDim.x >> 6), wave = (blockIdx.x - a.work) * (blockDim.x >> 6) + (threadIdx.x >> 6);
    const int64_t all = keys ? a.k_rows : a.q_rows;
    const int each = a.dim / 8, pieces = (keys ? a.kv_heads : a.heads) * each;   // of 16 bytes
    auto zero = [&](int64_t from, int64_t to, int64_t step) {
        for (int64_t row = from; row < to; row += step)
            for (int p = lane; p < pieces; p += 64) *(i32x4 *)(x.data + (row * x.row + p / each * x.head + p % each * 8) * 2) = i32x4{0, 0, 0, 0};
    };
    auto gap = [&](int s, int64_t &from, int64_t &to) {   // between sequences s - 1 and s
        from = 0, to = all;
        if (s > 0) {
            const AttnSeq before = attn_seq(a, s - 1);
            from = min(all, max((int64_t)0, keys ? before.k0 + before.nk : before.q0 + before.nq));
        }
        if (s < a.n_seq) {
            const AttnSeq behind = attn_seq(a, s);
            to = min(all, keys ? behind.k0 : behind.q0);
        }
    };
    int64_t from, to;
    gap(0, from, to);
    zero(from + wave, to, waves);
    if (a.n_seq == 0) return;
    gap(a.n_seq, from, to);
    zero(from + wave, to, waves);
    for (int64_t s0 = 1 + (int64_t)wave * 64; s0 < a.n_seq; s0 += (int64_t)waves * 64) {
        from = to = 0;
        if (s0 + lane < a.n_seq) gap((int)s0 + lane, from, to);
        for (uint64_t some = __ballot(from < to); some; some &= some - 1) {
            const int l = __ffsll((unsigned long long)some) - 1;
            zero(__shfl(from, l), __shfl(to, l), 1);
        }
    }
}

// A lane's row as an operand: elements 16 * s + 8 * half .. + 7 in regs[s], zeros past the head's.
template <typename V, int N>
__device__ __forceinline__ void load_row(V (&regs)[N], const char *row, int half, int dim) {
#pragma unroll
    for (int s = 0; s < N; ++s) regs[s] = *(const V *)(row + min(16 * s + 8 * half, dim - 8) * 2);
    if (dim < 16 * N) {
#pragma unroll
        for (int s = 0; s < N; ++s)
            if (16 * s + 8 * half >= dim) regs[s] = V{};
    }
}

__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}
// Sixteen bytes for each lane from base + offset (base and `to` the same in all lanes) to LDS, the lanes' side by side from `to` on.  It has no
// result in registers; tiles_ready() waits for it.  Not the builtin: with that one the compiler waits for every load under way before LDS reads
// that it cannot tell apart from the loads' targets, and so for the next tile before it reads this one.  Into the text it does not see: the wait state
// between the write of M0 and the load that reads it is kept here.
__device__ __forceinline__ void load_to_lds(uint32_t to, const char *base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory", "m0");
}

// Four bytes for each lane likewise.
__device__ __forceinline__ void load_word_to_lds(uint32_t to, const float *base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory", "m0");
}

// A tile of 64 rows in LDS.  A row's sixteen-byte pieces are stored in an order of its own, piece c at place c ^ fold(row), with which both
// kinds of read meet each of the 64 banks once a clock: sixteen bytes of sixteen rows, and 64 bytes of four rows (transposed).  Measured, a
// compute unit reads 219 to 235 bytes a clock so; with rows 16 or 32 bytes further apart instead, 122 to 125 by one kind of read or both.
template <int DP>
struct Tile {
    static constexpr int kRowBytes = DP == 96 ? 256 : DP * 2, kPlaces = kRowBytes / 16, kBytes = 64 * kRowBytes;
    static __device__ __forceinline__ constexpr int fold(int row) {
        return kPlaces == 4 ? (row >> 2) & 3 : kPlaces == 8 ? ((row >> 1) & 1) * 4 | ((row >> 2) & 3) : (row & 3) * 4 | ((row >> 2) & 3);
    }
    // From memory straight into LDS, a wave's 64 pieces at a time, by kWaves waves, of which this one is number `wave`.  Rows past the last and elements past the head's are taken from
    // the last there are, so that nothing hangs on a condition: such rows' probabilities are zero, and such elements meet zeros of the
    // other operand or are not stored.  rows, dim > 0; 64 * row_bytes < 2^32.
    // kKeep: addresses may be kept in registers from one call to the next; else they are worked out each time, for kernels that have none to spare (what
    // is kept in memory is waited for together with the loads before it).
    template <bool kKeep = true, int kWaves = 4>
    static __device__ __forceinline__ void fetch(char *tile, const char *base, uint32_t row_bytes, int rows, int dim, int wave) {
        int lane = kKeep ? threadIdx.x & 63 : __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
        if (!kKeep) asm volatile("" : "+v"(lane));
        constexpr int kRows = 64 / kPlaces, kNext = kWaves * kRows;   // of a wave's load, and how much further its next one is
        const int row = wave * kRows + lane / kPlaces;
        const uint32_t to = lds_address(tile) + wave * 1024;
        const uint32_t col = min(lane % kPlaces ^ fold(row), dim / 8 - 1) * 16;
        const uint32_t odd = kNext % 16 == 0 ? col : min(lane % kPlaces ^ fold(row + kNext), dim / 8 - 1) * 16;   // a fold has a period of 16 rows
#pragma unroll
        for (int i = 0; i < kPlaces / kWaves; ++i)
            load_to_lds(to + i * kWaves * 1024, base, (uint32_t)min(row + i * kNext, rows - 1) * row_bytes + (i & 1 ? odd : col));
    }
    // The first 32 rows likewise, by one wave.
    static constexpr int kHalfLoads = kPlaces / 2;
    static __device__ __forceinline__ void fetch_half(char *tile, const char *base, uint32_t row_bytes, int rows, int dim) {
        const int lane = threadIdx.x & 63;
        constexpr int kRows = 64 / kPlaces;
        const uint32_t to = lds_address(tile);
#pragma unroll
        for (int i = 0; i < kHalfLoads; ++i) {
            const int row = i * kRows + lane / kPlaces, col = min(lane % kPlaces ^ fold(row), dim / 8 - 1);
            load_to_lds(to + i * 1024, base, (uint32_t)min(row, rows - 1) * row_bytes + col * 16);
        }
    }
    // Waits until of this wave's fetches of 32 rows only the last is still under way.
    static __device__ __forceinline__ void half_ready() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kHalfLoads) : "memory"); }
    // First operand, rows as they are: row row0 + lane % 32 (row0 a multiple of 32), elements 16 * step + 8 * (lane / 32) .. + 7.
    template <typename P>
    static __device__ __forceinline__ typename P::vec8 rows(const char *tile, int row0, int step, int lane) {
        const int row = lane & 31, mine = row * kRowBytes + (((lane >> 5) ^ fold(row)) << 4);
        return *(const typename P::vec8 *)(tile + row0 * kRowBytes + (mine ^ (step << 5)));
    }
    // First operand, the tile transposed: row d = 32 * block + lane % 32, over the sixteen tile rows row0 .. row0 + 15 (row0 a multiple of 16)
    // in the order that a result's registers have (see above).
    template <typename P>
    static __device__ __forceinline__ typename P::vec8 cols(const char *tile, int row0, int block, int lane) {
        const int row = 4 * (lane >> 5) + ((lane & 15) >> 2), piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        const int lo_at = row * kRowBytes + ((piece ^ fold(row)) << 4) + 8 * (lane & 1);
        const int hi_at = (row + 8) * kRowBytes + ((piece ^ fold(row + 8)) << 4) + 8 * (lane & 1);
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + row0 * kRowBytes + (lo_at ^ (block << 6))));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + row0 * kRowBytes + (hi_at ^ (block << 6))));
        const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(typename P::vec8, both);
    }
    // The same where the tile is not known at compile time: one address for all reads, which differ in bits that are zero in a tile's own (aligned
    // to 256 bytes) and in constants that the instruction adds; `further` is that of another tile.  (fold(row + 8) is fold(row) ^ 2.)
    static __device__ __forceinline__ uint32_t rows_base(const char *tile, int row0, int lane) {
        const int row = lane & 31;
        return lds_address(tile) + row0 * kRowBytes + row * kRowBytes + (((lane >> 5) ^ fold(row)) << 4);
    }
    template <typename P>
    static __device__ __forceinline__ typename P::vec8 rows_at(uint32_t base, int step, int further) {
        return *(const __attribute__((address_space(3))) typename P::vec8 *)(uintptr_t)((base ^ (step << 5)) + further);
    }
    static __device__ __forceinline__ uint32_t cols_base(const char *tile, int row0, int lane) {
        const int row = 4 * (lane >> 5) + ((lane & 15) >> 2), piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        return lds_address(tile) + row0 * kRowBytes + row * kRowBytes + ((piece ^ fold(row)) << 4) + 8 * (lane & 1);
    }
    template <typename P>
    static __device__ __forceinline__ typename P::vec8 cols_at(uint32_t base, int row0, int block, int further) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((base ^ (block << 6)) + row0 * kRowBytes + further));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((base ^ (block << 6) ^ 32) + (row0 + 8) * kRowBytes + further));
        const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(typename P::vec8, both);
    }
};
// The compiler waits for loaded registers where they are first used, and inside a loop for everything under way.  Done with them here.
template <typename V, int N>
__device__ __forceinline__ void arrived(V (&regs)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(regs[i]));
}
// This wave's LDS reads have their results: what it read may be fetched over.
__device__ __forceinline__ void done_reading() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// Waits for this wave's fetches, then for the other waves: the tiles fetched last can be read, and those read before written.
__device__ __forceinline__ void tiles_ready() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Second operand from eight registers of a result, rounded to the inputs' type (to nearest, ties to even).
template <typename P>
__device__ __forceinline__ typename P::vec8 operand(const f32x16 &x, int half) {
    typename P::vec8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (typename P::elem)x[8 * half + e];
    return v;
}

// What rounding took from that.
template <typename P>
__device__ __forceinline__ typename P::vec8 operand_rest(const f32x16 &x, int half, typename P::vec8 rounded) {
    typename P::vec8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (typename P::elem)(x[8 * half + e] - (float)rounded[e]);
    return v;
}

// Row of register r of a 32 x 32 result.
__device__ __forceinline__ constexpr int result_row(int r, int half) { return 8 * (r / 4) + 4 * half + r % 4; }

// Over the two halves of a column.
__device__ __forceinline__ float column_max(float x) {
    const int i = __builtin_bit_cast(int, x);
    const auto both = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    return fmaxf(__builtin_bit_cast(float, (int)both[0]), __builtin_bit_cast(float, (int)both[1]));
}
__device__ __forceinline__ float column_sum(float x) {
    const int i = __builtin_bit_cast(int, x);
    const auto both = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    return __builtin_bit_cast(float, (int)both[0]) + __builtin_bit_cast(float, (int)both[1]);
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
    return x;
}

// Buckets of distance.  A bucket's number is how many cuts are at most the distance, as a symbol's is of its value.
//
// The distances that a step's 64 (or 128) rows against a workgroup's 128 meet are 191 (255) in a row, and as many new ones as rows come with each
// step.  They are kept in a ring of 256 (512), twice, so that a stretch is read without wrapping.
template <int SIZE>
struct DistanceRing {
    static constexpr int kMask = SIZE - 1;
    float value[2 * SIZE];         // the head's bias times log2(e)
    uint8_t bucket[2 * SIZE];
    uint8_t is_cut[8][64];         // by wave
    float of_bucket[kAttnBuckets];
    int cut[kAttnBuckets];         // filled up with INT32_MAX
};
// Two cuts for each lane of a wave.
struct LaneCuts {
    int lo, hi;
};
template <int SIZE>
__device__ __forceinline__ void ring_cuts(DistanceRing<SIZE> &ring, const AttnArgs &a, const AttnCuts &c) {
    if (threadIdx.x < kAttnBuckets) ring.cut[threadIdx.x] = (int)threadIdx.x < a.n_buckets - 1 ? c.at[threadIdx.x] : INT32_MAX;
}
// Times log2(e).  Scores of 32 bits that large have nothing left of the products, so a bias that can only be meant as a mask is one: rows that it
// leaves without keys are zeros, whichever low value stands for it, and not the mean of the values or, in the gradients, 2^(score - lse) of anything.
__device__ __forceinline__ float bias_value(float x) { return x < GBT_BIAS_SHUT ? -INFINITY : x * GBT_LOG2E; }
template <int SIZE>
__device__ __forceinline__ void ring_head(DistanceRing<SIZE> &ring, const AttnArgs &a, int head) {
    for (int i = threadIdx.x; i < a.n_buckets; i += blockDim.x) ring.of_bucket[i] = bias_value(a.bias[(int64_t)i * a.heads + head]);
}
// The bucket of distance t0 + lane, for a whole wave.  The lane of each cut among the 64 distances marks its place in LDS; how many marks are at
// or before a distance is then a count of bits.
__device__ __forceinline__ int lane_bucket(uint8_t *mark, const LaneCuts &cuts, int t0, int lane) {
    const uint32_t lo = (uint32_t)cuts.lo - (uint32_t)t0, hi = (uint32_t)cuts.hi - (uint32_t)t0;
    int n = __popcll(__ballot(cuts.lo < t0)) + __popcll(__ballot(cuts.hi < t0));
    const bool lo_in = cuts.lo >= t0 && lo < 64u, hi_in = cuts.hi >= t0 && hi < 64u;
    if (__any(lo_in || hi_in)) {
        mark[lane] = 0;
        __builtin_amdgcn_wave_barrier();
        if (lo_in) mark[lo] = 1;
        if (hi_in) mark[hi] = 1;
        __builtin_amdgcn_wave_barrier();
        const uint64_t marks = __ballot(mark[lane] != 0);
        n += __popcll(marks & (~0ull >> (63 - lane)));
    }
    return n;
}
// The 64 distances from t0 on into the ring, by one wave.
template <int SIZE>
__device__ __forceinline__ void ring_put(DistanceRing<SIZE> &ring, int t0, int wave, int lane) {
    const int n = lane_bucket(ring.is_cut[wave], LaneCuts{ring.cut[lane], ring.cut[lane + 64]}, t0, lane);
    const int at = (t0 + lane) & (SIZE - 1);
    ring.value[at] = ring.value[at + SIZE] = ring.of_bucket[n];
    ring.bucket[at] = ring.bucket[at + SIZE] = (uint8_t)n;
}

}  // namespace
