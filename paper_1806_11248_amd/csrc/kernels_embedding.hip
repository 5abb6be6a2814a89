// Rows of an embedding table by id, and the table's gradient.
//
// Lookup: out[t] = scale * table[id_t], a product in 32 bits, rounded to out's type.  Gradient: grad[v] = scale * (sum of dout[t] over the places t with id_t = v), a sum of rows that
// lie anywhere, of which one id may have none and another a third of all.  Places are sorted by id (stable, by digits), and a group of lanes adds up
// a chunk of them, however the ids are spread; sums of ids that go on in the next chunk are written aside in 32 bits and added up by a second launch in
// the chunks' order.  Where the table has few rows nothing is sorted: they are added up in LDS.  No atomics on values: the same result on every run.
// Bound: memory.
#include "embedding.h"

namespace {

template <typename E>
struct alignas(sizeof(E) * 8 < 16 ? sizeof(E) * 8 : 16) Eight {
    E x[8];
};

// Eight elements of a row for each lane: next to each other where rows are aligned for it, otherwise as many apart as the group has lanes.
struct Lane {
    int first, step, width;   // element e is column first + e * step
    __device__ Lane(const EmbedArgs &a, int slab, int lane) {
        const int lanes = 1 << a.log_lanes;
        width = a.width;
        step = a.vector ? 1 : lanes;
        first = slab * 8 * lanes + (a.vector ? lane * 8 : lane);
    }
    __device__ bool some() const { return first < width; }
};

template <typename E, bool kVector>
__device__ __forceinline__ void read_eight(float (&x)[8], const E *row, const Lane &l) {
    if (kVector) {
        const Eight<E> v = *(const Eight<E> *)(row + l.first);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v.x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = l.first + e * l.step < l.width ? (float)row[l.first + e * l.step] : 0.0f;
    }
}
template <typename E, bool kVector>
__device__ __forceinline__ void write_eight(E *row, const float (&x)[8], const Lane &l) {
    if (kVector) {
        Eight<E> v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v.x[e] = (E)x[e];
        *(Eight<E> *)(row + l.first) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (l.first + e * l.step < l.width) row[l.first + e * l.step] = (E)x[e];
    }
}

// The id as an unsigned number; whatever lies outside the table is n_rows.
__device__ __forceinline__ uint32_t id_at(const void *ids, int id_bytes, int64_t i, int64_t n_rows) {
    const uint64_t id = id_bytes == 4 ? (uint64_t)(int64_t)((const int32_t *)ids)[i] : ((const uint64_t *)ids)[i];
    return (uint32_t)min(id, (uint64_t)n_rows);
}

// ------------------------------------------------------------------ lookup --
template <typename T, typename O, bool kVector>
__global__ __launch_bounds__(256) void embedding_kernel(EmbedArgs a) {
    const int lane = threadIdx.x & ((1 << a.log_lanes) - 1);
    const int64_t groups = (int64_t)gridDim.x * (256 >> a.log_lanes);
    for (int64_t i = (int64_t)blockIdx.x * (256 >> a.log_lanes) + (threadIdx.x >> a.log_lanes); i < a.n_ids; i += groups) {
        const uint32_t id = id_at(a.ids, a.id_bytes, i, a.n_rows);
        const T *row = (const T *)a.table + (int64_t)id * a.table_stride;
        O *to = (O *)a.out + i * a.out_stride;
#pragma unroll 4
        for (int slab = 0; slab < a.slabs; ++slab) {
            const Lane l(a, slab, lane);
            if (!l.some()) break;
            float x[8] = {};
            if (id < a.n_rows) {
                read_eight<T, kVector>(x, row, l);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= a.scale;
            }
            write_eight<O, kVector>(to, x, l);
        }
    }
}

// -------------------------------------------------------------------- sort --
// One pass of a stable sort by digits: each workgroup's tile of ids is counted by digit in one launch, and placed in the next, in which every workgroup
// adds up for itself what comes before its own.
__device__ __forceinline__ uint32_t sort_key(const SortPass &p, int64_t i) { return p.ids ? id_at(p.ids, p.id_bytes, i, p.n_rows) : p.key_in[i]; }

__global__ __launch_bounds__(512) void sort_count_kernel(SortPass p) {
    __shared__ uint32_t count[kSortDigits];
    const int digits = 1 << p.bits;
    for (int d = threadIdx.x; d < digits; d += 512) count[d] = 0;
    __syncthreads();
    const int64_t end = min(p.n, (blockIdx.x + 1) * p.tile);
    for (int64_t i = blockIdx.x * p.tile + threadIdx.x; i < end; i += 512) atomicAdd(&count[(sort_key(p, i) >> p.shift) & (digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += 512) p.hist[(int64_t)blockIdx.x * digits + d] = count[d];
}

__global__ __launch_bounds__(512) void sort_place_kernel(SortPass p) {
    __shared__ uint32_t total[kSortDigits], base[kSortDigits], count[8][kSortDigits], of_wave[8];
    const int digits = 1 << p.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < digits; d += 512) total[d] = base[d] = 0;
    __syncthreads();
    // all tiles' counts of each digit, and those of the tiles before this one
    const int stride = max(1, 512 / digits);
    for (int d = threadIdx.x & (digits - 1); d < digits; d += 512) {
        uint32_t all = 0, before = 0;
#pragma unroll 8
        for (int t = threadIdx.x / digits; t < p.tiles; t += stride) {
            const uint32_t c = p.hist[(int64_t)t * digits + d];
            all += c;
            before += t < (int)blockIdx.x ? c : 0;
        }
        atomicAdd(&total[d], all);
        atomicAdd(&base[d], before);
    }
    __syncthreads();
    // and those of the smaller digits: two neighbouring digits a thread
    const int d0 = 2 * threadIdx.x;
    const uint32_t c0 = d0 < digits ? total[d0] : 0, c1 = d0 + 1 < digits ? total[d0 + 1] : 0;
    uint32_t upto = c0 + c1;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t x = __shfl_up(upto, s);
        if (lane >= s) upto += x;
    }
    if (lane == 63) of_wave[wave] = upto;
    __syncthreads();
    uint32_t smaller = upto - c0 - c1;
    for (int w = 0; w < wave; ++w) smaller += of_wave[w];
    if (d0 < digits) base[d0] += smaller;
    if (d0 + 1 < digits) base[d0 + 1] += smaller + c0;

    const int64_t end = min(p.n, (blockIdx.x + 1) * p.tile);
    for (int64_t first = blockIdx.x * p.tile; first < end; first += kSortItems) {
        for (int d = threadIdx.x; d < 8 * digits; d += 512) count[d / digits][d & (digits - 1)] = 0;
        __syncthreads();
        // a wave ranks 512 ids in a row, 64 at a time
        uint32_t key[8], pos[8], rank[8];
        const int64_t mine = first + wave * 512 + lane;
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (mine + r * 64 < end) {
                key[r] = sort_key(p, mine + r * 64);
                pos[r] = p.ids ? (uint32_t)(mine + r * 64) : p.pos_in[mine + r * 64];
            }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const bool there = mine + r * 64 < end;
            const uint32_t digit = there ? (key[r] >> p.shift) & (digits - 1) : 0;
            uint64_t same = __ballot(there);
            for (int b = 0; b < p.bits; ++b) {
                const uint64_t with = __ballot((digit >> b) & 1);
                same &= (digit >> b) & 1 ? with : ~with;
            }
            if (there) {
                const int below = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
                volatile uint32_t *at = &count[wave][digit];
                const uint32_t before = *at;
                rank[r] = before + below;
                if (below == 0) *at = before + __popcll(same);
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        for (int d = threadIdx.x; d < digits; d += 512) {
            uint32_t at = base[d];
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const uint32_t c = count[w][d];
                count[w][d] = at;
                at += c;
            }
            base[d] = at;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (mine + r * 64 < end) {
                const uint32_t to = count[wave][(key[r] >> p.shift) & (digits - 1)] + rank[r];
                p.key_out[to] = key[r];
                p.pos_out[to] = pos[r];
            }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient --
template <typename T, bool kVector>
__device__ __forceinline__ void finish(const EmbedArgs &a, uint32_t id, float (&sum)[8], const Lane &l) {
    T *row = (T *)a.table + (int64_t)id * a.table_stride;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] *= a.scale;
    if (a.accumulate) {
        float old[8];
        read_eight<T, kVector>(old, row, l);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += old[e];
    }
    write_eight<T, kVector>(row, sum, l);
}

// The first sorted place from `from` on whose key is at least `key`.
__device__ __forceinline__ int64_t lower_bound(const uint32_t *keys, int64_t from, int64_t to, uint32_t key) {
    while (from < to) {
        const int64_t mid = (from + to) >> 1;
        if (keys[mid] < key) from = mid + 1;
        else to = mid;
    }
    return from;
}
// The same by a whole wave for one key, 64 places at a time: a step is a load's latency (of 900,000 four of them, not twenty).
__device__ __forceinline__ int64_t wave_lower_bound(const uint32_t *keys, int64_t from, int64_t to, uint32_t key) {
    const int lane = threadIdx.x & 63;
    while (from < to) {
        const int64_t step = (to - from + 63) / 64, at = from + lane * step;   // lane's place, the first of its stretch
        const int less = __popcll(__ballot(at < to && keys[min(at, to - 1)] < key));
        if (less == 0) return from;
        // the first `less` stretches begin below the key, so the bound is in the last of them or right behind it
        to = min(to, from + less * step);
        from += (less - 1) * step + 1;
    }
    return from;
}

// Workgroups before the first `sums` clear rows without places, the others add up chunks.
template <typename T, typename O, bool kVector>
__global__ __launch_bounds__(256) void embedding_sum_kernel(EmbedArgs a, unsigned sums) {
    constexpr int kAhead = 8;   // rows under way
    const float zeros[8] = {};
    if (blockIdx.x >= sums) {
        const int lane = threadIdx.x & 63;
        const int64_t row0 = ((int64_t)(blockIdx.x - sums) * 4 + (threadIdx.x >> 6)) * a.zero_rows, row1 = min(a.n_rows, row0 + a.zero_rows);
        if (row0 >= row1) return;
        const int64_t lo = wave_lower_bound(a.key, 0, a.n_ids, (uint32_t)row0), hi = wave_lower_bound(a.key, lo, a.n_ids, (uint32_t)row1);
        bool without = false;
        if (row0 + lane < row1) {
            const int64_t at = lower_bound(a.key, lo, hi, (uint32_t)(row0 + lane));
            without = at >= hi || a.key[at] != (uint32_t)(row0 + lane);
        }
        const int lanes = 1 << a.log_lanes, group = lane >> a.log_lanes, groups = 64 >> a.log_lanes;
        const uint64_t empty = __ballot(without);
        for (int r = group; r < row1 - row0; r += groups)
            if ((empty >> r) & 1)
                for (int slab = 0; slab < a.slabs; ++slab) {
                    const Lane l(a, slab, lane & (lanes - 1));
                    if (l.some()) write_eight<T, kVector>((T *)a.table + (row0 + r) * a.table_stride, zeros, l);
                }
        return;
    }
    const int64_t unit = (int64_t)blockIdx.x * (256 >> a.log_lanes) + (threadIdx.x >> a.log_lanes);
    const int chunk = (int)(unit / a.slabs), slab = (int)(unit % a.slabs);
    const Lane l(a, slab, threadIdx.x & ((1 << a.log_lanes) - 1));
    if (chunk >= a.chunks || !l.some()) return;
    const int64_t first = (int64_t)chunk * a.chunk;
    const int count = (int)min((int64_t)a.chunk, a.n_ids - first);
    const uint32_t *keys = a.key + first, *places = a.pos + first;
    const uint32_t none = (uint32_t)a.n_rows;
    uint32_t run = keys[0];
    if (run == none) return;
    bool from_left = first > 0 && keys[-1] == run;
    float *part = a.part + ((int64_t)chunk * 2 * a.slabs + slab) * (8 << a.log_lanes) + (threadIdx.x & ((1 << a.log_lanes) - 1)) * 8;
    const int64_t to_second = (int64_t)a.slabs * (8 << a.log_lanes);
    float sum[8] = {};
    auto put_aside = [&](float *to) {
        *(float4 *)to = float4{sum[0], sum[1], sum[2], sum[3]};
        *(float4 *)(to + 4) = float4{sum[4], sum[5], sum[6], sum[7]};
    };
    uint32_t next_key[kAhead], next_place[kAhead];
    auto fetch = [&](int i) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            next_key[u] = i + u < count ? keys[i + u] : none;
            next_place[u] = i + u < count ? places[i + u] : 0;
        }
    };
    fetch(0);
    for (int i = 0; i < count; i += kAhead) {
        uint32_t key[kAhead];
        float x[kAhead][8];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            key[u] = next_key[u];
            if (key[u] != none) read_eight<O, kVector>(x[u], (const O *)a.out + (int64_t)next_place[u] * a.out_stride, l);
        }
        fetch(i + kAhead);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (key[u] == none) break;
            if (key[u] != run) {
                if (from_left) put_aside(part);
                else finish<T, kVector>(a, run, sum, l);
                from_left = false;
                run = key[u];
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[u][e];
        }
    }
    if (from_left) put_aside(part);
    else if (first + count < a.n_ids && keys[count] == run) put_aside(part + to_second);
    else finish<T, kVector>(a, run, sum, l);
}

// By 256 threads, a group of lanes each an equal share of `count` rows, read by `row(i)` into eight floats; their sum to the first group, in a fixed order.
template <typename Read>
__device__ __forceinline__ void shared_sum(float (&sum)[8], int log_lanes, int count, float (*part)[8], Read read) {
    const int groups = 256 >> log_lanes, group = threadIdx.x >> log_lanes, each = (count + groups - 1) / groups;
    const int from = group * each, to = min(count, from + each);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
#pragma unroll 4
    for (int i = from; i < to; ++i) {
        float x[8];
        read(x, i);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += x[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) part[threadIdx.x][e] = sum[e];
    __syncthreads();
    if (group == 0)
        for (int g = 1; g < min(groups, (count + max(each, 1) - 1) / max(each, 1)); ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += part[(g << log_lanes) + threadIdx.x][e];
}

// The runs that begin in a chunk and go on: their parts, in the chunks' order.  Each of sixteen waves looks at a chunk; a run of up to kShortRun parts is its own
// affair, a longer one all waves'.  (As long as a run has more chunks than waves look at, at most one of them begins here.)
constexpr int kJoinWaves = 16, kShortRun = 16;
template <typename T, bool kVector>
__global__ __launch_bounds__(64 * kJoinWaves) void embedding_join_kernel(EmbedArgs a) {
    __shared__ float shared[64 * kJoinWaves][8];
    __shared__ int long_chunk, long_parts;
    __shared__ uint32_t long_run;
    const int slab = blockIdx.x % a.slabs, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t chunk = (int64_t)(blockIdx.x / a.slabs) * kJoinWaves + wave;
    const int lanes = 1 << a.log_lanes, groups = 64 >> a.log_lanes;
    const int64_t row = (int64_t)a.slabs * (8 << a.log_lanes), at = (int64_t)slab * (8 << a.log_lanes) + (lane & (lanes - 1)) * 8;
    const Lane l(a, slab, lane & (lanes - 1));
    if (threadIdx.x == 0) long_chunk = -1;
    __syncthreads();
    // how many parts the run that begins in this chunk has
    auto parts_of = [&](int64_t c, uint32_t *run) -> int {
        const int64_t first = c * a.chunk, last = first + a.chunk - 1;   // a whole chunk, or it would have no next one
        const uint32_t before = a.key[max(first - 1, (int64_t)0)], begin = a.key[first], behind = a.key[last + 1];
        *run = a.key[last];
        if (*run == (uint32_t)a.n_rows || behind != *run) return 0;
        if (begin == *run && first > 0 && before == *run) return 0;
        return (int)((wave_lower_bound(a.key, last + 1, a.n_ids, *run + 1) - 1) / a.chunk - c + 1);
    };
    // part i of the run that begins in chunk c
    auto add_part = [&](float (&sum)[8], int64_t c, int i) {
        const float *from = a.part + (c + i) * 2 * row + (i == 0 ? row : 0) + at;
        const float4 lo = *(const float4 *)from, hi = *(const float4 *)(from + 4);
        sum[0] += lo.x, sum[1] += lo.y, sum[2] += lo.z, sum[3] += lo.w, sum[4] += hi.x, sum[5] += hi.y, sum[6] += hi.z, sum[7] += hi.w;
    };
    // equal shares of the parts by `count` groups, of which this lane's is number `group`, to the first, in their order
    auto join = [&](int64_t c, int parts, int group, int count, float (&sum)[8]) {
        const int each = (parts + count - 1) / count, to = min(parts, (group + 1) * each);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
#pragma unroll 8
        for (int i = group * each; i < to; ++i) add_part(sum, c, i);
        return (parts + each - 1) / each;   // groups with a share
    };
    // the same, by sums of 64 parts in 64 bits: a run of 2^24 places was off by 1.5e-4 where they are equal and each addition is rounded the same way
    auto join_long = [&](int64_t c, int parts, int group, int count, double (&total)[8]) {
        const int each = (parts + count - 1) / count, to = min(parts, (group + 1) * each);
#pragma unroll
        for (int e = 0; e < 8; ++e) total[e] = 0.0;
        for (int i0 = group * each; i0 < to; i0 += 64) {
            float sum[8] = {};
#pragma unroll 8
            for (int i = i0; i < min(to, i0 + 64); ++i) add_part(sum, c, i);
#pragma unroll
            for (int e = 0; e < 8; ++e) total[e] += (double)sum[e];
        }
        return (parts + each - 1) / each;
    };
    uint32_t run = 0;
    const int parts = chunk < a.chunks - 1 ? parts_of(chunk, &run) : 0;
    float sum[8];
    if (parts > kShortRun) {
        if (lane == 0) long_chunk = (int)chunk, long_parts = parts, long_run = run;
    } else if (parts > 0) {
        const int shares = join(chunk, parts, lane >> a.log_lanes, groups, sum);
        for (int g = 1; g < shares; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __shfl(sum[e], (g << a.log_lanes) + (lane & (lanes - 1)));
                if (lane < lanes) sum[e] += x;
            }
        if (lane < lanes && l.some()) finish<T, kVector>(a, run, sum, l);
    }
    __syncthreads();
    const int c = long_chunk;
    if (c < 0) return;
    double total[8];
    const int shares = join_long(c, long_parts, threadIdx.x >> a.log_lanes, groups * kJoinWaves, total);
#pragma unroll
    for (int e = 0; e < 8; ++e) shared[threadIdx.x][e] = (float)total[e];
    __syncthreads();
    if (threadIdx.x >= (unsigned)lanes) return;
    for (int g = 1; g < shares; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) total[e] += (double)shared[(g << a.log_lanes) + threadIdx.x][e];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = (float)total[e];
    if (l.some()) finish<T, kVector>(a, long_run, sum, l);
}

// Few ids: a workgroup owns some rows of the table, and looks through all ids for theirs.  One launch, nothing sorted.
template <typename T, typename O, bool kVector>
__global__ __launch_bounds__(256) void embedding_few_kernel(EmbedArgs a) {
    __shared__ float shared[256][8];
    __shared__ uint16_t place[kEmbedFewIds];
    __shared__ uint8_t of_row[kEmbedFewIds];
    __shared__ int of_wave[4];
    __shared__ uint32_t present;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slab = blockIdx.x % a.slabs;
    const int64_t row0 = (int64_t)(blockIdx.x / a.slabs) * a.zero_rows;
    const int rows = (int)min((int64_t)a.zero_rows, a.n_rows - row0);
    if (threadIdx.x == 0) present = 0;
    int found = 0;
    for (int first = 0; first < (int)a.n_ids; first += 256) {
        const int i = first + threadIdx.x;
        const int64_t r = i < (int)a.n_ids ? (int64_t)id_at(a.ids, a.id_bytes, i, a.n_rows) - row0 : -1;
        const bool mine = r >= 0 && r < rows;
        const uint64_t some = __ballot(mine);
        if (lane == 0) of_wave[wave] = __popcll(some);
        __syncthreads();
        int at = found + __builtin_amdgcn_mbcnt_hi((uint32_t)(some >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)some, 0u));
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            at += w < wave ? of_wave[w] : 0;
            found += of_wave[w];
        }
        if (mine) {
            place[at] = (uint16_t)i;
            of_row[at] = (uint8_t)r;
            atomicOr(&present, 1u << r);
        }
        __syncthreads();
    }
    __syncthreads();
    const Lane l(a, slab, threadIdx.x & ((1 << a.log_lanes) - 1));
    const float zeros[8] = {};
    const uint32_t there = present;
    if (!a.accumulate && l.some())
        for (int r = threadIdx.x >> a.log_lanes; r < rows; r += 256 >> a.log_lanes)
            if (!((there >> r) & 1)) write_eight<T, kVector>((T *)a.table + (row0 + r) * a.table_stride, zeros, l);
    for (uint32_t left = there; left; left &= left - 1) {
        const int r = __ffs(left) - 1;
        float sum[8];
        shared_sum(sum, a.log_lanes, found, shared, [&](float (&x)[8], int i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.0f;
            if (l.some() && of_row[i] == r) read_eight<O, kVector>(x, (const O *)a.out + (int64_t)place[i] * a.out_stride, l);
        });
        if (threadIdx.x < (1u << a.log_lanes) && l.some()) finish<T, kVector>(a, (uint32_t)(row0 + r), sum, l);
    }
}

// Few rows: every lane has its eight columns of all of them in LDS (2 KB a row and wave), and adds a place's row to the one that its id names.  Ids and
// gradients are read once, as they lie, and nothing is sorted: a wave's 8 places of 64 columns are 1 KB side by side.  An addition waits for the one before it, which
// may be of the same row, some 150 cycles; two to four waves on a compute unit make 13 to 27 bytes a cycle of that, and HBM has 9 for each.  A lane's sixteen bytes
// lie 64 to a line whatever their row, so no two of a wave's lanes meet in a bank.  900,000 places of 12 rows of 64 elements, bfloat16: 31 us and 8 to join
// (3.9 TB/s; 58 where the next rows' registers were copied, which waits for them).
// All reads are made, of some place and column where there is none: loads that nobody skips can be counted, and those of the next places stay under way.
template <typename O, bool kVector>
__device__ __forceinline__ void read_raw(Eight<O> &x, const O *row, const Lane &l) {
    if (kVector) {
        x = *(const Eight<O> *)(row + (l.some() ? l.first : 0));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x.x[e] = row[min(l.first + e * l.step, l.width - 1)];
    }
}

// A group of lanes adds at most kBehind places up behind one another, then the wave's sums go to those before: an addition is off by half a step of its sum, and
// a sum of 2^17 equal places, of which each is rounded the same way, was off by 1e-3.
template <typename O, bool kVector>
__global__ __launch_bounds__(64) void embedding_rows_kernel(EmbedArgs a) {
    constexpr int kAhead = 8;   // places of a group whose rows are under way while as many are added up
    constexpr int kBehind = 512;
    extern __shared__ __attribute__((aligned(16))) float4 sums[];   // [n_rows][2][64]
    const int lane = threadIdx.x, lanes = 1 << a.log_lanes, groups = 64 >> a.log_lanes, group = lane >> a.log_lanes, rows = (int)a.n_rows;
    const int64_t begin = (int64_t)blockIdx.x * a.chunk, end = min(a.n_ids, begin + a.chunk);
    const Lane l(a, 0, lane & (lanes - 1));
    uint32_t seen = 0;
    for (int64_t first = begin; first < end; first += kBehind * groups) {
        const int count = (int)min((int64_t)(kBehind * groups), end - first);
        for (int r = 0; r < 2 * rows; ++r) sums[r * 64 + lane] = float4{0.0f, 0.0f, 0.0f, 0.0f};
        struct Places {
            uint32_t id[kAhead];
            Eight<O> x[kAhead];
        } even, odd;
        auto fetch_ids = [&](Places &p, int i) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t id = id_at(a.ids, a.id_bytes, first + min(i + u * groups, count - 1), rows);
                p.id[u] = i + u * groups < count ? id : (uint32_t)rows;
            }
        };
        auto fetch_rows = [&](Places &p, int i) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) read_raw<O, kVector>(p.x[u], (const O *)a.out + (first + min(i + u * groups, count - 1)) * a.out_stride, l);
        };
        auto add = [&](const Places &p) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const bool there = p.id[u] < (uint32_t)rows;
                const uint32_t row = there ? p.id[u] : 0;
                seen |= (uint32_t)there << row;
                float4 *to = sums + row * 128 + lane, lo = to[0], hi = to[64];
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = there ? (float)p.x[u].x[e] : 0.0f;
                lo.x += x[0], lo.y += x[1], lo.z += x[2], lo.w += x[3], hi.x += x[4], hi.y += x[5], hi.z += x[6], hi.w += x[7];
                to[0] = lo, to[64] = hi;
            }
        };
        const int step = kAhead * groups;
        fetch_ids(even, group);
        fetch_rows(even, group);
        for (int i = group; i < count + group; i += 2 * step) {   // the same for all groups
            fetch_ids(odd, i + step);
            fetch_rows(odd, i + step);
            add(even);
            fetch_ids(even, i + 2 * step);
            fetch_rows(even, i + 2 * step);
            add(odd);
        }
        __syncthreads();
        // the wave's groups, for each lane from another one on, so that no two meet in a bank
        float *part = a.part + (int64_t)blockIdx.x * rows * 8 * lanes;
        for (int o = lane; o < 2 * rows * lanes; o += 64) {
            const int r = o >> a.log_lanes, at = o & (lanes - 1);
            float4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
            for (int g = 0; g < groups; ++g) {
                const float4 x = sums[r * 64 + (((g + r) & (groups - 1)) << a.log_lanes) + at];
                v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
            }
            float4 *to = (float4 *)(part + ((r >> 1) * lanes + at) * 8 + (r & 1) * 4);
            if (first > begin) {
                const float4 x = *to;
                v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
            }
            *to = v;
        }
        __syncthreads();
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) seen |= __shfl_xor(seen, s);
    if (lane == 0) a.seen[blockIdx.x] = seen;
}

// The waves' sums of one row, an equal share of them by each group of lanes, in a fixed order.
template <typename T, bool kVector>
__global__ __launch_bounds__(1024) void embedding_rows_join_kernel(EmbedArgs a) {
    __shared__ float shared[16][64][8];
    const int row = blockIdx.x, lanes = 1 << a.log_lanes, at = threadIdx.x & (lanes - 1), width = 8 << a.log_lanes;
    const int groups = 1024 >> a.log_lanes, group = threadIdx.x >> a.log_lanes, each = (a.chunks + groups - 1) / groups, to = min(a.chunks, (group + 1) * each);
    float sum[8] = {};
#pragma unroll 8
    for (int i = group * each; i < to; ++i) {
        const float *from = a.part + ((int64_t)i * a.n_rows + row) * width + at * 8;
        const float4 lo = *(const float4 *)from, hi = *(const float4 *)(from + 4);
        sum[0] += lo.x, sum[1] += lo.y, sum[2] += lo.z, sum[3] += lo.w, sum[4] += hi.x, sum[5] += hi.y, sum[6] += hi.z, sum[7] += hi.w;
    }
    uint32_t seen = 0;
    for (int i = threadIdx.x; i < a.chunks; i += 1024) seen |= a.seen[i];
#pragma unroll
    for (int s = 0; s < 6; ++s)
        if (s >= a.log_lanes)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += __shfl_xor(sum[e], 1 << s);
#pragma unroll
    for (int e = 0; e < 8; ++e) shared[threadIdx.x >> 6][threadIdx.x & 63][e] = sum[e];
    const bool some = __syncthreads_or((seen >> row) & 1);
    const Lane l(a, 0, at);
    if (threadIdx.x >= (unsigned)lanes || !l.some()) return;
    if (!some) {   // no place has this id
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
        if (!a.accumulate) write_eight<T, kVector>((T *)a.table + row * a.table_stride, sum, l);
        return;
    }
    for (int w = 1; w < 16; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += shared[w][at][e];
    finish<T, kVector>(a, (uint32_t)row, sum, l);
}

template <typename Launch>
void by_type(int dtype, Launch launch) {
    if (dtype == GBT_F32) launch(0.0f);
    else if (dtype == GBT_BF16) launch((__bf16)0.0f);
    else launch((_Float16)0.0f);
}
constexpr int64_t kMostWorkgroups = 1 << 16;   // of the lookup, which goes on with the next ids

}  // namespace

hipError_t gbt_launch_embedding(hipStream_t stream, const EmbedArgs &a) {
    const int each = 256 >> a.log_lanes;
    const unsigned grid = (unsigned)std::min<int64_t>((a.n_ids + each - 1) / each, kMostWorkgroups);
    by_type(a.table_dtype, [&](auto t) {
        by_type(a.out_dtype, [&](auto o) {
            if (a.vector) embedding_kernel<decltype(t), decltype(o), true><<<grid, 256, 0, stream>>>(a);
            else embedding_kernel<decltype(t), decltype(o), false><<<grid, 256, 0, stream>>>(a);
        });
    });
    return hipGetLastError();
}

hipError_t gbt_launch_sort_pass(hipStream_t stream, const SortPass &p) {
    sort_count_kernel<<<p.tiles, 512, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    sort_place_kernel<<<p.tiles, 512, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t gbt_launch_embedding_grad(hipStream_t stream, const EmbedArgs &a) {
    const int64_t units = (int64_t)a.chunks * a.slabs, each = 256 >> a.log_lanes;
    const unsigned sums = (unsigned)((units + each - 1) / each);
    const int64_t waves = (a.n_rows + a.zero_rows - 1) / a.zero_rows;
    const unsigned clears = a.accumulate ? 0 : (unsigned)((waves + 3) / 4);
    by_type(a.table_dtype, [&](auto t) {
        by_type(a.out_dtype, [&](auto o) {
            if (a.vector) embedding_sum_kernel<decltype(t), decltype(o), true><<<sums + clears, 256, 0, stream>>>(a, sums);
            else embedding_sum_kernel<decltype(t), decltype(o), false><<<sums + clears, 256, 0, stream>>>(a, sums);
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.chunks < 2) return e;
    by_type(a.table_dtype, [&](auto t) {
        const unsigned grid = (unsigned)((a.chunks - 1 + kJoinWaves - 1) / kJoinWaves * a.slabs);
        if (a.vector) embedding_join_kernel<decltype(t), true><<<grid, 64 * kJoinWaves, 0, stream>>>(a);
        else embedding_join_kernel<decltype(t), false><<<grid, 64 * kJoinWaves, 0, stream>>>(a);
    });
    return hipGetLastError();
}

hipError_t gbt_launch_embedding_grad_rows(hipStream_t stream, const EmbedArgs &a) {
    by_type(a.out_dtype, [&](auto o) {
        const unsigned grid = (unsigned)a.chunks;
        if (a.vector) embedding_rows_kernel<decltype(o), true><<<grid, 64, a.n_rows * 2048, stream>>>(a);
        else embedding_rows_kernel<decltype(o), false><<<grid, 64, a.n_rows * 2048, stream>>>(a);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    by_type(a.table_dtype, [&](auto t) {
        const unsigned grid = (unsigned)a.n_rows;
        if (a.vector) embedding_rows_join_kernel<decltype(t), true><<<grid, 1024, 0, stream>>>(a);
        else embedding_rows_join_kernel<decltype(t), false><<<grid, 1024, 0, stream>>>(a);
    });
    return hipGetLastError();
}

hipError_t gbt_launch_embedding_grad_few(hipStream_t stream, const EmbedArgs &a) {
    const unsigned grid = (unsigned)((a.n_rows + a.zero_rows - 1) / a.zero_rows * a.slabs);
    by_type(a.table_dtype, [&](auto t) {
        by_type(a.out_dtype, [&](auto o) {
            if (a.vector) embedding_few_kernel<decltype(t), decltype(o), true><<<grid, 256, 0, stream>>>(a);
            else embedding_few_kernel<decltype(t), decltype(o), false><<<grid, 256, 0, stream>>>(a);
        });
    });
    return hipGetLastError();
}
