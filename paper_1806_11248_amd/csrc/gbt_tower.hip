// The C ABI of the operators around a tower over histories (see include/gbt.h): checks of arguments, workspaces, launches.
#include <string.h>

#include <new>

#include "embedding.h"
#include "norm_rotate.h"
#include "ortho.h"

namespace {

bool known_type(int32_t dtype) { return dtype == GBT_F32 || dtype == GBT_BF16 || dtype == GBT_F16; }
int64_t size_of(int32_t dtype) { return dtype == GBT_F32 ? 4 : 2; }
constexpr int64_t kMostWorkgroups = (1 << 23) - 1024;   // of a launch, of up to 512 threads, of which there can be 2^32

// --------------------------------------------------------------- embedding --
const char *embedding_fault(const gbt_embedding_params &p, int32_t *code) {
    *code = GBT_EUNSUPPORTED;
    if (!known_type(p.table_dtype) || !known_type(p.out_dtype)) return "table_dtype or out_dtype is none of GBT_F32, GBT_BF16, GBT_F16";
    if (p.n_ids > ((int64_t)1 << 30)) return "more than 2^30 ids";
    if (p.n_rows > ((int64_t)1 << 30)) return "more than 2^30 rows";
    if (p.width > (1 << 20)) return "width > 2^20";
    *code = GBT_EINVAL;
    if (p.id_bytes != 4 && p.id_bytes != 8) return "id_bytes is neither 4 nor 8";
    if (p.n_ids < 0 || p.n_rows < 0 || p.width < 1) return "n_ids, n_rows or width out of range";
    if (p.table_stride < 0 || p.out_stride < 0 || p.table_stride > ((int64_t)1 << 40) || p.out_stride > ((int64_t)1 << 40)) return "a stride out of range";
    if (!isfinite(p.scale)) return "scale is not finite";
    if (p.n_ids > 0 && (!p.ids || ((uintptr_t)p.ids & (uintptr_t)(p.id_bytes - 1)))) return "ids is NULL or not aligned";
    return nullptr;
}
bool rows_of_eight(const void *x, int64_t stride, int64_t size) { return ((uintptr_t)x & 15u) == 0 && stride * size % 16 == 0; }

void fill(EmbedArgs &a, const gbt_embedding_params &p, const void *table, void *out) {
    memset(&a, 0, sizeof a);
    a.ids = p.ids;
    a.id_bytes = p.id_bytes;
    a.width = p.width;
    while (a.log_lanes < 6 && (8 << a.log_lanes) < p.width) ++a.log_lanes;
    a.slabs = (p.width + (8 << a.log_lanes) - 1) / (8 << a.log_lanes);
    a.vector = p.width % 8 == 0 && rows_of_eight(table, p.table_stride, size_of(p.table_dtype)) && rows_of_eight(out, p.out_stride, size_of(p.out_dtype));
    a.n_ids = p.n_ids;
    a.n_rows = p.n_rows;
    a.table_stride = p.table_stride;
    a.out_stride = p.out_stride;
    a.scale = p.scale;
    a.table = table;
    a.out = out;
    a.table_dtype = p.table_dtype;
    a.out_dtype = p.out_dtype;
}

// Few ids are looked for by the workgroups that own rows, unless these are too many.  (us, bfloat16, of ids, rows and columns by those and sorted: 32 of 40 of 64 7.5 and 16;
// 2000 8.0 and 22; 2000 of 40 of 2048 10 and 23; 500 of 5000 of 512 7.8 and 30, 2000 12 and 34; 2000 of 100,000 of 512 41 and 64.  Only where ids are many and rows so few
// that most compute units own none it loses: 500 of 2 of 2048 21 and 25, 2048 73 and 22.)
constexpr int64_t kFewRowsWorkgroups = 4096;   // aimed at; a workgroup owns 32 rows at most
bool takes_few_ids(const gbt_embedding_params &p) { return p.n_ids <= kEmbedFewIds && p.n_rows <= kFewRowsWorkgroups * 32; }

struct SortLayout {
    int passes, bits[4], tiles;
    int64_t tile, chunk, chunks;
    size_t key[2], pos[2], hist, part, bytes;
};
SortLayout sort_layout(const gbt_embedding_params &p) {
    SortLayout l;
    int bits = 1;
    while (bits < 31 && ((int64_t)1 << bits) <= p.n_rows) ++bits;   // n_rows itself is a key
    l.passes = (bits + 9) / 10;
    for (int i = 0; i < l.passes; ++i) l.bits[i] = bits / l.passes + (i < bits % l.passes);
    l.tile = ((p.n_ids + kSortTiles - 1) / kSortTiles + kSortItems - 1) / kSortItems * kSortItems;
    l.tiles = (int)((p.n_ids + l.tile - 1) / l.tile);
    EmbedArgs a;
    fill(a, p, nullptr, nullptr);
    // Places that a group of lanes adds up: as many as leave some 4000 waves.  (us of the sums and of joining them for chunks of 16, 32, 64, 128: 900,000 ids
    // of 12 rows of 64 elements 31 + 36, 25 + 21, 41 + 15, 78 + 11; 32,768 of 120,000 rows of 2048 225 + 24, 220 + 15, 266 + 12, 317 + 8.)
    const int64_t per_wave = 64 >> a.log_lanes;
    l.chunk = std::min<int64_t>(64, std::max<int64_t>(16, (p.n_ids * a.slabs / (4096 * per_wave) + 7) / 8 * 8));
    while ((p.n_ids + l.chunk - 1) / l.chunk * a.slabs > kMostWorkgroups) l.chunk *= 2;
    l.chunks = (p.n_ids + l.chunk - 1) / l.chunk;
    const size_t list = gbt_align((size_t)p.n_ids * 4);
    l.key[0] = 0, l.key[1] = list, l.pos[0] = 2 * list, l.pos[1] = 3 * list;
    l.hist = 4 * list;
    l.part = l.hist + gbt_align((size_t)l.tiles * kSortDigits * 4);
    l.bytes = l.part + (size_t)l.chunks * 2 * a.slabs * (8 << a.log_lanes) * 4;
    return l;
}

// Few rows are added up in LDS, up to a width of which a wave takes two places at once: wider ones wait for too many additions behind one another.  (us, bfloat16,
// of 32 rows in LDS and 33 sorted: 900,000 places of 64 elements 52 and 59, of 8 16 and 87; 10,000 of 64 12 and 26; 2,100 of 256 17 and 22, 30,000 30 and
// 28, 200,000 57 and 56; 30,000 of 512 42 and 31.  Of 12 rows the first takes 37, and took 86 sorted.)
bool takes_few_rows(const gbt_embedding_params &p) { return !takes_few_ids(p) && p.n_rows <= kEmbedFewRows && p.width <= 256 && p.n_rows > 0 && p.n_ids > 0; }
// By up to four waves on a compute unit, as many as its LDS takes (three for 24 rows, two for 32), of at least 16 places for each group of lanes.
struct RowsLayout {
    int64_t chunk, chunks;
    size_t seen, bytes;
};
RowsLayout rows_layout(const gbt_embedding_params &p) {
    RowsLayout l;
    EmbedArgs a;
    fill(a, p, nullptr, nullptr);
    const int64_t waves = 256 * std::min<int64_t>(4, 80 / p.n_rows), step = 8 * (64 >> a.log_lanes);
    l.chunk = (std::max((p.n_ids + waves - 1) / waves, 2 * step) + step - 1) / step * step;
    l.chunks = (p.n_ids + l.chunk - 1) / l.chunk;
    l.seen = (size_t)l.chunks * p.n_rows * (8 << a.log_lanes) * 4;
    l.bytes = l.seen + gbt_align((size_t)l.chunks * 4);
    return l;
}

}  // namespace

extern "C" int32_t gbt_embedding(gbt_ctx *ctx, const gbt_embedding_params *params, const void *table, void *out) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, params, GBT_EINVAL, "NULL argument");
    const gbt_embedding_params &p = *params;
    int32_t code;
    const char *fault = embedding_fault(p, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    GBT_REQUIRE(ctx, (table || p.n_rows == 0) && (out || p.n_ids == 0), GBT_EINVAL, "table or out is NULL");
    GBT_REQUIRE(ctx, (((uintptr_t)table & (uintptr_t)(size_of(p.table_dtype) - 1)) | ((uintptr_t)out & (uintptr_t)(size_of(p.out_dtype) - 1))) == 0, GBT_EINVAL,
                "table or out is not aligned");
    GBT_REQUIRE(ctx, p.out_stride >= p.width || p.n_ids <= 1, GBT_EINVAL, "out: rows overlap");
    if (p.n_ids == 0) return GBT_OK;
    EmbedArgs a;
    fill(a, p, table, out);
    GBT_HIP(ctx, gbt_launch_embedding(ctx->stream, a));
    return GBT_OK;
}

extern "C" size_t gbt_embedding_backward_workspace_bytes(const gbt_embedding_params *params) {
    int32_t code;
    if (!params || embedding_fault(*params, &code) || takes_few_ids(*params) || params->n_ids == 0) return 0;
    return takes_few_rows(*params) ? rows_layout(*params).bytes : sort_layout(*params).bytes;
}

extern "C" int32_t gbt_embedding_backward(gbt_ctx *ctx, const gbt_embedding_params *params, const void *dout, void *grad, int32_t accumulate,
                                          void *workspace, size_t workspace_bytes) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, params, GBT_EINVAL, "NULL argument");
    const gbt_embedding_params &p = *params;
    int32_t code;
    const char *fault = embedding_fault(p, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    GBT_REQUIRE(ctx, (grad || p.n_rows == 0) && (dout || p.n_ids == 0), GBT_EINVAL, "dout or grad is NULL");
    GBT_REQUIRE(ctx, (((uintptr_t)grad & (uintptr_t)(size_of(p.table_dtype) - 1)) | ((uintptr_t)dout & (uintptr_t)(size_of(p.out_dtype) - 1))) == 0, GBT_EINVAL,
                "dout or grad is not aligned");
    GBT_REQUIRE(ctx, p.table_stride >= p.width || p.n_rows <= 1, GBT_EINVAL, "grad: rows overlap");
    const size_t need = gbt_embedding_backward_workspace_bytes(params);
    GBT_REQUIRE(ctx, workspace || need == 0, GBT_EINVAL, "workspace is NULL");
    GBT_REQUIRE(ctx, workspace_bytes >= need, GBT_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    GBT_REQUIRE(ctx, ((uintptr_t)workspace & 15u) == 0 || need == 0, GBT_EINVAL, "workspace is not 16-byte aligned");
    if (p.n_rows == 0 || (p.n_ids == 0 && accumulate)) return GBT_OK;
    EmbedArgs a;
    fill(a, p, grad, const_cast<void *>(dout));
    a.accumulate = accumulate != 0;
    if (takes_few_ids(p)) {
        a.zero_rows = (int)((p.n_rows + kFewRowsWorkgroups - 1) / kFewRowsWorkgroups);
        GBT_HIP(ctx, gbt_launch_embedding_grad_few(ctx->stream, a));
        return GBT_OK;
    }
    if (takes_few_rows(p)) {
        const RowsLayout l = rows_layout(p);
        a.part = (float *)workspace;
        a.seen = (uint32_t *)((char *)workspace + l.seen);
        a.chunk = (int)l.chunk;
        a.chunks = (int)l.chunks;
        GBT_HIP(ctx, gbt_launch_embedding_grad_rows(ctx->stream, a));
        return GBT_OK;
    }
    // rows that a wave clears: as many as leave some 8000 waves
    a.zero_rows = (int)std::min<int64_t>(64, std::max<int64_t>(1, p.n_rows / 8192));
    if (p.n_ids > 0) {
        const SortLayout l = sort_layout(p);
        char *ws = (char *)workspace;
        SortPass s;
        memset(&s, 0, sizeof s);
        s.id_bytes = p.id_bytes;
        s.n = p.n_ids;
        s.n_rows = p.n_rows;
        s.tile = l.tile;
        s.tiles = l.tiles;
        s.hist = (uint32_t *)(ws + l.hist);
        for (int i = 0; i < l.passes; ++i) {
            s.ids = i == 0 ? p.ids : nullptr;
            s.key_in = (const uint32_t *)(ws + l.key[(i + 1) & 1]);
            s.pos_in = (const uint32_t *)(ws + l.pos[(i + 1) & 1]);
            s.key_out = (uint32_t *)(ws + l.key[i & 1]);
            s.pos_out = (uint32_t *)(ws + l.pos[i & 1]);
            s.bits = l.bits[i];
            GBT_HIP(ctx, gbt_launch_sort_pass(ctx->stream, s));
            s.shift += s.bits;
        }
        a.key = s.key_out;
        a.pos = s.pos_out;
        a.part = (float *)(ws + l.part);
        a.chunk = (int)l.chunk;
        a.chunks = (int)l.chunks;
    }
    GBT_HIP(ctx, gbt_launch_embedding_grad(ctx->stream, a));
    return GBT_OK;
}

// ------------------------------------------------- head norms and rotation --
namespace {

const char *rotate_fault(const gbt_norm_rotate_params &p, int32_t *code) {
    *code = GBT_EUNSUPPORTED;
    if (p.dtype != GBT_BF16 && p.dtype != GBT_F16) return "dtype is neither GBT_BF16 nor GBT_F16";
    if (p.head_dim < 8 || p.head_dim > GBT_MAX_HEAD_DIM || p.head_dim % 8) return "head_dim is no multiple of 8 in 8..128";
    if (p.turned % 8) return "turned is no multiple of 8";
    *code = GBT_EINVAL;
    if (p.heads < 1 || p.kv_heads < 1 || p.heads > (1 << 16) || p.kv_heads > (1 << 16)) return "heads or kv_heads out of range";
    if (p.turned < 0 || p.turned > p.head_dim) return "turned outside 0..head_dim";
    if (p.rows < 0 || p.rows > ((int64_t)1 << 40) || p.out_rows < 0 || p.out_rows > ((int64_t)1 << 40)) return "rows or out_rows out of range";
    if (p.n_seq < 0) return "n_seq < 0";
    if (!p.q_ptr && p.n_seq > 0 && p.rows % p.n_seq) return "rows is no multiple of n_seq without q_ptr";
    if (p.store && !p.k_ptr && p.n_seq > 0 && p.out_rows % p.n_seq) return "out_rows is no multiple of n_seq without k_ptr";
    if (!p.store && p.out_rows != p.rows) return "out_rows is not rows without a store";
    if (!(p.eps >= 0.0f && p.eps <= 1.0f)) return "eps outside 0..1";
    if (p.positions && p.position_bytes != 4 && p.position_bytes != 8) return "position_bytes is neither 4 nor 8";
    if (p.positions && ((uintptr_t)p.positions & (uintptr_t)(p.position_bytes - 1))) return "positions is not aligned";
    if (p.turned > 0 && (!p.turns || ((uintptr_t)p.turns & 7u))) return "turns is NULL or not aligned";
    if ((((uintptr_t)p.q_weight | (uintptr_t)p.k_weight | (uintptr_t)p.k_len) & 3u) || (((uintptr_t)p.q_ptr | (uintptr_t)p.k_ptr) & 7u))
        return "a weight or pointer array is not aligned";
    return nullptr;
}

void fill(RotateArgs &a, const gbt_norm_rotate_params &p) {
    memset(&a, 0, sizeof a);
    a.q_ptr = p.q_ptr;
    a.k_ptr = p.k_ptr;
    a.k_len = p.k_len;
    a.positions = p.positions;
    a.position_bytes = p.position_bytes;
    a.q_weight = p.q_weight;
    a.k_weight = p.k_weight;
    a.turns = p.turns;
    a.rows = p.rows;
    a.out_rows = p.out_rows;
    a.n_seq = p.n_seq;
    a.heads = p.heads;
    a.kv_heads = p.kv_heads;
    a.dim = p.head_dim;
    a.turned = p.turned;
    a.halves = p.halves != 0;
    a.store = p.store != 0;
    a.slots = p.k_ptr || p.k_len;
    a.eps = p.eps;
    while ((8 << a.log_lanes) < p.head_dim) ++a.log_lanes;
    const int at_once = 64 >> a.log_lanes;
    a.row_group = std::max(1, at_once / std::max(p.heads, p.kv_heads));
    a.parts = 1;
}
constexpr int kRotateBlocks = 2048;        // workgroups of four waves, which go on with the next rows
constexpr int kRotateGradBlocks = 1024;    // each leaves a sum of the weights' gradients

}  // namespace

extern "C" int32_t gbt_norm_rotate(gbt_ctx *ctx, const gbt_norm_rotate_params *params, const gbt_heads *q, const gbt_heads *k, const gbt_heads *v,
                                   const gbt_heads *q_out, const gbt_heads *k_out, const gbt_heads *v_out) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, params, GBT_EINVAL, "NULL argument");
    const gbt_norm_rotate_params &p = *params;
    int32_t code;
    const char *fault = rotate_fault(p, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    GBT_REQUIRE(ctx, !v == !v_out, GBT_EINVAL, "v and v_out: one without the other");
    GBT_VIEW(ctx, q, p.rows);
    GBT_VIEW(ctx, k, p.rows);
    GBT_VIEW_OUT(ctx, q_out, p.rows, p.heads);
    GBT_VIEW_OUT(ctx, k_out, p.out_rows, p.kv_heads);
    if (v) {
        GBT_VIEW(ctx, v, p.rows);
        GBT_VIEW_OUT(ctx, v_out, p.out_rows, p.kv_heads);
    }
    if (p.rows == 0) return GBT_OK;
    RotateArgs a;
    fill(a, p);
    a.q = view(q);
    a.k = view(k);
    a.q_out = view(q_out);
    a.k_out = view(k_out);
    if (v) {
        a.v = view(v);
        a.v_out = view(v_out);
    }
    const int64_t groups = (p.rows + a.row_group - 1) / a.row_group;
    const int at_once = 64 >> a.log_lanes, passes = (p.heads + at_once - 1) / at_once + (v ? 2 : 1) * ((p.kv_heads + at_once - 1) / at_once);
    if (groups * passes <= 4 * kRotateBlocks) a.parts = passes;   // few rows: a wave for each of a row's passes
    a.blocks = (int)std::min<int64_t>((groups * a.parts + 3) / 4, kRotateBlocks);
    GBT_HIP(ctx, gbt_launch_norm_rotate(ctx->stream, a, p.dtype));
    return GBT_OK;
}

extern "C" size_t gbt_norm_rotate_backward_workspace_bytes(const gbt_norm_rotate_params *params) {
    int32_t code;
    if (!params || rotate_fault(*params, &code)) return 0;
    return (size_t)kRotateGradBlocks * kRotateDim * sizeof(float);
}

extern "C" int32_t gbt_norm_rotate_backward(gbt_ctx *ctx, const gbt_norm_rotate_params *params, const gbt_heads *dq_out, const gbt_heads *dk_out,
                                            const gbt_heads *q, const gbt_heads *k, const gbt_heads *dq, const gbt_heads *dk, float *dq_weight,
                                            float *dk_weight, void *workspace, size_t workspace_bytes) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, params, GBT_EINVAL, "NULL argument");
    const gbt_norm_rotate_params &p = *params;
    int32_t code;
    const char *fault = rotate_fault(p, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    GBT_REQUIRE(ctx, !p.store, GBT_EUNSUPPORTED, "the gradient of keys in a store");
    GBT_VIEW(ctx, dq_out, p.rows);
    GBT_VIEW(ctx, dk_out, p.rows);
    GBT_VIEW(ctx, q, p.rows);
    GBT_VIEW(ctx, k, p.rows);
    GBT_VIEW_OUT(ctx, dq, p.rows, p.heads);
    GBT_VIEW_OUT(ctx, dk, p.rows, p.kv_heads);
    GBT_REQUIRE(ctx, dq_weight && dk_weight && (((uintptr_t)dq_weight | (uintptr_t)dk_weight) & 3u) == 0, GBT_EINVAL,
                "dq_weight or dk_weight is NULL or not aligned");
    const size_t need = gbt_norm_rotate_backward_workspace_bytes(params);
    GBT_REQUIRE(ctx, workspace, GBT_EINVAL, "workspace is NULL");
    GBT_REQUIRE(ctx, workspace_bytes >= need, GBT_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    GBT_REQUIRE(ctx, ((uintptr_t)workspace & 15u) == 0, GBT_EINVAL, "workspace is not 16-byte aligned");
    RotateArgs a;
    fill(a, p);
    a.q = view(q);
    a.k = view(k);
    a.q_out = view(dq_out);
    a.k_out = view(dk_out);
    a.dq = view(dq);
    a.dk = view(dk);
    a.dq_weight = dq_weight;
    a.dk_weight = dk_weight;
    a.part = (float *)workspace;
    // workgroups for q and for k, by their waves' passes
    const int at_once = 64 >> a.log_lanes;
    a.row_group = std::max(1, at_once / p.heads);
    a.k_row_group = std::max(1, at_once / p.kv_heads);
    const int64_t q_items = (p.rows + a.row_group - 1) / a.row_group, k_items = (p.rows + a.k_row_group - 1) / a.k_row_group;
    const int64_t q_work = q_items * ((p.heads + at_once - 1) / at_once), k_work = k_items * ((p.kv_heads + at_once - 1) / at_once);
    const int64_t q_most = std::max<int64_t>(1, (q_items + 3) / 4), k_most = std::max<int64_t>(1, (k_items + 3) / 4);
    a.q_blocks = (int)std::min(q_most, std::max<int64_t>(1, std::min<int64_t>(kRotateGradBlocks - 1, kRotateGradBlocks * q_work / std::max<int64_t>(1, q_work + k_work))));
    a.blocks = a.q_blocks + (int)std::min<int64_t>(k_most, kRotateGradBlocks - a.q_blocks);
    GBT_HIP(ctx, gbt_launch_norm_rotate_grad(ctx->stream, a, p.dtype));
    return GBT_OK;
}

// --------------------------------------------------- orthogonalised updates --
namespace {

constexpr int64_t kMostMatrices = 1 << 16;
constexpr int64_t kGroupBytes = (int64_t)2 << 30;   // of workspace that matrices taken together may need, where one alone does not need more

const char *matrices_fault(const gbt_matrix *m, int64_t n, int32_t *code) {
    *code = GBT_EINVAL;
    if (n < 0 || (n > 0 && !m)) return "n_matrices < 0 or matrices is NULL";
    *code = GBT_EUNSUPPORTED;
    if (n > kMostMatrices) return "more than 65536 matrices";
    for (int64_t i = 0; i < n; ++i) {
        *code = GBT_EUNSUPPORTED;
        if (!known_type(m[i].dtype)) return "a matrix's dtype is none of GBT_F32, GBT_BF16, GBT_F16";
        if (std::max(m[i].rows, m[i].cols) > (1 << 20) || std::min(m[i].rows, m[i].cols) > (1 << 15)) return "a matrix of more than 2^20 x 2^15";
        *code = GBT_EINVAL;
        if (m[i].rows < 0 || m[i].cols < 0) return "a matrix's rows or cols < 0";
        if (!isfinite(m[i].scale)) return "a matrix's scale is not finite";
        if (m[i].rows > 0 && m[i].cols > 0 && (!m[i].src || !m[i].dst || (((uintptr_t)m[i].src | (uintptr_t)m[i].dst) & (uintptr_t)(size_of(m[i].dtype) - 1))))
            return "a matrix's src or dst is NULL or not aligned";
    }
    return nullptr;
}

// Kinds of matrices, which are worked on apart: small or not, and by how many steps are taken on A = X X^T alone before X is multiplied and A taken anew.
//
// An error of A grows by the square of the singular values' factor with each such step where singular values are small, and makes a relative one of the
// result there.  In large matrices sums leave more than that, and rounding to sixteen bits hides all but its share.  (Five steps, averaged gradients; float32, one step at a
// time, two, and products of 32 bits in torch: 64 x 64 6.2e-7, 1.8e-6, 1.0e-6 off; 400 x 400 1.6e-6, 2.6e-6, 2.0e-6; 700 x 2400 1.7e-6, 2.2e-6, 2.2e-6; 900 x 900 2.1e-6,
// 2.2e-6, 2.7e-6; 4096 x 4096 4.0e-6, 3.4e-6, 8.4e-6.  float16, the share of elements that are not the rounded 64-bit ones, two steps, three, and 32-bit products rounded: 64 x 64
// 1.0%, 3.2%, 0.6%; 128 x 128 1.1%, 3.0%, 0.7%; 200 x 1500 1.0%, 1.5%, 0.6%; 512 x 2048 1.4%, 0.8%, 1.0%.  Two in place of one: 4096 x 4096, 4096 x 8192 and two of
// 1024 x 4096 10.5 in place of 11.4 ms.  Three for large matrices of sixteen bits would take 26 of 512 x 512 to 512 x 2048 from 917 us to 845, but as a kind of their own
// beside small ones most lists of both to a half more: 643 x 2467 and four smaller shapes, 20 matrices, 949 in place of 720.)
enum OrthoKind { kSmallOne, kSmallTwo, kOne, kTwo };
OrthoKind kind_of(const gbt_matrix &m) {
    const bool wide = m.dtype == GBT_F32;
    const int64_t p = std::min(m.rows, m.cols), w = std::max(m.rows, m.cols);
    if (p <= kOrthoSmallP && w <= kOrthoSmallW) return wide ? kSmallOne : kSmallTwo;
    return wide && p < 768 ? kOne : kTwo;
}
bool small_kind(OrthoKind kind) { return kind <= kSmallTwo; }
// For singular values' factors up to `factor`: an error may grow by 2^4.
int steps_together(double factor, OrthoKind kind) { return kind == kSmallOne || kind == kOne || factor > 4.0 ? 1 : 2; }

// The power of two that a matrix with singular values up to `most`, and so with no larger elements, is held times; `least`: as if most were at least 2^least.
float scale_for(double most, int least) { return most <= ldexp(1.0, least) ? ldexpf(kScaleUp, -least) : (float)exp2(15.0 - ceil(log2(most))); }

// The matrices with elements in the order that they are worked on in: by kind, and of each kind those with the most to do first.
struct OrthoOrder {
    int32_t *at;
    int64_t count = 0;
    OrthoOrder(const gbt_matrix *m, int64_t n) : at(new (std::nothrow) int32_t[(size_t)std::max<int64_t>(1, n)]) {
        if (!at) return;
        for (int64_t i = 0; i < n; ++i)
            if (m[i].rows > 0 && m[i].cols > 0) at[count++] = (int32_t)i;
        std::sort(at, at + count, [m](int32_t x, int32_t y) {
            if (kind_of(m[x]) != kind_of(m[y])) return kind_of(m[x]) < kind_of(m[y]);
            const int64_t of_x = m[x].rows * m[x].cols * std::min(m[x].rows, m[x].cols), of_y = m[y].rows * m[y].cols * std::min(m[y].rows, m[y].cols);
            return of_x != of_y ? of_x > of_y : x < y;
        });
    }
    ~OrthoOrder() { delete[] at; }
    OrthoOrder(const OrthoOrder &) = delete;
    OrthoOrder &operator=(const OrthoOrder &) = delete;
};
// Does a result lie over another matrix's memory, or over its own source but for the same place?  -1: no host memory to find out.
int results_overlap(const gbt_matrix *m, const OrthoOrder &order) {
    struct Span {
        uintptr_t begin, end;
        bool written;
    };
    Span *span = new (std::nothrow) Span[(size_t)std::max<int64_t>(1, 2 * order.count)];
    if (!span) return -1;
    int64_t n = 0;
    for (int64_t i = 0; i < order.count; ++i) {
        const gbt_matrix &x = m[order.at[i]];
        const uintptr_t bytes = (uintptr_t)(x.rows * x.cols * size_of(x.dtype)), dst = (uintptr_t)x.dst, src = (uintptr_t)x.src;
        span[n++] = Span{dst, dst + bytes, true};
        if (src != dst) span[n++] = Span{src, src + bytes, false};
    }
    std::sort(span, span + n, [](const Span &x, const Span &y) { return x.begin < y.begin; });
    uintptr_t end = 0, end_written = 0;   // of the spans so far, of the written ones
    int overlap = 0;
    for (int64_t i = 0; i < n; ++i) {
        overlap |= span[i].begin < (span[i].written ? end : end_written);
        end = std::max(end, span[i].end);
        if (span[i].written) end_written = std::max(end_written, span[i].end);
    }
    delete[] span;
    return overlap;
}
int64_t tiles_of(int64_t side) { return (side + kOrthoTile - 1) / kOrthoTile; }

enum OrthoTiles { kTilesGram, kTilesSym, kTilesFull };   // of X X^T; of products of symmetric matrices; of F X

// The tiles of the matrices order.at[first .. first + count) (of symmetric results the upper halves) in the order of a launch's workgroups; their number,
// with gaps.  Into `out` where that is not NULL.
//
// Workgroups go to the eight XCDs in turn, and tiles of one matrix share what they read.  So a matrix goes to one XCD, or, where that would leave others
// idle, in parts of at least eight tiles and a hundred-and-twenty-eighth of all the work, each to the XCD with the least so far, the largest matrices first.
// Of a matrix, eight rows of tiles at a time, column by column.
int64_t lay_tiles(const gbt_matrix *matrices, const OrthoOrder &order, int64_t first, int64_t count, OrthoTiles kind, OrthoTile *out) {
    const bool full = kind == kTilesFull;
    int64_t down, across, tiles, depth;
    auto look = [&](int64_t i) {
        const gbt_matrix &m = matrices[order.at[first + i]];
        const int64_t p = tiles_of(std::min(m.rows, m.cols)), w = tiles_of(std::max(m.rows, m.cols));
        down = p, across = full ? w : p, depth = kind == kTilesGram ? w : p;
        tiles = full ? p * w : p * (p + 1) / 2;
    };
    double all = 0.0, load[8] = {};
    int64_t used[8] = {};
    for (int64_t i = 0; i < count; ++i) {
        look(i);
        all += (double)tiles * (double)depth;
    }
    for (int64_t i = 0; i < count; ++i) {
        look(i);
        const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(8, tiles / 8), (int64_t)ceil(128.0 * (double)tiles * (double)depth / all)));
        int64_t next = 0, part = -1;
        int xcd = 0;
        for (int64_t band = 0; band < down; band += 8)
            for (int64_t j = full ? 0 : band; j < across; ++j)
                for (int64_t r = band; r < std::min(band + 8, full ? down : std::min(down, j + 1)); ++r, ++next) {
                    if (next * parts / tiles != part) {
                        part = next * parts / tiles;
                        xcd = (int)(std::min_element(load, load + 8) - load);
                    }
                    if (out) out[used[xcd] * 8 + xcd] = OrthoTile{(int32_t)i, (int16_t)r, (int16_t)j};
                    ++used[xcd];
                    load[xcd] += (double)depth;
                }
    }
    return *std::max_element(used, used + 8) * 8;
}

// Matrices of one kind that are worked on together, and what they need.
struct OrthoGroup {
    int64_t first, count;   // of the order
    OrthoKind kind;
    int64_t pieces, fill_tiles, tiles[3];   // tiles: by OrthoTiles
    size_t bytes;
};
// The next group, from *at on; false: there is none.  Into `list` where that is not NULL, its matrices as the kernels take them.
bool next_group(const gbt_matrix *matrices, const OrthoOrder &order, int64_t *at, OrthoGroup *g, OrthoMatrix *list) {
    *g = OrthoGroup{};
    g->first = *at;
    int64_t used = 0;
    for (; *at < order.count; ++*at) {
        const gbt_matrix &m = matrices[order.at[*at]];
        OrthoMatrix o;
        memset(&o, 0, sizeof o);
        o.tall = m.rows > m.cols;
        o.p = (int32_t)std::min(m.rows, m.cols);
        o.w = (int32_t)std::max(m.rows, m.cols);
        const int64_t down = tiles_of(o.p), across = tiles_of(o.w), fill = 2 * down * across;
        o.pp = (int32_t)down * kOrthoTile;
        o.ww = (int32_t)across * kOrthoTile;
        const int64_t of_x = (int64_t)o.pp * o.ww * 4, of_a = (int64_t)o.pp * o.pp * 4, need = 3 * of_x + 5 * of_a;
        const OrthoKind kind = kind_of(m);
        if (g->count > 0 && (kind != g->kind || (!small_kind(kind) && (used + need > kGroupBytes || g->fill_tiles + fill > kMostWorkgroups)))) break;
        o.src = m.src;
        o.dst = m.dst;
        o.cols = m.cols;
        o.dtype = m.dtype;
        o.scale = m.scale;
        o.pieces = (int32_t)((m.rows * m.cols + kOrthoPiece - 1) / kOrthoPiece);
        o.piece_begin = g->pieces;
        o.fill_begin = g->fill_tiles;
        o.x = used, o.xt[0] = used + of_x, o.xt[1] = used + 2 * of_x;
        o.gram = used + 3 * of_x, o.factor[0] = o.gram + of_a, o.factor[1] = o.gram + 2 * of_a, o.between = o.gram + 3 * of_a, o.total = o.gram + 4 * of_a;
        if (list) list[*at] = o;
        g->kind = kind;
        ++g->count;
        if (small_kind(kind)) continue;
        used += need;
        g->pieces += o.pieces;
        g->fill_tiles += fill;
        g->bytes = (size_t)used + gbt_align((size_t)g->pieces * sizeof(double));
    }
    if (g->count == 0) return false;
    if (small_kind(g->kind)) return true;
    for (int kind = 0; kind < 3; ++kind) g->tiles[kind] = lay_tiles(matrices, order, g->first, g->count, (OrthoTiles)kind, nullptr);
    return true;
}
// The list: the matrices in their order, then each group's tiles.
int64_t list_bytes_of(const gbt_matrix *matrices, const OrthoOrder &order) {
    int64_t at = 0, tiles = 0;
    OrthoGroup g;
    while (next_group(matrices, order, &at, &g, nullptr)) tiles += g.tiles[0] + g.tiles[1] + g.tiles[2];
    return std::max<int64_t>(16, order.count * (int64_t)sizeof(OrthoMatrix) + tiles * (int64_t)sizeof(OrthoTile));
}
}  // namespace

extern "C" size_t gbt_matrix_list_bytes(const gbt_matrix *matrices, int64_t n_matrices) {
    int32_t code;
    if (matrices_fault(matrices, n_matrices, &code)) return 0;
    const OrthoOrder order(matrices, n_matrices);
    return order.at ? (size_t)list_bytes_of(matrices, order) : 0;
}

extern "C" int32_t gbt_matrix_list(gbt_ctx *ctx, const gbt_matrix *matrices, int64_t n_matrices, void *list_out, size_t list_bytes) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, list_out, GBT_EINVAL, "NULL argument");
    GBT_REQUIRE(ctx, ((uintptr_t)list_out & 15u) == 0, GBT_EINVAL, "list_out is not 16-byte aligned");
    int32_t code;
    const char *fault = matrices_fault(matrices, n_matrices, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    const OrthoOrder order(matrices, n_matrices);
    GBT_REQUIRE(ctx, order.at, GBT_ENOMEM, "no host memory for the list");
    const int overlap = results_overlap(matrices, order);
    GBT_REQUIRE(ctx, overlap >= 0, GBT_ENOMEM, "no host memory for the list");
    GBT_REQUIRE(ctx, overlap == 0, GBT_EINVAL, "a matrix's dst overlaps another matrix, or its own src in part");
    const size_t need = (size_t)list_bytes_of(matrices, order);
    GBT_REQUIRE(ctx, list_bytes >= need, GBT_ENOMEM, "list of %zu bytes, %zu needed", list_bytes, need);
    char *table = new (std::nothrow) char[need];
    GBT_REQUIRE(ctx, table, GBT_ENOMEM, "no host memory for the list");
    memset(table, 0xff, need);   // tiles of no matrix
    int64_t at = 0;
    OrthoTile *tiles = (OrthoTile *)(table + order.count * sizeof(OrthoMatrix));
    OrthoGroup g;
    while (next_group(matrices, order, &at, &g, (OrthoMatrix *)table)) {
        for (int kind = 0; kind < 3; ++kind) {
            if (g.tiles[kind]) lay_tiles(matrices, order, g.first, g.count, (OrthoTiles)kind, tiles);
            tiles += g.tiles[kind];
        }
    }
    // in pieces that the staging takes
    int32_t st = GBT_OK;
    for (size_t i = 0; i < need && st == GBT_OK; i += 1 << 20) st = gbt_upload(ctx, table + i, std::min<size_t>(1 << 20, need - i), (char *)list_out + i);
    delete[] table;
    return st;
}

extern "C" size_t gbt_orthogonalise_workspace_bytes(const gbt_matrix *matrices, int64_t n_matrices) {
    int32_t code;
    if (matrices_fault(matrices, n_matrices, &code)) return 0;
    size_t most = 0;
    const OrthoOrder order(matrices, n_matrices);
    if (!order.at) return 0;
    int64_t at = 0;
    OrthoGroup g;
    while (next_group(matrices, order, &at, &g, nullptr)) most = std::max(most, g.bytes);
    return most;
}

extern "C" int32_t gbt_orthogonalise(gbt_ctx *ctx, const void *list, const gbt_matrix *matrices, int64_t n_matrices, int32_t steps, float a, float b, float c,
                                     void *workspace, size_t workspace_bytes) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, list, GBT_EINVAL, "NULL argument");
    GBT_REQUIRE(ctx, ((uintptr_t)list & 15u) == 0, GBT_EINVAL, "list is not 16-byte aligned");
    int32_t code;
    const char *fault = matrices_fault(matrices, n_matrices, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    GBT_REQUIRE(ctx, steps >= 1 && steps <= 32, GBT_EINVAL, "steps outside 1..32");
    // how large singular values can become, and the factor that they are multiplied by: what is kept in sixteen bits has to hold both, and is scaled by them
    GBT_REQUIRE(ctx, isfinite(a) && isfinite(b) && isfinite(c), GBT_EINVAL, "a coefficient is not finite");
    OrthoScales up;
    double most = 1.0, factor = 0.0;
    up.x[0] = scale_for(most, -20);
    for (int s = 0; s < steps; ++s) {
        double next = 0.0, of_step = 0.0;
        for (int i = 0; i <= 4096; ++i) {
            const double x = most * i / 4096.0, f = fabs((double)a + (double)b * x * x + (double)c * x * x * x * x);
            of_step = std::max(of_step, f);
            next = std::max(next, x * f);
        }
        most = next;
        factor = std::max(factor, of_step);
        up.x[s + 1] = scale_for(most, -20);
        up.factor[s] = scale_for(of_step, -10);
        GBT_REQUIRE(ctx, most <= 4.0 && factor <= 64.0, GBT_EINVAL, "coefficients under which singular values pass 4 or their factors 64");
    }
    const size_t need = gbt_orthogonalise_workspace_bytes(matrices, n_matrices);
    GBT_REQUIRE(ctx, workspace || need == 0, GBT_EINVAL, "workspace is NULL");
    GBT_REQUIRE(ctx, workspace_bytes >= need, GBT_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    GBT_REQUIRE(ctx, ((uintptr_t)workspace & 255u) == 0 || need == 0, GBT_EINVAL, "workspace is not 256-byte aligned");
    const OrthoOrder order(matrices, n_matrices);
    GBT_REQUIRE(ctx, order.at, GBT_ENOMEM, "no host memory for the order of the matrices");
    int64_t at = 0;
    const OrthoTile *tiles = (const OrthoTile *)((const char *)list + order.count * sizeof(OrthoMatrix));
    OrthoGroup g;
    for (; next_group(matrices, order, &at, &g, nullptr); tiles += g.tiles[0] + g.tiles[1] + g.tiles[2]) {
        OrthoArgs o;
        memset(&o, 0, sizeof o);
        o.list = (const OrthoMatrix *)list + g.first;
        o.count = (int)g.count;
        o.workspace = (char *)workspace;
        o.squares = (double *)((char *)workspace + g.bytes - gbt_align((size_t)g.pieces * sizeof(double)));
        o.a = a;
        o.b = b;
        o.c = c;
        const int together = steps_together(factor, g.kind);
        o.up_x = up.x[0];
        if (small_kind(g.kind)) {
            OrthoSmallScales of;
            memset(&of, 0, sizeof of);
            of.x = up.x[0];
            for (int t = 0; t < steps; ++t) {
                of.step[t] = OrthoSmallScales::Step{{1.0f / up.gram(t), kScaleDown, up.after(t), up.after(t)}, up.gram(t), up.factor[t] / up.gram(t),
                                                    up.apply(t, std::min(t + together, steps), steps), 0.0f};
            }
            GBT_HIP(ctx, gbt_launch_ortho_small(ctx->stream, o, of, steps, together));
            continue;
        }
        GBT_HIP(ctx, gbt_launch_ortho_begin(ctx->stream, o, g.pieces, g.fill_tiles));
        auto product = [&](OrthoProduct of) {
            const OrthoTiles kind = of == kOrthoGram ? kTilesGram : of == kOrthoApply ? kTilesFull : kTilesSym;
            o.tiles = tiles + (kind > 0 ? g.tiles[0] : 0) + (kind > 1 ? g.tiles[1] : 0);
            o.count_tiles = g.tiles[kind];
            return gbt_launch_ortho_product(ctx->stream, o, of, ctx->num_cu);
        };
        for (int s = 0; s < steps; s += together) {
            const int n = std::min(together, steps - s);
            o.less = kScaleDown;
            GBT_HIP(ctx, product(kOrthoGram));
            for (o.step = 0;; ++o.step) {
                const int t = s + o.step;
                o.up_gram = up.gram(t);
                o.up_factor = up.factor[t];
                o.less = 1.0f / o.up_gram;
                GBT_HIP(ctx, product(kOrthoFactor));
                if (o.step == n - 1) break;
                o.less = up.after(t);   // F A, then A of the next step
                GBT_HIP(ctx, product(kOrthoBetween));
                GBT_HIP(ctx, product(kOrthoNext));
            }
            o.less = kScaleDown;
            if (n == 2) GBT_HIP(ctx, product(kOrthoTotal));
            o.last = s + n == steps;
            o.less = up.apply(s, s + n, steps);
            GBT_HIP(ctx, product(kOrthoApply));
            o.xt ^= 1;
        }
    }
    return GBT_OK;
}
