// The C ABI of the operators for rows with a history (see include/gbt.h): checks of arguments, workspaces, launches.
#include "attention.h"

#include <string.h>

#include <new>

namespace {

// Workgroups that a call with few query rows is cut into where its keys allow, were all sequences the longest: two are on a compute unit at a time, and
// most sequences are shorter.  A row's pieces are joined by 256 lanes at most.  (us for 512, 2048, 4096: 64 stores of 30 to 3000 rows, 8 key heads of 64
// elements, 58, 51, 51; 128 102, 93, 89; 128 of 30 to 10000 320, 284, 253; 200 of 3000 246, 246, 223; 16 of 2000 to 30000, 4 of 128, 134, 115, 116; but 1000
// of 30 to 1500, 1 of 64 for 8 heads 49, 55, 55.)
constexpr int64_t kFewWorkgroups = 4096, kFewPieces = 256;
// Shorter pieces cost more by their beginnings and ends than they gain by being many: 32 stores of 1000 rows, 8 heads of 128 elements, at least 256, 512,
// 1024 rows a piece: 32, 29, 25 us; 4 of 2000, 2 heads of 64: 9.3, 10.3, 12.3; 4 of 500: 9.2, 7.0, 7.0.
constexpr int64_t kFewLeast = 1024;

struct FewPlan {
    int64_t columns;         // (query, head of the group) pairs of a key head
    int pieces, piece_len;   // of the key axis
};
bool takes_few(const gbt_attention_params &p) { return (int64_t)(p.heads / p.kv_heads) * p.max_q <= kAttnFewRows; }
FewPlan few_plan(const gbt_attention_params &p) {
    FewPlan f;
    f.columns = (int64_t)(p.heads / p.kv_heads) * p.max_q;
    const int64_t base = std::max<int64_t>(1, (int64_t)p.kv_heads * p.n_seq);
    const int64_t want = std::max<int64_t>(1, kFewWorkgroups / base);
    const int64_t len = std::max<int64_t>(1, std::max((p.max_k + want - 1) / want, (p.max_k + kFewPieces - 1) / kFewPieces));
    f.piece_len = (int)((std::max(len, kFewLeast) + 127) / 128 * 128);
    f.pieces = (int)std::max<int64_t>(1, (p.max_k + f.piece_len - 1) / f.piece_len);
    return f;
}
int64_t blocks_of(int64_t rows) { return (rows + kAttnQueries - 1) / kAttnQueries; }

// What is wrong with the parameters, or NULL.  *code: GBT_EINVAL or GBT_EUNSUPPORTED.
const char *params_fault(const gbt_attention_params &p, int32_t *code) {
    *code = GBT_EUNSUPPORTED;
    if (p.dtype != GBT_BF16 && p.dtype != GBT_F16) return "dtype is neither GBT_BF16 nor GBT_F16";
    if (p.head_dim < 8 || p.head_dim > GBT_MAX_HEAD_DIM || p.head_dim % 8) return "head_dim is no multiple of 8 in 8..128";
    if (p.n_buckets > GBT_MAX_BUCKETS) return "n_buckets > 128";
    *code = GBT_EINVAL;
    if (p.heads < 1 || p.kv_heads < 1 || p.heads % p.kv_heads || p.heads > (1 << 16)) return "heads is no multiple of kv_heads, or out of range";
    if (p.n_seq < 0 || p.max_q < 0 || p.max_k < 0 || p.max_q > (1 << 29) || p.max_k > (1 << 29)) return "n_seq, max_q or max_k out of range";
    if (p.q_rows < 0 || p.k_rows < 0 || p.q_rows > ((int64_t)1 << 40) || p.k_rows > ((int64_t)1 << 40)) return "q_rows or k_rows out of range";
    if (p.n_buckets < 0) return "n_buckets < 0";
    if (!(p.scale >= 1e-6f && p.scale <= 1e6f)) return "scale outside 1e-6..1e6";
    if (p.n_seq > 0 && !p.q_ptr && p.q_rows / p.n_seq < p.max_q) return "q_rows < n_seq * max_q without q_ptr";
    if (p.n_seq > 0 && !p.k_ptr && p.k_rows / p.n_seq < p.max_k) return "k_rows < n_seq * max_k without k_ptr";
    if (p.n_buckets > 0) {
        if (!p.bias) return "bias is NULL";
        if (((uintptr_t)p.bias & 3u) != 0) return "bias is not aligned";
        if (p.n_buckets > 1 && !p.cuts) return "cuts is NULL";
        for (int i = 1; i < p.n_buckets - 1; ++i)
            if (p.cuts[i] <= p.cuts[i - 1]) return "cuts do not increase";
    }
    const int64_t limit = ((int64_t)1 << 23) - 1024;   // workgroups of a launch, of up to 512 threads, of which there can be 2^32
    if (std::max({blocks_of(p.max_q) * p.heads, blocks_of(p.max_k) * p.kv_heads, takes_few(p) ? (int64_t)p.max_q * p.heads : 0}) >
        limit / std::max(1, p.n_seq))
        return "too many sequences for max_q or max_k";
    return nullptr;
}

bool view_ok(const gbt_heads *h) {
    return h && ((uintptr_t)h->data & 15u) == 0 && h->row_stride >= 0 && h->head_stride >= 0 && h->row_stride % 8 == 0 && h->head_stride % 8 == 0 &&
           h->row_stride < ((int64_t)1 << 24) && h->head_stride < ((int64_t)1 << 40);
}
// No two of its heads' rows share elements: what is written to.
bool apart(const gbt_heads &h, int64_t rows, int64_t heads, int64_t dim) {
    int64_t near = h.row_stride, n_near = rows, far = h.head_stride, n_far = heads;
    if (n_far <= 1 || (n_near > 1 && near > far)) {
        std::swap(near, far);
        std::swap(n_near, n_far);
    }
    if (n_near <= 1) return n_far <= 1 || far >= dim;
    return near >= dim && (n_far <= 1 || (far - dim) / near >= n_near - 1);
}
AttnView view(const gbt_heads *h) { return AttnView{(char *)h->data, h->row_stride, h->head_stride}; }

#define GBT_VIEW(ctx, h, rows)                                                                                                        \
    GBT_REQUIRE(ctx, view_ok(h), GBT_EINVAL, #h ": NULL, not 16-byte aligned, or strides that are negative, no multiples of 8 or (rows) 2^24 and more");    \
    GBT_REQUIRE(ctx, (h)->data || (rows) == 0, GBT_EINVAL, #h ": data is NULL")
#define GBT_VIEW_OUT(ctx, h, rows, heads)                                                                                             \
    GBT_VIEW(ctx, h, rows);                                                                                                           \
    GBT_REQUIRE(ctx, apart(*(h), rows, heads, p.head_dim), GBT_EINVAL, #h ": rows or heads overlap")

void fill(AttnArgs &a, AttnCuts &c, const gbt_attention_params &p) {
    memset(&a, 0, sizeof a);
    a.q_ptr = p.q_ptr;
    a.k_ptr = p.k_ptr;
    a.k_len = p.k_len;
    a.q_rows = p.q_rows;
    a.k_rows = p.k_rows;
    a.n_seq = p.n_seq;
    a.heads = p.heads;
    a.kv_heads = p.kv_heads;
    a.group = p.heads / p.kv_heads;
    a.dim = p.head_dim;
    a.max_q = p.max_q;
    a.max_k = p.max_k;
    a.causal = p.causal != 0;
    a.n_buckets = p.n_buckets;
    a.scale = p.scale;
    a.scale2 = p.scale * GBT_LOG2E;
    a.bias = p.bias;
    for (int i = 0; i < kAttnBuckets - 1; ++i) c.at[i] = i < p.n_buckets - 1 ? p.cuts[i] : INT32_MAX;
}

}  // namespace

extern "C" size_t gbt_attention_workspace_bytes(const gbt_attention_params *params) {
    int32_t code;
    if (!params || params_fault(*params, &code)) return 0;
    if (!takes_few(*params)) return 0;
    const FewPlan f = few_plan(*params);
    if (f.pieces == 1) return 0;
    return (size_t)params->n_seq * params->kv_heads * f.columns * f.pieces * (params->head_dim + 2) * sizeof(float);
}

extern "C" int32_t gbt_attention(gbt_ctx *ctx, const gbt_attention_params *params, const gbt_heads *q, const gbt_heads *k, const gbt_heads *v,
                                 const gbt_heads *out, float *lse_out, void *rest_out, void *workspace, size_t workspace_bytes) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, params, GBT_EINVAL, "NULL argument");
    const gbt_attention_params &p = *params;
    int32_t code;
    const char *fault = params_fault(p, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    GBT_VIEW(ctx, q, p.q_rows);
    GBT_VIEW(ctx, k, p.k_rows);
    GBT_VIEW(ctx, v, p.k_rows);
    GBT_VIEW_OUT(ctx, out, p.q_rows, p.heads);
    GBT_REQUIRE(ctx, ((uintptr_t)rest_out & 15u) == 0 && ((uintptr_t)lse_out & 3u) == 0, GBT_EINVAL, "rest_out or lse_out is not aligned");
    const size_t need = gbt_attention_workspace_bytes(params);
    GBT_REQUIRE(ctx, workspace || need == 0, GBT_EINVAL, "workspace is NULL");
    GBT_REQUIRE(ctx, workspace_bytes >= need, GBT_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    GBT_REQUIRE(ctx, ((uintptr_t)workspace & 15u) == 0 || need == 0, GBT_EINVAL, "workspace is not 16-byte aligned");
    if (p.q_rows == 0) return GBT_OK;
    AttnArgs a;
    AttnCuts c;
    fill(a, c, p);
    a.q = view(q);
    a.k = view(k);
    a.v = view(v);
    a.out = view(out);
    a.lse = lse_out;
    a.rest = (char *)rest_out;
    if (p.n_seq > 0 && p.max_q > 0 && takes_few(p)) {
        const FewPlan f = few_plan(p);
        a.pieces = f.pieces;
        a.piece_len = f.piece_len;
        a.part = (float *)workspace;
        GBT_HIP(ctx, gbt_launch_attention_few(ctx->stream, a, c, p.dtype));
    } else {
        GBT_HIP(ctx, gbt_launch_attention(ctx->stream, a, c, p.dtype));
    }
    return GBT_OK;
}

namespace {

// Workgroups that a block of keys is shared by: its heads' queries one after the other are all the work there is, so where blocks are few they
// go to several workgroups, as many heads each first (the tiles of queries are then not cut), and never less than four tiles each.
// (Two histories of 4096, groups of four heads, kernel and join: one workgroup a block 666 us, two 491, three, of one or two heads, 586, four 525.)
constexpr int64_t kKeyWorkgroups = 768;
struct KeyParts {
    int heads, queries;
};
KeyParts key_parts(const gbt_attention_params &p) {
    const int group = p.heads / p.kv_heads;
    const int64_t base = std::max<int64_t>(1, blocks_of(p.max_k) * p.kv_heads * p.n_seq), want = std::max<int64_t>(1, kKeyWorkgroups / base);
    KeyParts k;
    k.heads = (int)std::min<int64_t>(want, group);
    while (group % k.heads) --k.heads;
    k.queries = (int)std::min<int64_t>(std::max<int64_t>(1, want / k.heads), std::max(1, p.max_q / 256));
    return k;
}
int64_t part_rows(const gbt_attention_params &p) { return std::min<int64_t>(p.k_rows, (int64_t)p.n_seq * p.max_k); }
struct BackwardLayout {
    size_t row_minus, strips, part, bytes;
};
BackwardLayout backward_layout(const gbt_attention_params &p) {
    const KeyParts k = key_parts(p);
    const size_t row = gbt_align((size_t)p.heads * p.q_rows * sizeof(float));
    BackwardLayout l;
    l.row_minus = row;
    l.strips = l.row_minus + row;
    l.part = l.strips + gbt_align((size_t)p.heads * p.n_seq * blocks_of(p.max_k) * k.queries * p.n_buckets * sizeof(float));
    const int parts = k.heads * k.queries;
    l.bytes = l.part + (parts > 1 ? gbt_align((size_t)parts * 2 * part_rows(p) * p.kv_heads * p.head_dim * sizeof(float)) : 0);
    return l;
}
}  // namespace

extern "C" size_t gbt_attention_backward_workspace_bytes(const gbt_attention_params *params) {
    int32_t code;
    if (!params || params_fault(*params, &code)) return 0;
    return backward_layout(*params).bytes;
}

extern "C" int32_t gbt_attention_backward(gbt_ctx *ctx, const gbt_attention_params *params, const gbt_heads *dout, const gbt_heads *q, const gbt_heads *k,
                                          const gbt_heads *v, const gbt_heads *out, const float *lse, const void *rest, const gbt_heads *dq,
                                          const gbt_heads *dk, const gbt_heads *dv, float *dbias_out, void *workspace, size_t workspace_bytes) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, params, GBT_EINVAL, "NULL argument");
    const gbt_attention_params &p = *params;
    int32_t code;
    const char *fault = params_fault(p, &code);
    GBT_REQUIRE(ctx, !fault, code, "%s", fault);
    GBT_VIEW(ctx, dout, p.q_rows);
    GBT_VIEW(ctx, q, p.q_rows);
    GBT_VIEW(ctx, k, p.k_rows);
    GBT_VIEW(ctx, v, p.k_rows);
    GBT_VIEW(ctx, out, p.q_rows);
    GBT_VIEW_OUT(ctx, dq, p.q_rows, p.heads);
    GBT_VIEW_OUT(ctx, dk, p.k_rows, p.kv_heads);
    GBT_VIEW_OUT(ctx, dv, p.k_rows, p.kv_heads);
    GBT_REQUIRE(ctx, lse || p.q_rows == 0, GBT_EINVAL, "lse is NULL");
    GBT_REQUIRE(ctx, dbias_out || p.n_buckets == 0, GBT_EINVAL, "dbias_out is NULL");
    GBT_REQUIRE(ctx, ((uintptr_t)rest & 15u) == 0 && (((uintptr_t)lse | (uintptr_t)dbias_out) & 3u) == 0, GBT_EINVAL,
                "rest, lse or dbias_out is not aligned");
    const BackwardLayout l = backward_layout(p);
    const size_t need = l.bytes;
    GBT_REQUIRE(ctx, workspace || need == 0, GBT_EINVAL, "workspace is NULL");
    GBT_REQUIRE(ctx, workspace_bytes >= need, GBT_ENOMEM, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    GBT_REQUIRE(ctx, ((uintptr_t)workspace & 15u) == 0, GBT_EINVAL, "workspace is not 16-byte aligned");
    AttnArgs a;
    AttnCuts c;
    fill(a, c, p);
    a.dout = view(dout);
    a.q = view(q);
    a.k = view(k);
    a.v = view(v);
    a.out = view(out);
    a.dq = view(dq);
    a.dk = view(dk);
    a.dv = view(dv);
    a.lse = (float *)lse;
    a.rest = (char *)rest;
    a.row_less = (float *)workspace;
    a.row_minus = (float *)((char *)workspace + l.row_minus);
    a.strips = (float *)((char *)workspace + l.strips);
    a.part = (float *)((char *)workspace + l.part);
    const KeyParts k_parts = key_parts(p);
    a.head_parts = k_parts.heads;
    a.q_parts = k_parts.queries;
    a.part_rows = part_rows(p);
    a.dbias = dbias_out;
    GBT_HIP(ctx, gbt_launch_attention_grad(ctx->stream, a, c, p.dtype));
    return GBT_OK;
}

// ------------------------------------------------------------------ clipping --
namespace {

constexpr size_t kListBytes = 4u << 20;

// Elements of a piece: some sixteen pieces for each of the kernels' workgroups where there are so many elements, and never so few that a
// workgroup's own launch outweighs them.  A multiple of 8, so that a tensor's pieces are all aligned as its first one is.
int64_t piece_elements(const gbt_gradient *g, int64_t n) {
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) total += g[i].n;
    const int64_t each = total / 32768;
    return std::min<int64_t>(std::max<int64_t>((each + 1023) / 1024 * 1024, 2048), (int64_t)1 << 30);
}
bool gradients_ok(const gbt_gradient *g, int64_t n) {
    if (n < 0 || (n > 0 && !g)) return false;
    for (int64_t i = 0; i < n; ++i) {
        if (g[i].dtype != GBT_F32 && g[i].dtype != GBT_BF16 && g[i].dtype != GBT_F16) return false;
        if (g[i].n < 0 || g[i].n > ((int64_t)1 << 44)) return false;
        const uintptr_t mask = g[i].dtype == GBT_F32 ? 3u : 1u;
        if (g[i].n > 0 && (!g[i].src || !g[i].dst || (((uintptr_t)g[i].src | (uintptr_t)g[i].dst) & mask))) return false;
    }
    return true;
}
int64_t count_pieces(const gbt_gradient *g, int64_t n, int64_t each) {
    int64_t pieces = 0;
    for (int64_t i = 0; i < n; ++i) pieces += (g[i].n + each - 1) / each;
    return pieces;
}

}  // namespace

extern "C" size_t gbt_gradient_list_bytes(const gbt_gradient *gradients, int64_t n_gradients) {
    if (!gradients_ok(gradients, n_gradients)) return 0;
    const size_t bytes = std::max<size_t>(16, (size_t)count_pieces(gradients, n_gradients, piece_elements(gradients, n_gradients)) * sizeof(ClipPiece));
    return bytes <= kListBytes ? bytes : 0;
}

extern "C" int32_t gbt_gradient_list(gbt_ctx *ctx, const gbt_gradient *gradients, int64_t n_gradients, void *list_out, size_t list_bytes,
                                     int32_t *pieces_out) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, list_out && pieces_out, GBT_EINVAL, "NULL argument");
    GBT_REQUIRE(ctx, ((uintptr_t)list_out & 15u) == 0, GBT_EINVAL, "list_out is not 16-byte aligned");
    GBT_REQUIRE(ctx, gradients_ok(gradients, n_gradients), GBT_EINVAL, "a gradient's pointer, size, type or alignment");
    const size_t need = gbt_gradient_list_bytes(gradients, n_gradients);
    GBT_REQUIRE(ctx, need > 0, GBT_EUNSUPPORTED, "a list of more than %zu bytes", kListBytes);
    GBT_REQUIRE(ctx, list_bytes >= need, GBT_ENOMEM, "list of %zu bytes, %zu needed", list_bytes, need);
    const int64_t each = piece_elements(gradients, n_gradients), count = count_pieces(gradients, n_gradients, each);
    ClipPiece *table = new (std::nothrow) ClipPiece[(size_t)std::max<int64_t>(1, count)];
    GBT_REQUIRE(ctx, table, GBT_ENOMEM, "no host memory for the list");
    int64_t at = 0;
    for (int64_t i = 0; i < n_gradients; ++i) {
        const gbt_gradient &g = gradients[i];
        const int64_t size = g.dtype == GBT_F32 ? 4 : 2;
        for (int64_t e = 0; e < g.n; e += each)
            table[at++] = ClipPiece{(const char *)g.src + e * size, (char *)g.dst + e * size, (int32_t)std::min(each, g.n - e), g.dtype};
    }
    const int32_t st = count > 0 ? gbt_upload(ctx, table, (size_t)count * sizeof(ClipPiece), list_out) : GBT_OK;
    delete[] table;
    if (st == GBT_OK) *pieces_out = (int32_t)count;
    return st;
}

extern "C" int32_t gbt_clip_gradients(gbt_ctx *ctx, const void *list, int32_t pieces, double max_norm, float *norm_out, void *workspace,
                                      size_t workspace_bytes) {
    if (!ctx) return GBT_EINVAL;
    GBT_REQUIRE(ctx, list && norm_out && workspace, GBT_EINVAL, "NULL argument");
    GBT_REQUIRE(ctx, pieces >= 0, GBT_EINVAL, "pieces < 0");
    GBT_REQUIRE(ctx, max_norm >= 0.0, GBT_EINVAL, "max_norm is negative or no number");
    GBT_REQUIRE(ctx, (((uintptr_t)list | (uintptr_t)workspace) & 15u) == 0 && ((uintptr_t)norm_out & 3u) == 0, GBT_EINVAL, "list, workspace or norm_out is not aligned");
    GBT_REQUIRE(ctx, workspace_bytes >= 16384, GBT_ENOMEM, "workspace < 16384 bytes");
    GBT_HIP(ctx, gbt_launch_clip(ctx->stream, (const ClipPiece *)list, pieces, max_norm, norm_out, (double *)workspace));
    return GBT_OK;
}
