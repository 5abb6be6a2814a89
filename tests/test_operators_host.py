"""What the operators for histories decide on the host: layouts, workspaces, cuts between buckets of distance (no GPU)."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def b():
    import paper_1806_11248_amd as g
    if not os.path.exists(g.LIB_PATH):
        from paper_1806_11248_amd import build
        build.build()
    g.load()
    return g.binding


def _params(b, **kw):
    cuts = kw.pop("cuts", [-2, 0, 5])
    arr = (C.c_int32 * max(1, len(cuts)))(*cuts)
    p = dict(dtype=1, heads=8, kv_heads=2, head_dim=64, n_seq=3, max_q=100, max_k=100, causal=1, n_buckets=len(cuts) + 1, scale=0.125,
             q_rows=300, k_rows=300, q_ptr=None, k_ptr=None, k_len=None, bias=4096, cuts=C.addressof(arr))
    p.update(kw)
    out = b.AttentionParams(*p.values())
    out.keep = arr
    return out


def test_struct_layouts_match_header(b):
    assert C.sizeof(b.Heads) == 24 and C.sizeof(b.Gradient) == 32
    assert C.sizeof(b.AttentionParams) == 10 * 4 + 2 * 8 + 5 * 8
    header = open(os.path.join(ROOT, "include", "gbt.h")).read()
    body = re.search(r"typedef struct gbt_attention_params \{(.*?)\} gbt_attention_params;", header, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip(" *") for line in re.findall(r"(?:const )?(?:int32_t|int64_t|float) ([^;]*);", body) for n in line.split(",")]
    assert names == [n for n, _ in b.AttentionParams._fields_]


def test_workspaces(b):
    L = b._lib
    fwd, bwd = L.gbt_attention_workspace_bytes, L.gbt_attention_backward_workspace_bytes
    assert fwd(C.byref(_params(b))) == 0                                   # blocks of queries need none
    few = _params(b, max_q=1, q_rows=3, max_k=20_000, k_rows=60_000)
    # pieces of the keys: at most 256 a row, of head_dim + 2 floats for each of 3 sequences and 8 heads
    assert 3 * 8 * 2 * 66 * 4 <= fwd(C.byref(few)) <= 3 * 8 * 256 * 66 * 4
    assert fwd(C.byref(_params(b, max_q=1, q_rows=3, max_k=500, k_rows=1500))) == 0     # one piece, no joining
    # two floats for each head and query row, the bias gradient of every block of keys
    assert bwd(C.byref(_params(b))) >= 2 * 8 * 300 * 4 + 8 * 3 * 4 * 4
    assert bwd(C.byref(_params(b, n_seq=0, q_rows=0, k_rows=0, max_q=0, max_k=0))) >= 0
    assert fwd(None) == 0 and bwd(None) == 0


def test_the_backward_workspace_goes_by_the_rows_in_use(b):
    """Partial sums of the keys' gradients are as many as the sequences can have rows, whatever the size of the store that they lie in."""
    def need(**kw):
        return b._lib.gbt_attention_backward_workspace_bytes(C.byref(_params(b, q_ptr=64, k_ptr=64, k_len=64, causal=0, **kw)))

    for kw in (dict(n_seq=3, heads=8, kv_heads=8, head_dim=128, max_q=1500, max_k=700, q_rows=4500), dict(n_seq=2, heads=16, kv_heads=4, head_dim=128, max_q=512,
               max_k=512, q_rows=1024), dict(n_seq=1, heads=4, kv_heads=1, head_dim=64, max_q=4096, max_k=40, q_rows=4096)):
        rows = kw["n_seq"] * kw["max_k"]
        tight = need(k_rows=rows, **kw)
        two_tensors = 2 * rows * kw["kv_heads"] * kw["head_dim"] * 4
        assert tight > 2 * two_tensors                                       # several parts
        assert need(k_rows=rows // 2, **kw) <= tight                         # fewer rows than n_seq * max_k
        assert need(k_rows=rows + 7, **kw) <= tight + 4096 and need(k_rows=1000 * rows, **kw) <= tight + 4096


@pytest.mark.parametrize("wrong", [
    dict(dtype=0), dict(dtype=3), dict(heads=0), dict(kv_heads=3), dict(heads=-8, kv_heads=-2), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136),
    dict(n_seq=-1), dict(max_q=-1), dict(max_k=1 << 30), dict(q_rows=-1), dict(n_buckets=-1), dict(n_buckets=129), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e-9), dict(bias=None), dict(bias=4098), dict(cuts=[0, 0, 1]), dict(cuts=[3, 2, 1]),
    dict(q_rows=299), dict(k_rows=299), dict(n_seq=1 << 30, q_ptr=64, k_ptr=64)])
def test_parameters_that_are_refused_need_no_workspace(b, wrong):
    assert b._lib.gbt_attention_backward_workspace_bytes(C.byref(_params(b, **wrong))) == 0
    assert b._lib.gbt_attention_workspace_bytes(C.byref(_params(b, max_q=1, max_k=20_000, k_rows=60_000, **{k: v for k, v in wrong.items()
                                                                                                            if k not in ("max_q", "max_k", "k_rows")}))) == 0 \
        or set(wrong) & {"max_q", "max_k", "k_rows", "q_rows"}


def test_gradient_lists(b):
    def need(*entries):
        arr = (b.Gradient * max(1, len(entries)))(*[b.Gradient(*e) for e in entries])
        return b._lib.gbt_gradient_list_bytes(arr, len(entries))

    assert need() >= 16
    assert need((64, 64, 10, 0)) == need((64, 64, 2048, 0)) < need((64, 64, 2049, 0))
    assert need((64, 64, 0, 0)) >= 16                                          # nothing of it is read
    assert need((0, 0, 0, 1)) >= 16
    for bad in ((64, 64, -1, 0), (64, 64, 5, 3), (64, 64, 5, -1), (0, 64, 5, 0), (64, 0, 5, 0), (66, 64, 5, 0), (65, 64, 5, 1), (64, 65, 5, 2)):
        assert need(bad) == 0
    assert need((64, 64, 1 << 40, 1)) > 0                                      # longer pieces, not a longer list
    many = (b.Gradient * 200_000)(*[b.Gradient(64, 64, 1, 0)] * 200_000)
    assert b._lib.gbt_gradient_list_bytes(many, 200_000) == 0                  # more than 4 MB


@pytest.mark.parametrize("buckets,far", [(1, 10), (2, 1), (3, 5), (7, 40), (32, 128), (128, 500), (64, 100_000)])
@pytest.mark.parametrize("causal", [False, True])
def test_distance_cuts(buckets, far, causal):
    import paper_1806_11248_amd as g
    cuts = g.distance_cuts(buckets, far, causal)
    assert len(cuts) == buckets - 1 and all(x < y for x, y in zip(cuts, cuts[1:]))
    if causal:
        assert not cuts or cuts[-1] == 0
    back = [c for c in cuts if c <= 0]
    for i in range(max(1, len(back) // 2) if back else 0):
        assert back[-1 - i] == -i                                              # the nearest distances have a bucket each
    if len(back) > 8 and far > 2 * len(back):
        assert abs(back[0] + far) <= 1                                         # and the last begins where they were asked to reach
