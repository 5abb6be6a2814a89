"""What the operators around a tower decide on the host: layouts, workspaces, refusals; and the 64-bit forms that they are compared with (no GPU)."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import tower_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def b():
    import paper_1806_11248_amd as g
    if not os.path.exists(g.LIB_PATH):
        from paper_1806_11248_amd import build
        build.build()
    g.load()
    return g.binding


@pytest.mark.parametrize("name,struct", [("gbt_embedding_params", "EmbeddingParams"), ("gbt_norm_rotate_params", "NormRotateParams"), ("gbt_matrix", "Matrix")])
def test_struct_layouts_match_header(b, name, struct):
    header = open(os.path.join(ROOT, "include", "gbt.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), header, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    of = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}
    fields = []
    for kind, names in re.findall(r"(?:const )?(int32_t|int64_t|float|double|void) ([^;]*);", body):
        fields += [(n.strip(" *"), C.c_void_p if "*" in n else of[kind]) for n in names.split(",")]
    assert fields == getattr(b, struct)._fields_


def _embedding(b, **kw):
    p = dict(table_dtype=0, out_dtype=1, id_bytes=8, width=64, n_ids=10_000, n_rows=500, table_stride=64, out_stride=64, ids=4096, scale=1.0)
    p.update(kw)
    return b.EmbeddingParams(*p.values())


def test_embedding_workspace(b):
    need = b._lib.gbt_embedding_backward_workspace_bytes
    assert need(None) == 0
    # four lists of 32 bits, counts of up to 1024 digits a tile, two sums of a row a chunk of at least 16 places
    assert 4 * 4 * 10_000 <= need(C.byref(_embedding(b))) <= 4 * 4 * 10_000 + 4096 * 8 + 2 * 4 * 64 * 10_000 // 16 + 4096
    assert need(C.byref(_embedding(b, n_ids=2048))) == 0 and need(C.byref(_embedding(b, n_ids=0))) == 0          # nothing is sorted
    assert need(C.byref(_embedding(b, n_ids=2048, n_rows=1 << 20))) > 0                                          # too many rows to look through the ids for
    assert need(C.byref(_embedding(b, n_ids=1 << 30, n_rows=1 << 30))) > 16 << 30
    # few rows: sums of all of them, and which were met, by up to four waves on each of 256 compute units; one row more, or wider ones, are sorted
    few = need(C.byref(_embedding(b, n_ids=900_000, n_rows=12)))
    assert 1000 * (12 * 64 * 4 + 4) <= few <= 1024 * (12 * 64 * 4 + 4) + 512
    assert need(C.byref(_embedding(b, n_ids=900_000, n_rows=32))) < 4 * 4 * 900_000 <= need(C.byref(_embedding(b, n_ids=900_000, n_rows=33)))
    assert need(C.byref(_embedding(b, n_ids=900_000, n_rows=12, width=257))) >= 4 * 4 * 900_000
    assert need(C.byref(_embedding(b, n_ids=1 << 30, n_rows=1, width=1))) < 1 << 20
    for wrong in (dict(table_dtype=3), dict(out_dtype=-1), dict(id_bytes=2), dict(width=0), dict(width=(1 << 20) + 1), dict(n_ids=-1), dict(n_ids=(1 << 30) + 1),
                  dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(table_stride=-1), dict(out_stride=-1), dict(scale=math.nan), dict(scale=math.inf), dict(ids=None),
                  dict(ids=4100)):
        assert need(C.byref(_embedding(b, **wrong))) == 0, wrong


def _rotate(b, **kw):
    p = dict(dtype=1, heads=8, kv_heads=2, head_dim=64, turned=64, halves=1, store=0, n_seq=3, position_bytes=4, eps=1e-6, rows=300, out_rows=300, q_ptr=None, k_ptr=None,
             k_len=None, positions=None, q_weight=64, k_weight=64, turns=64)
    p.update(kw)
    return b.NormRotateParams(*p.values())


@pytest.mark.parametrize("wrong", [
    dict(dtype=0), dict(dtype=3), dict(heads=0), dict(kv_heads=0), dict(heads=1 << 17), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136), dict(turned=4), dict(turned=-8),
    dict(turned=72), dict(n_seq=-1), dict(n_seq=7), dict(eps=-1e-6), dict(eps=2.0), dict(eps=math.nan), dict(rows=-1), dict(out_rows=299), dict(positions=64, position_bytes=2),
    dict(positions=66), dict(turns=None), dict(turns=68), dict(q_weight=66), dict(k_weight=65), dict(q_ptr=4), dict(k_ptr=4), dict(k_len=2),
    dict(store=1, out_rows=301)])
def test_rotation_parameters_that_are_refused_need_no_workspace(b, wrong):
    need = b._lib.gbt_norm_rotate_backward_workspace_bytes
    assert need(C.byref(_rotate(b))) > 0
    assert need(C.byref(_rotate(b, **wrong))) == 0


def _matrices(b, *entries):
    return (b.Matrix * max(1, len(entries)))(*[b.Matrix(*e) for e in entries]), len(entries)


def test_matrices(b):
    L = b._lib
    ok = (64, 64, 100, 200, 0, 1.0)
    assert L.gbt_orthogonalise_workspace_bytes(*_matrices(b, (64, 64, 64, 384, 0, 1.0), (64, 64, 384, 5, 1, 1.0))) == 0      # one workgroup's, without
    assert L.gbt_orthogonalise_workspace_bytes(*_matrices(b, (64, 64, 65, 65, 0, 1.0))) > 0 and L.gbt_orthogonalise_workspace_bytes(*_matrices(b, (64, 64, 385, 2, 0, 1.0))) > 0
    assert L.gbt_matrix_list_bytes(*_matrices(b)) >= 16 and L.gbt_orthogonalise_workspace_bytes(*_matrices(b)) == 0
    # an entry for each matrix, and the tiles of each kind of product by eight XCDs
    assert L.gbt_matrix_list_bytes(*_matrices(b)) < L.gbt_matrix_list_bytes(*_matrices(b, ok)) < L.gbt_matrix_list_bytes(*_matrices(b, ok, ok)) <= 2000
    assert L.gbt_matrix_list_bytes(*_matrices(b, (64, 64, 4096, 4096, 0, 1.0))) >= 8 * (32 * 32 + 2 * 32 * 33 // 2)
    assert L.gbt_orthogonalise_workspace_bytes(*_matrices(b, (0, 0, 0, 5, 0, 1.0))) == 0                          # nothing of it is read
    # 12 bytes an element and 20 for each of X X^T's, of whole tiles
    big = (64, 64, 1024, 4096, 1, 1.0)
    one = L.gbt_orthogonalise_workspace_bytes(*_matrices(b, big))
    assert 12 * 1024 * 4096 + 20 * 1024 * 1024 <= one <= 1.05 * (12 * 1024 * 4096 + 20 * 1024 * 1024)
    # as many at a time as fit 2 GB
    assert one < L.gbt_orthogonalise_workspace_bytes(*_matrices(b, *[big] * 100)) <= 2 << 30 | 1 << 20
    huge = (64, 64, 20_000, 20_000, 1, 1.0)
    assert L.gbt_orthogonalise_workspace_bytes(*_matrices(b, huge)) > 2 << 30
    assert L.gbt_orthogonalise_workspace_bytes(*_matrices(b, huge, big)) == L.gbt_orthogonalise_workspace_bytes(*_matrices(b, huge))
    for bad in ((64, 64, -1, 5, 0, 1.0), (64, 64, 5, 5, 3, 1.0), (64, 64, 5, 5, -1, 1.0), (0, 64, 5, 5, 0, 1.0), (64, 0, 5, 5, 0, 1.0), (66, 64, 5, 5, 0, 1.0),
                (64, 65, 5, 5, 1, 1.0), (64, 64, 5, 5, 0, math.nan), (64, 64, 5, (1 << 20) + 1, 0, 1.0), (64, 64, 40_000, 40_000, 0, 1.0)):
        assert L.gbt_matrix_list_bytes(*_matrices(b, ok, bad)) == 0 and L.gbt_orthogonalise_workspace_bytes(*_matrices(b, ok, bad)) == 0, bad
    assert L.gbt_matrix_list_bytes(None, 3) == 0 and L.gbt_matrix_list_bytes(None, -1) == 0
    assert L.gbt_matrix_list_bytes(*_matrices(b, *[ok] * 65_537)) == 0


def test_null_contexts_are_refused(b):
    L = b._lib
    assert L.gbt_embedding(None, None, None, None) == b.EINVAL and L.gbt_embedding_backward(None, None, None, None, 0, None, 0) == b.EINVAL
    assert L.gbt_norm_rotate(*[None] * 8) == b.EINVAL and L.gbt_norm_rotate_backward(*[None] * 11, 0) == b.EINVAL
    assert L.gbt_matrix_list(None, None, 0, None, 0) == b.EINVAL and L.gbt_orthogonalise(None, None, None, 0, 5, 1.0, 0.0, 0.0, None, 0) == b.EINVAL


def test_rotation_turns():
    import paper_1806_11248_amd as g
    t = g.rotation_turns(64, 10_000.0, "cpu")
    assert t.dtype == torch.float64 and t.shape == (32,) and abs(float(t[0]) - 1 / (2 * math.pi)) < 1e-16
    assert abs(float(t[16]) * 2 * math.pi - 0.01) < 1e-16 and g.rotation_turns(0, device="cpu").shape == (0,)


def test_the_plain_forms():
    """Against other ways to write them."""
    rng = torch.Generator().manual_seed(0)
    table, ids = torch.randn(7, 5, generator=rng), torch.tensor([[3, -1], [6, 7], [3, 0]])
    out = tower_ref.lookup(table, ids, 2.0)
    assert torch.equal(out[0, 0], 2 * table[3].double()) and bool((out[0, 1] == 0).all()) and bool((out[1, 1] == 0).all())
    dout = torch.randn(3, 2, 5, generator=rng)
    grad, bound = tower_ref.lookup_gradient(dout, ids, 7, 2.0)
    assert torch.allclose(grad[3], 2 * (dout[0, 0] + dout[2, 0]).double()) and bool((grad[[1, 2, 4, 5]] == 0).all()) and bool((bound[3] > 0).all())
    x, w = torch.randn(4, 2, 16, generator=rng), torch.randn(16, generator=rng)
    turns = torch.tensor([0.25, 0.5, 0.0, 0.125], dtype=torch.float64)
    there = torch.tensor([True, True, True, False])
    for halves in (True, False):
        y, _ = tower_ref.rotate(x, w, turns, torch.tensor([0, 1, 2, 3]), there, 0.0, halves)
        n = x.double() / x.double().square().mean(-1, keepdim=True).sqrt() * w.double()
        assert torch.allclose(y[0], n[0]) and bool((y[3] == 0).all()) and torch.allclose(y[:, :, 8:], torch.where(there[:, None, None], n, 0.0)[:, :, 8:])
        a, c = (0, 4) if halves else (0, 1)
        assert torch.allclose(y[1, :, a], -n[1, :, c]) and torch.allclose(y[1, :, c], n[1, :, a])          # a quarter
        assert torch.allclose(y[2, :, a], -n[2, :, a]) and torch.allclose(y[2, :, c], -n[2, :, c])         # a half
    there, place, to = tower_ref.places(6, [1, 3, 3, 5], [0, 4, 4, 9], [3, 0, 1])
    assert there.tolist() == [False, True, True, True, True, False] and place.tolist()[1:5] == [1, 2, -1, 0] and to.tolist() == [-1, 1, 2, -1, 4, -1]
    g = torch.randn(6, 9, generator=rng)
    for shape in (g, g.t()):
        z, x = tower_ref.newton_schulz(shape, 3, (3.4445, -4.775, 2.0315))[0], shape.double() / torch.linalg.vector_norm(shape.double())
        for _ in range(3):
            gram = x @ x.t()
            x = 3.4445 * x + (-4.775 * gram + 2.0315 * gram @ gram) @ x
        assert torch.allclose(z, x, rtol=0, atol=1e-12)
