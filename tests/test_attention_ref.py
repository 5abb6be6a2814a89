"""The 64-bit attention that the GPU tests judge by: its gradients are those of its own values, by differences (no GPU)."""
import math

import pytest
import torch

from attention_ref import Reference


@pytest.mark.parametrize("causal", [False, True])
def test_reference_gradients_are_differences_of_its_values(causal):
    rng = torch.Generator().manual_seed(3)
    spans = [(0, 5, 0, 7), (5, 4, 7, 2), (9, 0, 9, 3), (9, 3, 12, 0)]       # more keys, fewer keys, no queries, no keys
    H, K, D, cuts = 4, 2, 8, [-3, -1, 0, 2]

    def r(*shape):
        return torch.randn(*shape, generator=rng, dtype=torch.float64)

    q, k, v, g, bias = r(12, H, D), r(12, K, D), r(12, K, D), r(12, H, D), r(5, H)

    def ref(q, k, v, bias, g=None):
        return Reference(q, k, v, spans, causal, 0.4, bias, cuts, g)

    a = ref(q, k, v, bias, g)
    for name, x, grad in (("q", q, a.dq), ("k", k, a.dk), ("v", v, a.dv), ("bias", bias, a.dbias)):
        for trial in range(3):
            d, h = r(*x.shape), 1e-5
            args = dict(q=q, k=k, v=v, bias=bias)
            hi = (ref(**{**args, name: x + h * d}).out * g).sum()
            lo = (ref(**{**args, name: x - h * d}).out * g).sum()
            assert math.isclose(float((hi - lo) / (2 * h)), float((grad * d).sum()), rel_tol=1e-7, abs_tol=1e-8), name
    if causal:       # queries before the first key of their sequence see none
        assert torch.equal(a.out[5:7], torch.zeros(2, H, D, dtype=torch.float64)) and torch.isinf(a.lse[:, 5:7]).all()
    assert torch.equal(a.out[9:12], torch.zeros(3, H, D, dtype=torch.float64))
    # a probability's row adds up to one, so a bias for every distance alike changes nothing
    assert float(a.dbias.sum(0).abs().max()) < 1e-12
