"""Calls of include/cnnk_rel.h that its documentation allows and where one value, address or size decides: against oracle/rel.py in float64."""
import numpy as np
import pytest
import torch

from test_gpu_rel import DEV, Case, map_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    assert torch.cuda.is_available(), "the GPU tests need a GPU"
    from paper_2503_23186_amd import rel
    return rel


# ---- values that are not finite ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,p", [(20, 0.0), (100, 0.0), (100, 0.2), (300, 0.1)])
@pytest.mark.parametrize("where", ["query", "key", "value", "overflow"])
def test_what_is_not_finite_is_handed_on(K, dtype, T, p, where):
    """One bad token of image 1, head 0: rows that see it have NaN in their outputs, statistics and gradients, other images and heads the bits they had."""
    B, heads, dh, bad = 3, 2, 64, T // 2
    bucket, n = map_of("grid", T)
    c = Case(K, dtype, B, T, heads, dh, bucket, n, p)
    clean = c.fwd()
    clean += c.bwd(*clean)
    q = c.gq.view(B, T, 3, heads, dh)
    if where == "overflow":                      # 1e38 * 1e2: q . k is +infinity, in this token's row alone
        q[1, bad, 0, 0] = 1e38
        q[1, :, 1, 0] = 1e2
    else:
        q[1, bad, ("query", "key", "value").index(where), 0, 5] = float("nan")
    o, m = c.fwd()
    dq, dt = c.bwd(o, m)
    rows = torch.zeros(B, T, heads, dtype=torch.bool, device=DEV)
    rows[1, bad if where in ("query", "overflow") else slice(None), 0] = True
    assert (torch.isnan(o.view(B, T, heads, dh)).any(-1) == rows).all()
    if where != "value":
        assert (torch.isnan(m[..., 1]) == rows.permute(0, 2, 1)).all()
    d = torch.isnan(dq.view(B, T, 3, heads, dh)).any(-1)
    assert d[..., 0, :][rows].all()                            # dq of those rows
    assert d[1, :, 1, 0].all()                                 # dk of the keys that they see
    if where != "value":                                       # dv_u = sum_t keep A[t, u] d_o_t / (1 - p): of the keys that one of those rows keeps, and of no others
        kept = np.ones((T, T), bool) if p == 0 else c.keep[1, 0] > 0
        assert (d[1, :, 2, 0].cpu().numpy() == kept[rows[1, :, 0].cpu().numpy()].any(0)).all()
    assert torch.isnan(dt[:, 0]).any() and torch.isfinite(dt[:, 1]).all() and torch.equal(dt[:, 1], clean[3][:, 1])
    keep = lambda t, k: t.view(B, T, k, heads, -1)
    for a, b, k in ((o, clean[0], 1), (dq, clean[2], 3)):
        a, b = keep(a, k), keep(b, k)
        assert torch.equal(a[0::2], b[0::2]) and torch.equal(a[:, :, :, 1], b[:, :, :, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [17, 130])
def test_a_table_that_is_not_a_number(K, dtype, T):
    """Rows that name the entry have NaN, of the others the results are those of a finite entry in its place."""
    heads, n = 2, 5
    bucket = np.random.default_rng(2).integers(0, 4, (T, T)).astype(np.int32)
    bucket[3, 2], bucket[T - 1] = 4, 4
    table = np.random.default_rng(4).standard_normal((n, heads)).astype(np.float32)
    c = Case(K, dtype, 2, T, heads, 64, bucket, n, 0.0, table=table)
    good, _ = c.fwd()
    c.gt[4, 1] = float("nan")
    o, m = c.fwd()
    dq, dt = c.bwd(o, m)
    bad = torch.zeros(2, T, heads, dtype=torch.bool, device=DEV)
    bad[:, 3, 1] = bad[:, T - 1, 1] = True
    assert (torch.isnan(o.view(2, T, heads, 64)).all(-1) == bad).all() and (torch.isnan(m[..., 1]) == bad.permute(0, 2, 1)).all()
    assert torch.equal(o.view(2, T, heads, 64)[~bad], good.view(2, T, heads, 64)[~bad])
    assert torch.isnan(dq.view(2, T, 3, heads, 64)[:, :, 0][bad]).all() and torch.isnan(dt[4, 1]) and torch.isfinite(dt[:, 0]).all()
