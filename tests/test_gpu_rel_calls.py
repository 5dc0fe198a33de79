"""Calls of include/cnnk_rel.h that its documentation allows and where one value, address or size decides: against oracle/rel.py in float64."""
import threading

import numpy as np
import pytest
import torch

from oracle import rel as R
from test_gpu_rel import DEV, Case, map_of
from test_gpu_rel_block import reference64
from util import host

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
def test_scores_that_overflow_downwards_mask(K, dtype, T):
    """-infinity: one key of a row, then all of them."""
    B, heads, dh = 2, 2, 64
    bucket, n = map_of("grid", T)
    c = Case(K, dtype, B, T, heads, dh, bucket, n, 0.0)
    q = c.gq.view(B, T, 3, heads, dh)
    q[0, 3, 0, 0], q[0, 3, 0, 0, 0] = 0.0, 1e38
    q[0, :, 1, 0, 0] = 0.0
    q[0, 5, 1, 0, 0] = -100.0
    o, m = c.fwd()
    masked = np.array(bucket)
    masked[3, 5] = -1
    want = R.attention(host(q).reshape(B, T, -1) * 1.0, heads, c.table, masked)
    assert np.abs(host(o)[0, 3, :dh] - want["o"][0, 3, :dh]).max() <= (2.0 ** -7 if dtype == "bf16" else 2.0 ** -18) * np.abs(want["bound_o"][0, 3, :dh]).max()
    q[0, :, 1, 0, 0] = -100.0
    o, m = c.fwd()
    assert (o[0, 3, :dh] == 0).all() and m[0, 0, 3].tolist() == [-np.inf, 0.0] and torch.isfinite(o).all()


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


# ---- plans of other maps ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,dh,p", [("bf16", 64, 0.0), ("bf16", 32, 0.2), ("f32", 16, 0.1), ("bf16", 128, 0.0)])
@pytest.mark.parametrize("T,other_T,other_n", [(20, 23, 9), (70, 70, 14), (70, 97, 9), (300, 300, 8), (300, 330, 5000)])
@pytest.mark.parametrize("kind", ["other", "zeros", "ones"])
def test_a_plan_of_another_map_gives_nan(K, dtype, dh, p, T, other_T, other_n, kind):
    """Plans of other sizes that have the call's bytes, and memory that holds none: NaN for every token, zeros past an image's end, nothing written elsewhere."""
    n, heads, lens = 9, 2, [T, T // 2, 0]
    rng = np.random.default_rng(T)
    c = Case(K, dtype, 3, T, heads, dh, rng.integers(-1, n, (T, T)).astype(np.int32), n, p, lens=lens)
    good, size = c.plan, K.cnnk_rel_plan_bytes(T, n)
    plan = torch.full((max(size, K.cnnk_rel_plan_bytes(other_T, other_n)),), 255 if kind == "ones" else 0, dtype=torch.uint8, device=DEV)
    if kind == "other":
        made = K.make_plan(torch.from_numpy(rng.integers(0, other_n, (other_T, other_T)).astype(np.int32)).to(DEV), other_n)
        plan[:made.numel()] = made
    o, m = c.fwd()
    inside = torch.arange(T, device=DEV)[None] < torch.tensor(lens, device=DEV)[:, None]
    need = K.cnnk_rel_attention_workspace_bytes(c.desc)
    dq, dt = torch.full_like(c.gq, 9.0), torch.full((n + 2, heads), 9.0, device=DEV)
    ws = torch.full((need + 1024,), 77, dtype=torch.uint8, device=DEV)
    K.cnnk_rel_attention_bwd(c.desc, c.gq, o, c.gg, c.gt, plan, c.gl, c.s, m, dq, dt[1:], ws[512:], need)
    assert torch.isnan(dq[inside]).all() and (dq[~inside] == 0).all() and torch.isnan(dt[1:-1]).all()
    assert (dt[0] == 9).all() and (dt[-1] == 9).all() and (ws[:512] == 77).all() and (ws[512 + need:] == 77).all()
    c.plan = plan
    o2, m2 = c.fwd()
    assert torch.isnan(o2[inside]).all() and (o2[~inside] == 0).all()
    assert torch.isnan(m2[..., 1].permute(0, 2, 1)[inside]).all() and torch.isneginf(m2[..., 0].permute(0, 2, 1)[~inside]).all()
    c.plan = good
    assert torch.equal(c.fwd()[0], o)


@pytest.mark.parametrize("T,n", [(3300, 16129), (4100, 12000)])
def test_a_long_image_with_a_plan_of_another_map(K, T, n):
    """One image whose dx becomes runs of a bucket in the walk: a plan of fewer buckets in its place."""
    heads, dh = 12, 16
    m = torch.zeros(T, T, dtype=torch.int32, device=DEV)
    made = K.make_plan(m, n - 70)
    plan = torch.zeros(K.cnnk_rel_plan_bytes(T, n), dtype=torch.uint8, device=DEV)
    plan[:made.numel()] = made
    d = K.rel_desc(1, T, heads, dh, K.BF16, n, 0.0, 0)
    x = lambda *s: torch.ones(*s, dtype=torch.bfloat16, device=DEV)
    qkv, o, g, table, stats = x(1, T, 3 * heads * dh), x(1, T, heads * dh), x(1, T, heads * dh), torch.ones(n, heads, device=DEV), torch.zeros(1, heads, T, 2, device=DEV)
    dq, dt, need = torch.zeros_like(qkv), torch.zeros_like(table), K.cnnk_rel_attention_workspace_bytes(d)
    ws = torch.full((need + 1024,), 77, dtype=torch.uint8, device=DEV)
    K.cnnk_rel_attention_bwd(d, qkv, o, g, table, plan, None, None, stats, dq, dt, ws[512:], need)
    assert torch.isnan(dq).all() and torch.isnan(dt).all() and (ws[:512] == 77).all() and (ws[512 + need:] == 77).all()


# ---- workspaces ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,B,T,heads,dh,buckets", [("bf16", 8, 300, 60, 16, 12000), ("bf16", 95, 40, 12, 64, 0), ("bf16", 64, 50, 24, 32, 0), ("f32", 7, 260, 60, 32, 0), ("bf16", 7, 2050, 12, 16, 0)])
def test_sums_stay_in_the_workspace(K, dtype, B, T, heads, dh, buckets):
    """Three images to a workgroup, in batches that three does not divide, so that heads begin everywhere in one: nothing behind the workspace is written, and with dtable = NULL
    nothing behind the rows; the table's gradient is that of one image after the other.

    A bucket has M = T * T / 91 * B terms of either sign, sums of k of them are about sqrt(k) of one, and adding to one rounds by 2^-24 of it at most.  The roundings of all
    M additions, independent, are together 2^-24 sqrt(1 + 2 + .. + M) = 2^-24 M / sqrt(2) of a term, 2^-24 sqrt(M / 2) of the sum; there are two such sums, and a factor 2 is for
    terms of unlike size."""
    n = buckets or 91
    g = torch.Generator(device=DEV).manual_seed(B)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    qkv, do, table = rand(B, T, 3 * heads * dh).to(t), rand(B, T, heads * dh).to(t), rand(n, heads)
    plan = K.make_plan(torch.randint(-1, 91, (T, T), generator=g, device=DEV, dtype=torch.int32), n)
    desc = lambda b, k=n: K.rel_desc(b, T, heads, dh, K.BF16 if dtype == "bf16" else K.F32, k, 0.0, 0)

    def run(b, q, d, dt, need):
        o, st, dq = torch.empty_like(d), torch.empty(b, heads, T, 2, device=DEV), torch.empty_like(q)
        ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
        K.cnnk_rel_attention_fwd(desc(b), q, table, plan, None, None, o, st)
        K.cnnk_rel_attention_bwd(desc(b), q, o, d, table, plan, None, None, st, dq, dt, ws, need)
        assert (ws[need:] == 77).all()
        return dq

    dt, one, want = torch.empty_like(table), torch.empty_like(table), torch.zeros_like(table, dtype=torch.float64)
    dq = run(B, qkv, do, dt, K.cnnk_rel_attention_workspace_bytes(desc(B)))
    assert torch.equal(run(B, qkv, do, None, K.cnnk_rel_attention_workspace_bytes(desc(B, 0))), dq)
    for b in range(B):
        alone = run(1, qkv[b:b + 1], do[b:b + 1], one, K.cnnk_rel_attention_workspace_bytes(desc(1)))
        assert torch.equal(alone[0], dq[b])
        want += one.double()
    assert float((dt.double() - want).norm() / want.norm()) <= 2.0 * 2.0 ** -24 * np.sqrt(T * T / 91 * B)      # sqrt(2) sums, times 2


@pytest.mark.parametrize("dtype,B,T,heads,dh", [("bf16", 20, 70, 56, 16), ("bf16", 11, 130, 52, 64), ("bf16", 11, 100, 60, 32), ("bf16", 7, 65, 80, 128), ("f32", 20, 70, 56, 64),
                                                ("f32", 11, 130, 52, 32), ("f32", 7, 65, 80, 128)])
@pytest.mark.parametrize("kind,p,ragged", [("grid", 0.1, False), ("random", 0.2, True), ("grid", 0.0, True)])
def test_workgroups_that_go_from_head_to_head(K, dtype, B, T, heads, dh, kind, p, ragged):
    """Two or three images to a workgroup, in batches that these do not divide: in the walk for dk and dv a workgroup goes on to the next head, loads its column of the table and adds
    up dx of several images that have tokens.  Every element against the oracle; padded batches with empty images at the ends of a workgroup's."""
    bucket, n = map_of(kind, T)
    lens = [(0, T, T - 1, 33, T // 2, 1, T, 0, 64)[i % 9] for i in range(B)] if ragged else None
    Case(K, dtype, B, T, heads, dh, bucket, n, p, lens=lens, past=np.nan).check()


# ---- long images ---------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,T,heads,dh,buckets", [(t,) + c for t in ("f32", "bf16") for c in ((300, 2, 64, 16382), (2049, 1, 32, 3), (4100, 1, 64, 16129), (8192, 1, 16, 40))] +
                         [("f32", 16384, 1, 16, 0), ("f32", 5000, 1, 128, 0)])
def test_long_images_to_fp32(K, dtype, T, heads, dh, buckets):
    """Norm of the error over the norm of the result, fp32 storage, and the table's gradient, an fp32 sum, with either.  Terms of either sign: a sum of k terms is about sqrt(k) of
    one, so that the roundings of T additions, independent, are 2^-24 sqrt(T / 2) of the sum, those of a score's dh products 2^-24 sqrt(dh / 2).  A probability has besides the
    rounding of the exponent, a number below 32 (16 2^-24), of the difference in front of it, below 16 (8 2^-24), of the logarithm of the sum (8 2^-24), and of the exponential and
    the products around it (fewer than 16 of 2^-24): e = 2^-24 (sqrt(T / 2) + sqrt(dh / 2) + 48).  dx has the errors of a probability and of dP: 2 e for the gradients.  A
    bucket's sum has chains of 32 pairs of a block, then of its runs: 64 or more threads share more than 4096, so that sqrt(T / 2) is not passed."""
    gen = torch.Generator(device=DEV).manual_seed(T + dh)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    qkv, g = rand(T, 3 * heads * dh).to(t), rand(T, heads * dh).to(t)
    table = plan = bucket = dt = None
    if buckets:
        table = rand(buckets, heads)
        bucket = torch.randint(-1, buckets, (T, T), generator=gen, device=DEV, dtype=torch.int32)
        plan, dt = K.make_plan(bucket, buckets), torch.full_like(table, 7.0)
    d = K.rel_desc(1, T, heads, dh, K.BF16 if dtype == "bf16" else K.F32, buckets, 0.0, 0)
    o, stats, dq = torch.full((T, heads * dh), 7.0, device=DEV, dtype=t), torch.empty(1, heads, T, 2, device=DEV), torch.full_like(qkv, 7.0)
    ws = torch.empty(K.cnnk_rel_attention_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    K.cnnk_rel_attention_fwd(d, qkv, table, plan, None, None, o, stats)
    K.cnnk_rel_attention_bwd(d, qkv, o, g, table, plan, None, None, stats, dq, dt, ws, ws.numel())
    wo, wd, wt = reference64(qkv, heads, dh, table, bucket, g)
    off = lambda a, b: float((a.double() - b).norm() / b.norm())
    e = 2.0 ** -24 * ((T / 2) ** 0.5 + (dh / 2) ** 0.5 + 48)
    if dtype == "f32":
        assert off(o, wo) <= e and off(dq, wd) <= 2 * e, (off(o, wo), off(dq, wd), e)
    if buckets:
        assert off(dt, wt) <= 2 * e, (off(dt, wt), e)


# ---- host threads --------------------------------------------------------------------------------------------------------------------

def test_calls_from_host_threads_at_once(K):
    """Tables that take different shares of more than 64 KB of LDS, each from a thread and on a stream of its own: every call is taken, the results are those of calls alone."""
    def case(n):
        T, heads, dh = 260, 2, 64
        g = torch.Generator(device=DEV).manual_seed(n)
        rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
        qkv, do, table = rand(2, T, 3 * heads * dh).bfloat16(), rand(2, T, heads * dh).bfloat16(), rand(n, heads)
        plan = K.make_plan(torch.randint(-1, n, (T, T), generator=g, device=DEV, dtype=torch.int32), n)
        d = K.rel_desc(2, T, heads, dh, K.BF16, n, 0.0, 0)
        o, st, dq, dt = torch.empty_like(do), torch.empty(2, heads, T, 2, device=DEV), torch.empty_like(qkv), torch.empty_like(table)
        ws = torch.empty(K.cnnk_rel_attention_workspace_bytes(d), dtype=torch.uint8, device=DEV)

        def step(stream):
            K.cnnk_rel_attention_fwd(d, qkv, table, plan, None, None, o, st, stream)
            K.cnnk_rel_attention_bwd(d, qkv, o, do, table, plan, None, None, st, dq, dt, ws, ws.numel(), stream)
        return step, (o, st, dq, dt)

    cases, streams, failed = [case(n) for n in (9000, 12000, 16382)], [torch.cuda.Stream() for _ in range(3)], []
    want = []
    for step, out in cases:
        step(0)
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
        for t in out:
            t.zero_()
    torch.cuda.synchronize()

    def work(step, stream):
        try:
            for _ in range(200):
                step(stream)
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(c[0], s.cuda_stream)) for c, s in zip(cases, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for (_, out), w in zip(cases, want):
        assert all(torch.equal(a, b) for a, b in zip(out, w))


# ---- the largest and the smallest -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("B,heads,buckets", [(8388599, 1, 0), (1, 1, 1), (128, 65535, 0), (65536, 100, 1)])
def test_images_of_one_token(K, B, heads, buckets):
    """As many as a launch can have: the output is v, its gradient d_o, bit for bit; q, k and the table have none (dP is delta, but for the rounding of two sums of 16
    products: 24 2^-24 of their terms' sizes, 16 * 4.5^2 at most, times |k| / 4; for the table the sum of B such numbers)."""
    dh, g = 16, torch.Generator(device=DEV).manual_seed(2)
    qkv, do = torch.randn(B, 1, 3 * heads * dh, generator=g, device=DEV, dtype=torch.float32).bfloat16().clamp_(-4.5, 4.5), torch.randn(B, 1, heads * dh, generator=g, device=DEV).bfloat16().clamp_(-4.5, 4.5)
    d = K.rel_desc(B, 1, heads, dh, K.BF16, buckets, 0.0, 0)
    table = plan = dt = None
    if buckets:
        table, plan, dt = torch.randn(1, heads, generator=g, device=DEV), K.make_plan(torch.zeros(1, 1, dtype=torch.int32, device=DEV), 1), torch.full((1, heads), 7.0, device=DEV)
    o, st, dq = torch.zeros_like(do), torch.zeros(B, heads, 1, 2, device=DEV), torch.full_like(qkv, 7.0)
    ws = torch.empty(K.cnnk_rel_attention_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    K.cnnk_rel_attention_fwd(d, qkv, table, plan, None, None, o, st)
    K.cnnk_rel_attention_bwd(d, qkv, o, do, table, plan, None, None, st, dq, dt, ws, ws.numel())
    w = heads * dh
    assert torch.equal(o, qkv[..., 2 * w:]) and torch.equal(dq[..., 2 * w:], do)
    one = 24 * 2.0 ** -24 * 2 * 16 * 4.5 ** 2
    assert float(dq[..., :2 * w].abs().max()) <= one * 4.5 / 4 * 1.01
    if buckets:
        assert float(dt.abs().max()) <= one * B


def test_as_many_heads_as_there_are(K):
    """65535 heads, with a bias: every one by the formula in 64 bits."""
    B, T, heads, dh, n = 3, 3, 65535, 16, 4
    g = torch.Generator(device=DEV).manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    qkv, do, table = rand(B, T, 3 * heads * dh), rand(B, T, heads * dh), rand(n, heads)
    bucket = torch.tensor([[0, 1, -1], [2, 3, 0], [1, -1, 2]], dtype=torch.int32, device=DEV)
    d, plan = K.rel_desc(B, T, heads, dh, K.F32, n, 0.0, 0), K.make_plan(bucket, n)
    o, st, dq, dt = torch.zeros_like(do), torch.zeros(B, heads, T, 2, device=DEV), torch.full_like(qkv, 7.0), torch.full_like(table, 7.0)
    ws = torch.empty(K.cnnk_rel_attention_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    K.cnnk_rel_attention_fwd(d, qkv, table, plan, None, None, o, st)
    K.cnnk_rel_attention_bwd(d, qkv, o, do, table, plan, None, None, st, dq, dt, ws, ws.numel())
    q, k, v = (x.requires_grad_() for x in qkv.double().view(B, T, 3, heads, dh).permute(2, 0, 3, 1, 4).contiguous().unbind(0))
    w = table.double().requires_grad_()
    x = (q[..., :, None, :] * k[..., None, :, :]).sum(-1) / 4 + w[bucket.long().clamp(min=0)].permute(2, 0, 1)
    y = (torch.softmax(x.masked_fill(bucket < 0, -1e300), -1)[..., None] * v[..., None, :, :]).sum(-2)
    y.backward(do.double().view(B, T, heads, dh).transpose(1, 2))
    off = lambda a, b: float((a.double() - b).norm() / b.norm())
    e = 2.0 ** -24 * 48                          # as in test_long_images_to_fp32, whose sums are longer
    assert off(o.view(B, T, heads, dh), y.detach().transpose(1, 2)) <= e and off(dt, w.grad) <= 2 * e
    for i, t in enumerate((q, k, v)):
        assert off(dq.view(B, T, 3, heads, dh)[:, :, i], t.grad.transpose(1, 2)) <= 2 * e


# ---- addresses -------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,T", [("bf16", 45), ("f32", 130)])
def test_every_alignment_that_is_asked_for_is_enough(K, dtype, T):
    """Activations and workspaces 16 bytes off a line, statistics 8, the table, its gradient and the lengths 4: the bits of aligned ones."""
    bucket, n = map_of("grid", T)
    c = Case(K, dtype, 2, T, 2, 32, bucket, n, 0.1, lens=[T, T - 9])
    o, m = c.fwd()
    dq, dt = c.bwd(o, m)

    def off(t, by):
        raw = torch.empty(t.numel() * t.element_size() + 256, dtype=torch.uint8, device=DEV)
        return raw[by:by + t.numel() * t.element_size()].view(t.dtype).view(t.shape) if by % t.element_size() == 0 else None

    def moved(t, by):
        x = off(t, by)
        x.copy_(t)
        return x

    c.gq, c.gg, c.gt, c.gl, c.s = moved(c.gq, 16), moved(c.gg, 48), moved(c.gt, 4), moved(c.gl, 4), moved(c.s, 8)
    o2, m2, dq2, dt2 = off(o, 16), off(m, 8), off(dq, 80), off(dt, 12)
    need = K.cnnk_rel_attention_workspace_bytes(c.desc)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    for at in (16, 240):
        K.cnnk_rel_attention_fwd(c.desc, c.gq, c.gt, c.plan, c.gl, c.s, o2, m2)
        K.cnnk_rel_attention_bwd(c.desc, c.gq, o2, c.gg, c.gt, c.plan, c.gl, c.s, m2, dq2, dt2, ws[at:], need)
        for a, b in ((o, o2), (m, m2), (dq, dq2), (dt, dt2)):
            assert torch.equal(a, b)
    wp = torch.empty(K.cnnk_rel_plan_workspace_bytes(T, n) + 16, dtype=torch.uint8, device=DEV)
    plan, bm = torch.empty_like(c.plan), moved(torch.from_numpy(np.ascontiguousarray(bucket, dtype=np.int32)).to(DEV), 4)
    K.cnnk_rel_plan(T, n, bm, plan, wp[16:], wp.numel() - 16)
    c.plan = plan
    assert torch.equal(c.fwd()[0], o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropout_at_every_alignment_that_is_asked_for(K, dtype):
    rows, C, t = 70, 264, torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device=DEV).manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    z, res, bias, s = rand(rows, C).to(t), rand(rows, C).to(t), rand(C), torch.tensor([3, 4], device=DEV)
    d = K.dropout_desc(rows, C, K.BF16 if dtype == "bf16" else K.F32, 0.3, 2)
    need = K.cnnk_dropout_workspace_bytes(d)
    got = []
    for by, small in ((0, 0), (16, 4), (112, 12)):
        at = lambda x, k: torch.empty(x.numel() * x.element_size() + 256, dtype=torch.uint8, device=DEV)[k:k + x.numel() * x.element_size()].view(x.dtype).view(x.shape).copy_(x)
        a, r, b, st = at(z, by), at(res, by), at(bias, by), at(s, by % 16 + 8 if by else 0)
        y, dz, db = at(z, by), at(z, by), at(bias, small)
        K.cnnk_dropout_fwd(d, a, b, r, st, y)
        K.cnnk_dropout_bwd(d, a, st, dz, db, at(torch.zeros(need, dtype=torch.uint8, device=DEV), by), need)
        got.append((y, dz, db))
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(other, got[0]))
