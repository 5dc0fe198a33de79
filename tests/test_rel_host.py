"""CPU checks of include/cnnk_rel.h: exported symbols, struct layouts, what is refused before anything is launched, and pins of the
oracle (oracle/rel.py): known answers of the generator, finite differences of every gradient, statistics of the masks."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from oracle import rel as R
from paper_2503_23186_amd import cnnk, rel

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4
A = 4096          # an address that is never read


def refused(status, f, *a, **k):
    with pytest.raises(cnnk.CnnkError) as e:
        f(*a, **k)
    assert e.value.status == status


def test_every_symbol_of_the_header_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cnnk_rel.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(cnnk_[a-z0-9_]+)\s*\(", text)))
    assert sorted(rel.EXPORTS) == names
    for n in names:
        assert hasattr(cnnk.lib, n), n
    assert C.sizeof(rel.DropoutDesc) == 32 and C.sizeof(rel.RelDesc) == 32


def test_dropout_refuses_bad_arguments():
    ok = rel.dropout_desc(8, 64, cnnk.BF16, 0.1)
    refused(NULL, rel.cnnk_dropout_fwd, ok, None, None, None, A, A)
    refused(NULL, rel.cnnk_dropout_fwd, ok, A, None, None, A, None)
    refused(NULL, rel.cnnk_dropout_fwd, ok, A, None, None, None, A)                 # no state
    for at in range(4):                                                             # z, bias, res, y off their 16 bytes
        p = [A, A, A, A]
        p[at] += 8
        refused(UNSUPPORTED, rel.cnnk_dropout_fwd, ok, p[0], p[1], p[2], A, p[3])
    refused(UNSUPPORTED, rel.cnnk_dropout_fwd, ok, A, None, None, A + 4, A)
    for d, status in ((rel.dropout_desc(0, 64, cnnk.BF16, 0.1), SHAPE), (rel.dropout_desc(8, 0, cnnk.BF16, 0.1), SHAPE),
                      (rel.dropout_desc(8, 64, cnnk.BF16, 0.1, span=-1), SHAPE), (rel.dropout_desc(8, 64, cnnk.BF16, -0.1), SHAPE),
                      (rel.dropout_desc(8, 64, cnnk.BF16, 1.0), SHAPE), (rel.dropout_desc(8, 64, cnnk.BF16, float("nan")), SHAPE),
                      (rel.dropout_desc(8, 64, cnnk.BF16, 0.999999), UNSUPPORTED), (rel.dropout_desc(8, 60, cnnk.BF16, 0.1), UNSUPPORTED),
                      (rel.dropout_desc(8, 64, 7, 0.1), UNSUPPORTED), (rel.dropout_desc(1 << 40, 64, cnnk.F32, 0.1), UNSUPPORTED)):
        refused(status, rel.cnnk_dropout_fwd, d, A, None, None, A, A)
        refused(status, rel.cnnk_dropout_bwd, d, A, A, A)
        assert rel.cnnk_dropout_workspace_bytes(d) == 0
    need = rel.cnnk_dropout_workspace_bytes(ok)
    assert need > 0
    refused(WORKSPACE, rel.cnnk_dropout_bwd, ok, A, A, A, A, None, 0)
    refused(WORKSPACE, rel.cnnk_dropout_bwd, ok, A, A, A, A, A, need - 1)
    refused(NULL, rel.cnnk_dropout_bwd, ok, None, A, A)
    refused(NULL, rel.cnnk_dropout_bwd, ok, A, None, A)
    refused(NULL, rel.cnnk_rng_advance, None)
    refused(UNSUPPORTED, rel.cnnk_rng_advance, A + 4)


def test_maps_and_plans_refuse_bad_arguments():
    refused(SHAPE, rel.cnnk_rel_buckets_grid, 0, 3, 1, A)
    refused(NULL, rel.cnnk_rel_buckets_grid, 3, 3, 1, None)
    refused(UNSUPPORTED, rel.cnnk_rel_buckets_grid, 91, 91, 0, A)                   # 8281 tokens
    refused(UNSUPPORTED, rel.cnnk_rel_buckets_grid, 65, 65, 0, A)                   # 16641 buckets
    refused(UNSUPPORTED, rel.cnnk_rel_buckets_grid, 100000, 100000, 0, A)
    refused(UNSUPPORTED, rel.cnnk_rel_buckets_grid, 3, 3, 1, A + 2)
    for T, n in ((0, 5), (5, 0), (8193, 5), (5, 16383), (-1, 5)):
        assert rel.cnnk_rel_plan_bytes(T, n) == 0 and rel.cnnk_rel_plan_workspace_bytes(T, n) == 0
    refused(SHAPE, rel.cnnk_rel_plan, 0, 5, A, A, A, 1 << 20)
    refused(UNSUPPORTED, rel.cnnk_rel_plan, 8193, 5, A, A, A, 1 << 30)
    need = rel.cnnk_rel_plan_workspace_bytes(17, 52)
    refused(NULL, rel.cnnk_rel_plan, 17, 52, None, A, A, need)
    refused(NULL, rel.cnnk_rel_plan, 17, 52, A, None, A, need)
    refused(WORKSPACE, rel.cnnk_rel_plan, 17, 52, A, A, None, 0)
    refused(WORKSPACE, rel.cnnk_rel_plan, 17, 52, A, A, A, need - 1)
    refused(UNSUPPORTED, rel.cnnk_rel_plan, 17, 52, A, A + 128, A, need)
    import torch
    with pytest.raises(ValueError):
        rel.make_plan(torch.zeros(4, 4, dtype=torch.int32), 3)                      # not on a GPU


def test_attention_refuses_bad_arguments():
    ok = rel.rel_desc(2, 17, 2, 64, cnnk.BF16, 52, 0.1)
    big = 1 << 40
    fwd = lambda d, qkv=A, table=A, plan=A, lens=A, rng=A, o=A, stats=A: rel.cnnk_rel_attention_fwd(d, qkv, table, plan, lens, rng, o, stats)
    bwd = lambda d, qkv=A, o=A, d_o=A, table=A, plan=A, lens=A, rng=A, stats=A, dqkv=A, dtable=A, ws=A, n=big: \
        rel.cnnk_rel_attention_bwd(d, qkv, o, d_o, table, plan, lens, rng, stats, dqkv, dtable, ws, n)
    D = lambda B=2, T=17, heads=2, dh=64, dt=cnnk.BF16, n=52, p=0.1: rel.rel_desc(B, T, heads, dh, dt, n, p)
    for d, status in ((D(B=0), SHAPE), (D(T=0), SHAPE), (D(heads=0), SHAPE), (D(dh=0), SHAPE), (D(n=-1), SHAPE), (D(p=1.0), SHAPE), (D(p=-0.5), SHAPE),
                      (D(p=float("nan")), SHAPE), (D(dh=48), UNSUPPORTED), (D(dh=256), UNSUPPORTED), (D(dt=5), UNSUPPORTED), (D(T=8193), UNSUPPORTED),
                      (D(T=16385, n=0), UNSUPPORTED), (D(n=16383), UNSUPPORTED), (D(T=16384, n=0, heads=512), UNSUPPORTED), (D(p=0.999999), UNSUPPORTED)):
        refused(status, fwd, d)
        refused(status, bwd, d)
        assert rel.cnnk_rel_attention_workspace_bytes(d) == 0
    for k in ("qkv", "table", "plan", "rng", "o"):
        refused(NULL, fwd, ok, **{k: None})
        refused(UNSUPPORTED, fwd, ok, **{k: A + 2})
    for k in ("lens", "stats"):
        refused(UNSUPPORTED, fwd, ok, **{k: A + 2})
    for k in ("qkv", "o", "d_o", "table", "plan", "rng", "stats", "dqkv"):
        refused(NULL, bwd, ok, **{k: None})
        refused(UNSUPPORTED, bwd, ok, **{k: A + 2})
    for k in ("lens", "dtable", "ws"):
        refused(UNSUPPORTED, bwd, ok, **{k: A + 2})
    need = rel.cnnk_rel_attention_workspace_bytes(ok)
    assert need > rel.cnnk_rel_attention_workspace_bytes(D(n=0)) > 0
    refused(WORKSPACE, bwd, ok, n=need - 1)
    refused(WORKSPACE, bwd, ok, ws=None)


# ---- the oracle --------------------------------------------------------------------------------------------------------

def test_generator_known_answers():
    """Ten rounds: the authors' published answers.  Seven: what their definition gives, a word at a time in Python's integers."""
    f = 0xFFFFFFFF
    got = lambda c, k, r: [int(x) for x in R.philox(c, k, r)]
    assert got((0, 0, 0, 0), (0, 0), 10) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert got((f, f, f, f), (f, f), 10) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    c, k = [0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0]
    want, key = list(c), list(k)
    for _ in range(7):
        a, b = want[0] * R.M0, want[2] * R.M1
        want = [(b >> 32) ^ want[1] ^ key[0], b & f, (a >> 32) ^ want[3] ^ key[1], a & f]
        key = [(key[0] + R.W0) & f, (key[1] + R.W1) & f]
    assert got(c, k, 7) == want


@pytest.mark.parametrize("p", [0.1, 0.5])
def test_masks_of_the_oracle_are_independent_draws(p):
    """Share of what is kept, its correlation with neighbours along every index, with another site and another step: within four
    standard deviations of independent draws."""
    n, B, H, T = 1 << 18, 4, 4, 128
    k0, k1, k2 = R.site_key(11, 3, 0), R.site_key(11, 3, 1), R.site_key(11, 4, 0)
    q, f = R.share(p)
    bound = 4.0 / np.sqrt(n)
    unit = lambda a: ((a > 0).astype(float) - (1 - q / 65536)) / np.sqrt(q / 65536 * (1 - q / 65536))
    e = unit(R.keep_elements(n, p, k0))
    a = unit(R.keep_pairs(B, H, T, p, k0))
    assert abs(e.mean()) < bound and abs(a.mean()) < bound
    assert abs((e[1:] * e[:-1]).mean()) < bound and abs((e[8:] * e[:-8]).mean()) < bound
    for axis in range(4):
        b = np.moveaxis(a, axis, 0)
        assert abs((b[1:] * b[:-1]).mean()) < bound * 1.2
    for k in (k1, k2):
        assert abs((e * unit(R.keep_elements(n, p, k))).mean()) < bound
        assert abs((a * unit(R.keep_pairs(B, H, T, p, k))).mean()) < bound


def test_gradients_of_the_oracle_against_differences():
    rng = np.random.default_rng(5)
    B, T, H, dh, n = 2, 7, 2, 16, 9
    qkv, table, g = rng.standard_normal((B, T, 3 * H * dh)), rng.standard_normal((n, H)), rng.standard_normal((B, T, H * dh))
    bucket = rng.integers(-1, n, (T, T)).astype(np.int32)
    bucket[3] = -1                                                                  # a row that sees nothing
    lens, keep = [5, 7], R.keep_pairs(B, H, T, 0.3, R.site_key(1, 2, 3))
    f = lambda q, t: (R.attention(q, H, t, bucket, lens, keep)["o"] * g).sum()
    r = R.attention(qkv, H, table, bucket, lens, keep, g)
    assert (r["o"][:, 3] == 0).all() and (r["o"][0, 5:] == 0).all() and (r["dqkv"][0, 5:] == 0).all()
    h = 1e-6
    for _ in range(60):
        i = tuple(rng.integers(0, s) for s in qkv.shape)
        d = np.zeros_like(qkv)
        d[i] = h
        assert abs((f(qkv + d, table) - f(qkv - d, table)) / (2 * h) - r["dqkv"][i]) < 1e-7
    for k in range(n):
        for c in range(H):
            d = np.zeros_like(table)
            d[k, c] = h
            assert abs((f(qkv, table + d) - f(qkv, table - d)) / (2 * h) - r["dtable"][k, c]) < 1e-7


def test_attention_refuses_more_threads_than_a_launch_can_have():
    D = lambda B, T, heads: rel.rel_desc(B, T, heads, 16, rel.BF16, 0, 0.0, 0)
    for B, T, heads in ((13421772, 130, 1), (67108863, 1, 1), (33554431, 64, 1), (2 ** 31 - 1, 1, 65535)):
        assert rel.cnnk_rel_attention_workspace_bytes(D(B, T, heads)) == 0
    for B, T, heads in ((8388599, 1, 1), (128, 1, 65535), (5592396, 130, 1)):
        tiles = (T + 31) // 32
        assert (B * heads + 8) * (tiles + 7) < 2 ** 26
        assert rel.cnnk_rel_attention_workspace_bytes(D(B, T, heads)) > 0
