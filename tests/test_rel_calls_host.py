"""CPU checks of calls of include/cnnk_rel.h: what the binding refuses, sizes of workspaces."""
import pytest
import torch

from paper_2503_23186_amd import cnnk, rel

A = 4096          # an address that is never read


def test_a_plan_tensor_of_fewer_bytes_is_refused():
    need = rel.cnnk_rel_plan_bytes(70, 9)
    d = rel.rel_desc(2, 70, 2, 64, cnnk.BF16, 9)
    for plan in (torch.zeros(need - 1, dtype=torch.uint8), torch.zeros(need // 4 - 1), torch.zeros(rel.cnnk_rel_plan_bytes(69, 9), dtype=torch.uint8)):
        with pytest.raises(ValueError):
            rel.cnnk_rel_attention_fwd(d, A, A, plan, None, None, A, A)
        with pytest.raises(ValueError):
            rel.cnnk_rel_attention_bwd(d, A, A, A, A, plan, None, None, A, A, A, A, 1 << 40)


@pytest.mark.parametrize("B,T,heads,dh,dtype,buckets,units", [
    (64, 197, 12, 64, cnnk.BF16, 732, 3),           # 7 blocks, 2 parts of four wavefronts, two workgroups to a CU: 64 * 12 * 2 / 512
    (16, 4096, 3, 64, cnnk.BF16, 16129, 3),         # LDS for one workgroup to a CU, of eight wavefronts: 128 / 8 = 16 parts, 48 * 16 / 256
    (4, 4096, 12, 64, cnnk.BF16, 16129, 3),
    (7, 4096, 12, 64, cnnk.BF16, 16129, 6),         # 5.25
    (9, 2601, 12, 32, cnnk.BF16, 10201, 5),         # 58 KB: two to a CU, of four: 82 blocks, 21 parts, 108 * 21 / 512
    (8, 4096, 2, 16, cnnk.BF16, 15000, 1),          # 77 KB: 16 * 32 / 512
    (8, 4096, 2, 16, cnnk.F32, 16382, 1),           # 83 KB, one to a CU: 16 * 16 / 256
    (7, 2601, 10, 128, cnnk.BF16, 10201, 6),        # one workgroup of four to a CU: 70 * 21 / 256 = 5.7
    (9, 200, 12, 64, cnnk.F32, 16382, 1),           # seven blocks: one part of seven wavefronts, 108 / 256
])
def test_images_of_a_workgroup_fill_the_device_that_the_launch_meets(B, T, heads, dh, dtype, buckets, units):
    """A head's images lie in 1 + (B - 1) / units workgroups, rounded up, at most; the workspace has the sums of each, in blocks of 4 KB, and three floats for each row."""
    blocks, rows = (T + 31) // 32, (B * heads * 3 * ((T + 63) // 64 * 64) * 4 + 255) // 256 * 256
    need = rel.cnnk_rel_attention_workspace_bytes(rel.rel_desc(B, T, heads, dh, dtype, buckets))
    slot = heads * blocks * blocks * 4096
    assert (need - rows) % slot == 0 and (need - rows) // slot == 1 + (B - 1 + units - 1) // units


@pytest.mark.parametrize("B,T,heads,dh,buckets,slots", [
    (8, 4096, 12, 64, 16129, 2),                    # six images to a workgroup: 0-5 6-7 | 0-3 4-7 | 0-1 2-7
    (8, 2601, 12, 32, 10201, 2),                    # four: they divide the batch, a workgroup has one head
    (7, 2601, 12, 128, 10201, 1),                   # seven
    (6, 4096, 10, 64, 16129, 2),                    # four: 0-3 4-5 | 0-1 2-5, every workgroup starts at an even image
    (1, 4096, 12, 64, 16129, 1)])
def test_the_workspace_has_no_more_sums_than_a_head_has_workgroups(B, T, heads, dh, buckets, slots):
    blocks, rows = (T + 31) // 32, (B * heads * 3 * ((T + 63) // 64 * 64) * 4 + 255) // 256 * 256
    need = rel.cnnk_rel_attention_workspace_bytes(rel.rel_desc(B, T, heads, dh, cnnk.BF16, buckets))
    assert need == rows + slots * heads * blocks * blocks * 4096


def test_a_table_that_is_not_learned_needs_the_rows_only():
    d, rows = rel.rel_desc(3, 70, 2, 64, cnnk.BF16, 9), rel.cnnk_rel_attention_workspace_bytes(rel.rel_desc(3, 70, 2, 64, cnnk.BF16, 0))
    assert rel.cnnk_rel_attention_workspace_bytes(d) > rows
    call = lambda ws_bytes, dtable: rel.cnnk_rel_attention_bwd(d, A, A, A, A, A, None, None, A, A, dtable, A + 1, ws_bytes)
    for ws_bytes, dtable, status in ((rows - 1, None, 4), (rows, None, 3), (rows, A, 4)):        # with enough it is the workspace's address that is refused
        with pytest.raises(cnnk.CnnkError) as e:
            call(ws_bytes, dtable)
        assert e.value.status == status


def test_sums_of_too_many_columns_are_refused():
    """A slab of 256 columns past 2^31 - 1: with dbias there are 2^30 at most."""
    for C, ok in ((1 << 30, True), ((1 << 30) + 8, False), ((1 << 31) - 8, False)):
        d = rel.dropout_desc(1, C, cnnk.F32, 0.1)
        assert (rel.cnnk_dropout_workspace_bytes(d) == 4 * C) == ok and (ok or rel.cnnk_dropout_workspace_bytes(d) == 0)
        with pytest.raises(cnnk.CnnkError) as e:
            rel.cnnk_dropout_bwd(d, A, A, A, A, None, 0)
        assert e.value.status == (4 if ok else 3)
