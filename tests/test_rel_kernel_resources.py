"""What the compiler made of the attention kernels with a relative position bias: registers that leave the wavefronts their launch bounds ask for, and what spills."""
import re

from test_kernel_resources import kernels  # noqa: F401

SPILLS = {"rel_mfma_fwd_kernel<unsigned short, 64, true, true>": 8, "rel_mfma_dkv_kernel<float, 64, true, true, false>": 12}      # bytes of scratch a lane, at most


def test_walks_keep_their_registers(kernels):  # noqa: F811
    """512 registers of a SIMD: forward in bf16 with heads of up to 64 four wavefronts, dq three, dk and dv two, with heads of 128 one."""
    count = {"fwd": 0, "dq": 0, "dkv": 0}
    for name, (registers, spilled, scratch) in kernels.items():
        m = re.match(r"rel_mfma_(fwd|dq|dkv)_kernel<(unsigned short|float), (\d+),", name)
        if not m:
            continue
        walk, bf16, dh = m[1], m[2] != "float", int(m[3])
        count[walk] += 1
        most = {"fwd": 128 if bf16 and dh <= 64 else 256, "dq": (168 if bf16 else 256) if dh <= 64 else 512, "dkv": 256 if dh <= 64 else 512}[walk]
        assert registers <= most, (name, registers)
        assert scratch <= SPILLS.get(name, 0), (name, spilled, scratch)
    assert count == {"fwd": 32, "dq": 32, "dkv": 44}      # 2 types x 4 head sizes x bias x dropout; with runs 2 types x 3 x dropout besides


def test_the_others_spill_nothing(kernels):  # noqa: F811
    names = [n for n in kernels if re.match(r"(rel_runs|rel_buckets|dropout|dropout_sum|plan_\w+|buckets_grid|rng_advance)_kernel", n)]
    assert len(names) == 15 and all(kernels[n][1:] == (0, 0) for n in names), names
