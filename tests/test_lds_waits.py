"""Barriers that wait for nothing by themselves, and the LDS writes in front of them: the scan of the generated assembly on
assembly written by hand, and on that of the kernels that were built."""
import os


from paper_2603_02188_amd import build
from paper_2603_02188_amd.check_isa import find_unwaited_lds_writes

KERNEL = """
_ZN4mlra18decode_mfma_kernelILi8ELi0ELb1ELb0EEEv: ; @decode
\tds_read_b128 v[0:3], v4
%s
\ts_barrier
\tds_read_b32 v1, v2
\ts_endpgm
_ZN4mlra5otherEv:
\tds_write_b32 v1, v2
\ts_barrier
\ts_endpgm
"""
READ, WRITE = "\tds_read_b32 v5, v6", "\tds_write_b128 v0, v[4:7] offset:64"


def _found(*body):
    return len(find_unwaited_lds_writes(KERNEL % "\n".join(body), "decode_mfma_kernel"))


def test_a_write_in_front_of_a_barrier_is_reported():
    assert _found(WRITE) == 1
    assert _found(WRITE, "\ts_waitcnt vmcnt(0)") == 1
    assert _found(WRITE, "\ts_waitcnt lgkmcnt(0)", "\tds_write_b32 v1, v2") == 1
    assert _found("\tds_add_u32 v1, v2") == 1
    assert _found() == _found(READ, "\tds_bpermute_b32 v1, v2, v3") == 0                # nothing is written
    assert _found(WRITE, "\ts_waitcnt vmcnt(3) lgkmcnt(0)") == 0
    assert _found(WRITE, "\t;;#ASMSTART", "\ts_waitcnt lgkmcnt(0)", "\t;;#ASMEND") == 0
    # the last n operations may be under way behind lgkmcnt(n)
    assert _found(WRITE, READ, "\ts_waitcnt lgkmcnt(2)") == 1
    assert _found(WRITE, READ, READ, "\ts_waitcnt lgkmcnt(2)") == 0


def test_every_path_to_the_barrier_counts():
    branch = ["\ts_cbranch_scc1 .LBB0_1", "\ts_waitcnt lgkmcnt(0)", ".LBB0_1:"]
    assert _found(WRITE, *branch) == 1                                                # one way round the wait
    assert _found("\ts_cbranch_scc1 .LBB0_1", WRITE, ".LBB0_1:") == 1                 # a write on one of two ways
    loop = [".LBB0_2:", "\ts_barrier", READ, WRITE, "\ts_cbranch_scc0 .LBB0_2", "\ts_waitcnt lgkmcnt(0)"]
    assert _found(*loop) == 1                                                         # the barrier of the next round
    assert _found(WRITE, "\ts_branch .LBB0_3", "\ts_barrier", ".LBB0_3:", "\ts_waitcnt lgkmcnt(0)") == 0


def _built(name):
    path = os.path.join(build.PKG, "_build", name + ".s")
    if not os.path.exists(path):
        build.build()
    return open(path).read()


def test_decode_kernels_on_a_cache_in_4_bits_wait_for_their_writes():
    """The step that widens a tile ends with writes; what is stored behind the barrier of the merge lies in the same place."""
    text = _built("decode_mx4")
    assert len([ln for ln in text.splitlines() if "; @" in ln and "ELb1ELb" in ln]) == 4      # two forms, with and without lse
    assert find_unwaited_lds_writes(text, "decode_mfma_kernel") == []


def test_other_kernels_wait_for_their_writes():
    """(The 256-channel form's zeros for half of the RoPE reads among them.)"""
    for name in ("decode_mfma", "decode_mx4", "mla_mfma", "mx4_mfma", "gqa_mfma", "proj_mfma", "pre_attn", "f32_mfma", "f32_proj"):
        assert find_unwaited_lds_writes(_built(name), build.LDS_WAITS) == [], name
