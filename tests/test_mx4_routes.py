"""Which kernels and which context split a decode call on a 4-bit latent cache takes: host logic, no GPU.  (The figures for the
number of compute units are those of a GPU with 256; without one the library plans for that.)"""
import ctypes
import random

import pytest
import torch

from paper_2603_02188_amd import binding as mlra

B, F = torch.bfloat16, torch.float32


def _info(batch=64, h=128, d_h=128, groups=1, n_blocks=4, d_cb=128, d_r=64, page=64, pages=128, dtype=B, out=None, lse=False, q_len=1):
    return mlra.mlra_mx4_decode_plan_info(batch, h, d_h, groups, n_blocks, d_cb, d_r, page, pages, dtype, out or dtype, lse, q_len)


@pytest.mark.parametrize("kw,kernel", [
    (dict(), "mfma"), (dict(lse=True), "mfma"), (dict(page=16), "mfma"), (dict(page=48), "mfma"), (dict(h=100, n_blocks=3), "mfma"),
    (dict(h=33, n_blocks=1), "mfma"), (dict(q_len=4), "mfma"), (dict(h=200), "mfma"),
    (dict(h=64), "mfma-paired"), (dict(h=8), "mfma-paired"), (dict(groups=2), "mfma-paired"), (dict(groups=2, q_len=3), "mfma-paired"),
    (dict(n_blocks=1, d_cb=512), "mfma-mla"), (dict(n_blocks=1, d_cb=512, h=16, lse=True), "mfma-mla"),
    (dict(n_blocks=1, d_cb=512, page=32, q_len=2), "mfma-mla"),
    # the kernel for every shape: fp32 in or out, other widths, pages that cut a tile, few heads on a block without a neighbour
    (dict(out=F), "mx4"), (dict(dtype=F), "mx4"), (dict(d_cb=64), "mx4"), (dict(d_cb=256, n_blocks=2), "mx4"), (dict(d_r=32), "mx4"),
    (dict(page=24), "mx4"), (dict(n_blocks=1, d_cb=512, page=48), "mx4"), (dict(n_blocks=2, d_cb=512), "mx4"),
    (dict(h=32, n_blocks=1), "mx4"), (dict(h=64, groups=2, n_blocks=2), "mx4"), (dict(h=64, n_blocks=3), "mfma"),
])
def test_kernels(kw, kernel):
    info = _info(**kw)
    assert info["kernel"] == kernel
    bf16 = kw.get("dtype", B) == B
    assert info["precise"] == (bf16 and (kw.get("out") == F or kw.get("lse", False)))
    assert info["merge_mfma"] == (bf16 and kw.get("out") != F)


@pytest.mark.parametrize("kw", [
    dict(batch=8, pages=512), dict(batch=16, n_blocks=1, pages=1024), dict(batch=4, groups=2, pages=2048),
    dict(batch=20, n_blocks=1, d_cb=512, pages=256), dict(batch=40, n_blocks=1, d_cb=512, h=70, pages=256),
    dict(batch=5, pages=256, q_len=3), dict(batch=5, groups=2, pages=256, q_len=2)])
def test_long_chunks_of_some_sequences_are_fitted(kw):
    for lse in (False, True):
        info = _info(lse=lse, **kw)
        assert info["fitted_from"] > 0 and info["fitted_from"] % 64 == 0 and not info["planned"] and info["merge_mfma"]
        assert info["chunk_slots"] * info["fitted_from"] >= 64 * kw["pages"]
    assert _info(out=F, **kw)["fitted_from"] == 0


@pytest.mark.parametrize("kw", [
    dict(batch=3, pages=512), dict(batch=65, pages=512), dict(batch=8, pages=64), dict(batch=64, groups=2), dict(batch=64),
    dict(batch=3, n_blocks=1, d_cb=512, pages=512), dict(batch=20, n_blocks=1, d_cb=512, pages=128, q_len=2),
    dict(batch=8, pages=512, d_h=64)])
def test_other_launches_are_not(kw):
    assert _info(**kw)["fitted_from"] == 0


def test_slots_hold_the_capacity_and_the_workspace_the_slots():
    rng = random.Random(3)
    for _ in range(2000):
        page, dtype, d_cb = rng.choice([1, 16, 48, 64, 100]), rng.choice([B, B, F]), rng.choice([32, 64, 128, 128, 256, 512])
        groups = rng.choice([1, 1, 2])
        kw = dict(batch=int(2 ** rng.uniform(0, 8)), h=groups * rng.choice([1, 16, 33, 64, 128]), groups=groups,
                  n_blocks=groups * rng.choice([1, 2]), d_cb=d_cb, page=page, pages=int(2 ** rng.uniform(0, 20)) // page + 1,
                  dtype=dtype, out=rng.choice([dtype, F]), lse=rng.random() < 0.5, q_len=rng.choice([1, 1, 2, 4]))
        info, cap, units = _info(**kw), kw["pages"] * page, kw["batch"] * kw["q_len"]
        assert info["chunk_slots"] * max(info["chunk_tokens"], info["fitted_from"]) >= cap, kw
        need = units * kw["n_blocks"] * info["chunk_slots"] * (kw["h"] // groups) * (d_cb + 2) * 4
        assert mlra.mlra_mx4_decode_workspace_bytes(kw["batch"], kw["q_len"], kw["h"], groups, kw["n_blocks"], d_cb, page,
                                                    kw["pages"]) >= need, kw


def test_errors():
    lib, info = mlra.load_library(), (ctypes.c_int32 * 7)()
    good = [4, 1, 128, 128, 1, 4, 128, 64, 64, 8, 0, 0, 0]
    assert lib.mlra_mx4_decode_plan_info(*good, info) == 0
    assert lib.mlra_mx4_decode_plan_info(*good, None) == -1
    for at, value, status in ((0, 0, -2), (1, 0, -2), (0, 65536, -2), (2, 0, -2), (3, 0, -2), (4, 3, -2), (5, 0, -2), (6, 48, -2), (6, 544, -2),
                              (7, 0, -2), (7, 129, -2), (8, 0, -2), (9, 0, -2), (9, 1 << 26, -2), (10, 2, -3), (11, -1, -3)):
        bad = list(good)
        bad[at] = value
        assert lib.mlra_mx4_decode_plan_info(*bad, info) == status, (at, value)
    assert lib.mlra_mx4_decode_plan_info(*[v if i != 2 else 127 for i, v in enumerate(good[:4])], 2, *good[5:], info) == -2
