"""Rows quantised into a 4-bit latent cache and read back, against the oracle, bit for bit: the scale is a power of two, so
that codes and values have no rounding of their own to allow for."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as orc
from paper_2603_02188_amd import binding as mlra
from paper_2603_02188_amd import inputs as gen

from mx4_util import DT, HostCache, stored

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(rng, shape):
    """Normal rows with groups of other sizes, a group of zeros and numbers on the ties."""
    x = rng.standard_normal(shape).astype(np.float32)
    g = x.reshape(-1, 32)
    g *= np.exp2(rng.integers(-3, 4, size=(len(g), 1))).astype(np.float32)
    g[1 % len(g)] = 0.0
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], dtype=np.float32)
    g[2 % len(g)] = np.concatenate((ties, -ties, ties * 0.5, -ties * 0.125)) * 2.0 ** -7
    return x


def _expected(hc, positions, lens, n_rows, rows, ropes, dtype):
    """The pools after the call."""
    latent, scales, rope = hc.latent.copy(), hc.scales.copy(), hc.rope.copy()
    for s, first in enumerate(positions):
        n = n_rows if lens is None else min(lens[s], n_rows)
        for j in range(n if first >= 0 else 0):
            t = first + j
            if t >= hc.table.shape[1] * hc.page or not 0 <= hc.table[s, t // hc.page] < len(latent):
                continue
            p, slot = hc.table[s, t // hc.page], t % hc.page
            codes, byte = orc.encode(rows[s, j].reshape(hc.n_blocks, hc.d_cb))
            latent[p, :, slot], scales[p, :, slot] = codes, byte
            rope[p, slot] = gen.to_f64(gen.to_storage(ropes[s, j].astype(np.float32), dtype), dtype)
    return latent, scales, rope


def _append(hc, positions, lens, n_rows, src, seed, rows=None, offset=0):
    rng = np.random.default_rng([seed, 7])
    batch, d_c = len(positions), hc.n_blocks * hc.d_cb
    rows = _rows(rng, (batch, n_rows, d_c)) if rows is None else rows
    c_dev, c_val = stored(rows, src)
    k_dev, k_val = stored(rng.standard_normal((batch, n_rows, hc.d_r)), src)
    if offset:                                   # rows that do not start on 16 bytes
        flat = torch.empty(c_dev.numel() + offset, dtype=c_dev.dtype, device="cuda")
        flat[offset:] = c_dev.flatten()
        c_dev = flat[offset:].view(c_dev.shape)
    cache = hc.device()
    mlra.mlra_mx4_append_kv(cache, c_dev, k_dev, _i32(positions), None if lens is None else _i32(lens))
    torch.cuda.synchronize()
    latent, scales, rope = _expected(hc, positions, lens, n_rows, c_val, k_val, hc.dtype)
    assert np.array_equal(cache.scales.cpu().numpy(), scales)
    assert np.array_equal(cache.latent.cpu().numpy(), latent)
    assert np.array_equal(cache.rope.double().cpu().numpy(), rope, equal_nan=True)
    return cache


@pytest.mark.parametrize("src", ["bf16", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_blocks,d_cb,d_r,page", [(4, 128, 64, 64), (1, 32, 1, 1), (3, 96, 7, 5), (1, 512, 64, 16),
                                                    (5, 160, 130, 33)])
def test_append(src, dtype, n_blocks, d_cb, d_r, page):
    # a skipped sequence, one new token, a piece over several pages, none of the rows, all of them
    hc = HostCache([40, 1, 21, 9, 23], n_blocks, d_cb, d_r, dtype, page, 1)
    _append(hc, [-1, 0, 2, 3, 0], [5, 1, 19, 0, 23], 23, src, 11)


@pytest.mark.parametrize("src", ["bf16", "f32"])
def test_append_one_token_each_and_unaligned_rows(src):
    hc = HostCache([70, 64, 1, 129], 4, 64, 32, "bf16", 64, 2)
    _append(hc, [69, 63, 0, 128], None, 1, src, 12)
    _append(hc, [60, 0, 0, 100], [9, 20, 1, 17], 20, src, 13, offset=1)


def test_append_skips_slots_beyond_the_capacity_and_bad_page_ids():
    hc = HostCache([32, 32, 32], 2, 32, 8, "bf16", 8, 3)
    hc.table[1, 1], hc.table[2, 0] = -1, len(hc.latent)          # (the checks are the kernel's own)
    _append(hc, [28, 6, 0], [9, 12, 12], 12, "f32", 14)
    _append(hc, [2 ** 31 - 1, 32, 31], [12, 12, 12], 12, "f32", 15)


def test_append_extremes():
    """NaN and infinities, the largest and smallest numbers, denormals, every binade, -0."""
    n = 300
    rows = np.zeros((1, n, 32), dtype=np.float32)
    rng = np.random.default_rng(5)
    for i in range(254):
        rows[0, i] = (rng.uniform(0.05, 2.0, 32) * rng.choice([-1, 1], 32) * 2.0 ** (i - 126.0)).astype(np.float32)
    rows[0, 254:260] = rng.standard_normal((6, 32))
    rows[0, 254, 3], rows[0, 255, 31], rows[0, 256, 0] = np.nan, np.inf, -np.inf
    rows[0, 260] = np.finfo(np.float32).max
    rows[0, 261, 5] = np.finfo(np.float32).smallest_subnormal
    rows[0, 262, :2] = [2.0 ** -126, 2.0 ** -127]
    rows[0, 263] = -0.0
    rows[0, 264, :3] = [1.75, np.nextafter(np.float32(1.75), np.float32(0)), 0.4375]
    rows[0, 265, :3] = [np.nextafter(np.float32(1.75), np.float32(0)), 0.3, -1.1]
    hc = HostCache([n], 1, 32, 8, "f32", 64, 4)
    cache = _append(hc, [0], None, n, "f32", 16, rows=rows)
    for out in (torch.bfloat16, torch.float32):                  # every value is exact in either type
        c, k = torch.zeros((1, n, 32), dtype=out, device="cuda"), torch.zeros((1, n, 8), dtype=out, device="cuda")
        mlra.mlra_mx4_read_kv(cache, _i32([0]), None, c, k)
        got, want = c[0].double().cpu().numpy(), orc.decode(*orc.encode(rows[0]))
        assert np.array_equal(got, want, equal_nan=True)
        assert np.isnan(got[254:257]).all() and np.isfinite(got[260]).all()


@pytest.mark.parametrize("dtype,dst", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("n_blocks,d_cb,d_r,page,offset", [(4, 128, 64, 64, 0), (3, 96, 7, 5, 1), (1, 512, 64, 16, 0),
                                                           (5, 160, 130, 33, 3)])
def test_read(dtype, dst, n_blocks, d_cb, d_r, page, offset):
    """Any piece of the sequences; rows that are not asked for, or have no slot, keep what they held."""
    hc = HostCache([40, 1, 0, 19, 23], n_blocks, d_cb, d_r, dtype, page, 6)
    d_c, n_rows, first, lens = n_blocks * d_cb, 24, [17, 0, 0, -1, 0], [23, 1, 0, 19, 30]
    flat = torch.full((5 * n_rows * d_c + offset,), 7.0, dtype=DT[dst], device="cuda")
    c = flat[offset:].view(5, n_rows, d_c)
    k = torch.full((5, n_rows, d_r), 7.0, dtype=DT[dst], device="cuda")
    mlra.mlra_mx4_read_kv(hc.device(), _i32(first), _i32(lens), c, k)
    want_c, want_k = np.full((5, n_rows, d_c), 7.0), np.full((5, n_rows, d_r), 7.0)
    for s in (0, 1, 4):
        m = min(lens[s], n_rows)
        rows, rope = np.full((m, d_c), np.nan), np.full((m, d_r), np.nan)
        have = min(m, hc.lens[s] - first[s])
        rows[:have] = hc.rows[s][first[s]:first[s] + have].reshape(have, d_c)
        rope[:have] = hc.ropes[s][first[s]:first[s] + have]
        if have < m:                              # (slot 23 of the last one is a page's unowned slot, or has no page)
            t = first[s] + have
            if t // page >= hc.table.shape[1]:
                rows[have:], rope[have:] = 7.0, 7.0
        want_c[s, :m], want_k[s, :m] = rows, rope
    assert np.array_equal(c.double().cpu().numpy(), want_c, equal_nan=True)
    assert np.array_equal(k.double().cpu().numpy(), gen.to_f64(gen.to_storage(want_k.astype(np.float32), dst), dst), equal_nan=True)


def test_rows_of_pages_beyond_4_gib():
    """Element offsets past 2^32 in the pools (pages of 2^20 tokens)."""
    page, nb, d_cb = 1 << 20, 8, 1024
    table = _i32([[1]])
    cache = mlra.Mx4Cache.empty(2, nb, page, d_cb, 8, table, _i32([page]))
    assert cache.latent.numel() > 1 << 32
    rows = torch.randn((1, 3, nb * d_cb), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    rope = torch.randn((1, 3, 8), device="cuda")
    mlra.mlra_mx4_append_kv(cache, rows, rope, _i32([page - 3]))
    c, k = torch.zeros((1, 2, nb * d_cb), device="cuda"), torch.zeros((1, 2, 8), device="cuda")
    mlra.mlra_mx4_read_kv(cache, _i32([page - 2]), None, c, k)
    want = orc.decode(*orc.encode(rows[0, 1:].double().cpu().numpy()))
    assert np.array_equal(c[0].double().cpu().numpy(), want)
    assert torch.equal(k[0], rope[0, 1:].bfloat16().float())
