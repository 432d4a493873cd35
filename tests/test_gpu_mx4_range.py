"""Decode attention on a 4-bit latent cache with values at the ends of their types' range, against the fp64 oracle.  Bars as in
test_gpu_mx4_decode.py."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as orc
from paper_2603_02188_amd import binding as mlra

from gpu_util import max_rel_err
from mx4_util import HostCache, queries, stored
from test_gpu_mx4_decode import _query_rest

pytestmark = pytest.mark.gpu

BF16_BAR = 1e-2 + 2.0 ** -8
SHAPES = [(4, 128, 128), (4, 128, 64), (1, 512, 64), (2, 64, 16)]      # the pipelined kernels, and the one for every shape


def _first_group_tiny(hc):
    """The first 32 channels of every row become +-{0, 0.5} 2^-125, the smallest that the format has."""
    hc.latent[..., :16] &= 0x99
    hc.scales[..., 0] = np.where(hc.scales[..., 0] == 255, 255, 2)
    for s, n in enumerate(hc.lens):
        for t in range(n):
            p, slot = hc.table[s, t // hc.page], t % hc.page
            hc.rows[s][t, :, :32] = orc.decode(hc.latent[p, :, slot, :16], hc.scales[p, :, slot, :1])


@pytest.mark.parametrize("with_lse", [False, True])
@pytest.mark.parametrize("n_blocks,d_cb,h", SHAPES)
def test_finite_queries_whose_sum_is_not(n_blocks, d_cb, h, with_lse):
    """32 query channels of 1e38 to 3e38 against cached channels of 1e-38: their magnitudes add up to an infinity, the scores are
    small."""
    lens, tau = [500, 65, 3], 1.0 / np.sqrt(192)
    hc = HostCache(lens, n_blocks, d_cb, 64, "bf16", 64, 31)
    _first_group_tiny(hc)
    rng = np.random.default_rng(32)
    (qa, qa64), (qr, qr64), (wv, wv64) = queries(rng, 3, 1, n_blocks, h, 1, d_cb, 64, 128, "bf16")
    qa64[..., :32] = rng.uniform(1e38, 3e38, qa64[..., :32].shape) * rng.choice([-1.0, 1.0], qa64[..., :32].shape)
    qa64[0, ..., 5] = 3.38e38                        # (close to the type's largest)
    qa, qa64 = stored(qa64, "bf16")
    lse = torch.empty((3, 1, n_blocks, h), device="cuda") if with_lse else None
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau, lse=lse).double().cpu().numpy()
    ref, ref_lse = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    err = max_rel_err(got, ref)
    print(f"       max rel err {err:.3e}", flush=True)
    assert err <= BF16_BAR
    if with_lse:                                     # (its bar: see _case there)
        size = max(1.0, float(np.abs(ref_lse).max()))
        bar = 5.0 * 2.0 ** -24 / np.sqrt(3.0) * np.sqrt(3.0 * d_cb + 6.0 * 64) * size + 1e-6
        rest = _query_rest(hc.rows, qa64, tau, 1) if d_cb in (128, 512) else 0.0
        assert (np.abs(lse.double().cpu().numpy() - ref_lse) <= bar + rest).all()


@pytest.mark.parametrize("with_lse", [False, True])
@pytest.mark.parametrize("n_blocks,d_cb,h,groups", [(4, 128, 128, 1), (4, 128, 64, 1), (2, 128, 40, 1), (4, 128, 128, 2), (3, 128, 100, 1),
                                                    (1, 512, 64, 1), (2, 64, 16, 1)])
def test_queries_that_are_not_finite_reach_their_heads_only(n_blocks, d_cb, h, groups, with_lse):
    """NaN and infinities in a query's latent or RoPE channels, of one block or all: every other head, and so every other sequence,
    is as without them to the last bit.  One chunk a sequence, and several."""
    hb = h // groups
    for lens in ([200, 130, 64], [2000, 130]):
        hc = HostCache(lens, n_blocks, d_cb, 64, "bf16", 64, 51)
        rng = np.random.default_rng(52)
        batch = len(lens)
        (qa, _), (qr, _), (wv, _) = queries(rng, batch, 1, n_blocks, hb, groups, d_cb, 64, 64, "bf16")
        lse = [torch.zeros((batch, 1, n_blocks, hb), device="cuda") for _ in range(2)]
        call = lambda a, r, l: mlra.mlra_mx4_decode_attn(hc.device(), a, r, wv, 0.07, groups=groups, lse=l if with_lse else None)
        want = call(qa, qr, lse[0])
        bad_a, bad_r, bad = qa.clone(), qr.clone(), torch.zeros((batch, h), dtype=torch.bool)
        for s, b, i, c, v in ((0, 0, 5, 40, "nan"), (1, n_blocks - 1, 7, 1, "inf"), (1, 0, hb - 1, d_cb - 1, "-inf")):
            bad_a[s, 0, b, i, c] = float(v)
            bad[s, b // (n_blocks // groups) * hb + i] = True
        for s, i, c, v in ((0, 3, 63, "-inf"), (0, h - 2, 0, "nan"), (1, 11, 31, "inf")):
            bad_r[s, 0, i, c] = float(v)
            bad[s, i] = True
        got = call(bad_a, bad_r, lse[1])
        assert got[:, 0][bad].isnan().all()
        assert torch.equal(got[:, 0][~bad], want[:, 0][~bad])
        if with_lse:                                 # (of a block; an infinite score makes an infinity or a NaN of it)
            same = ~(bad_a.isnan() | bad_a.isinf()).any(-1)[:, 0]                           # [batch][blocks][hb]
            rope = ~(bad_r.isnan() | bad_r.isinf()).any(-1)[:, 0].view(batch, groups, 1, hb)
            same = (same.view(batch, groups, -1, hb) & rope).view(batch, n_blocks, hb)
            assert torch.equal(lse[1][:, 0][same], lse[0][:, 0][same]) and not lse[1][:, 0][~same].isfinite().any()


@pytest.mark.parametrize("with_lse", [False, True])
@pytest.mark.parametrize("n_blocks,d_cb,h", SHAPES + [(3, 128, 100)])
def test_keys_of_minus_infinity_in_bf16(n_blocks, d_cb, h, with_lse):
    """Tokens whose score is -inf for every head, which have no weight: one among others, a tile, the last token, alone in its tile,
    and all of a chunk's but the first ones."""
    lens, tau = [500, 65, 129, 1200], 1.0 / np.sqrt(192)
    hc = HostCache(lens, n_blocks, d_cb, 64, "bf16", 64, 81)
    for s, tokens in enumerate(([7, 499], [64], list(range(64, 129)), list(range(70, 1200)))):
        for t in tokens:
            hc.rope[hc.table[s, t // 64], t % 64, 5] = hc.ropes[s][t, 5] = -np.inf
    rng = np.random.default_rng(82)
    (qa, qa64), (_, qr64), (wv, wv64) = queries(rng, 4, 1, n_blocks, h, 1, d_cb, 64, 128, "bf16")
    qr64[..., 5] = np.abs(qr64[..., 5]) + 0.1
    qr, qr64 = stored(qr64, "bf16")
    lse = torch.empty((4, 1, n_blocks, h), device="cuda") if with_lse else None
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau, lse=lse).double().cpu().numpy()
    ref, ref_lse = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    assert max_rel_err(got, ref) <= BF16_BAR
    if with_lse:
        assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 1e-2         # (exact to fp32: see the other tests' bars)


# fp32: RoPE numbers are the sum of three of bf16 there, whose products with an infinite one are NaN or infinities of either sign
F32 = [(4, 128, 64, 128), (2, 64, 32, 40), (1, 512, 64, 20), (2, 256, 128, 16), (2, 128, 128, 8)]


def _f32(n_blocks, d_cb, d_r, h, lens, seed):
    hc = HostCache(lens, n_blocks, d_cb, d_r, "f32", 64, seed)
    rng = np.random.default_rng([seed, 1])
    return hc, queries(rng, len(lens), 1, n_blocks, h, 1, d_cb, d_r, 32, "f32")


def _set_key(hc, s, t, channel, value):
    hc.rope[hc.table[s, t // hc.page], t % hc.page, channel] = hc.ropes[s][t, channel] = value


@pytest.mark.parametrize("n_blocks,d_cb,d_r,h", F32)
def test_a_score_of_minus_infinity_has_no_weight(n_blocks, d_cb, d_r, h):
    """Infinite keys whose products with every query are -inf: queries that are bf16 numbers (lower terms of zero), and others."""
    lens, tau = [200, 70], 0.1
    hc, ((qa, qa64), (_, qr64), (wv, wv64)) = _f32(n_blocks, d_cb, d_r, h, lens, 41)
    for s, t, channel, value in ((0, 10, 3, -np.inf), (0, 130, 3, -np.inf), (1, 0, 5, np.inf), (1, 69, 3, -np.inf)):
        _set_key(hc, s, t, channel, value)
    qr64[..., 3], qr64[..., 5] = np.abs(qr64[..., 3]) + 0.1, -np.abs(qr64[..., 5]) - 0.1
    qr64[..., ::2, 3], qr64[..., ::2, 5] = 1.0, -0.5
    qr, qr64 = stored(qr64, "f32")
    lse = torch.empty((2, 1, n_blocks, h), device="cuda")
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau, lse=lse).double().cpu().numpy()
    ref, ref_lse = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    err = max_rel_err(got, ref)
    print(f"       max rel err {err:.3e}", flush=True)
    assert err <= 1e-5
    # (scores of about 10: see the bar in test_gpu_mx4_decode.py)
    assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 1e-4


@pytest.mark.parametrize("n_blocks,d_cb,d_r,h", F32)
def test_infinite_and_nan_numbers_reach_their_heads_only(n_blocks, d_cb, d_r, h):
    """Heads whose product with an infinite key is +inf, and those whose query holds an infinity or a NaN, become NaN; the others'
    tokens with -inf do not count."""
    lens, tau = [200, 70], 0.1
    hc, ((qa, qa64), (_, qr64), (wv, wv64)) = _f32(n_blocks, d_cb, d_r, h, lens, 42)
    _set_key(hc, 0, 77, 2, np.inf)
    qr64[..., 2] = np.abs(qr64[..., 2]) + 0.1
    qr64[..., :h - 3, 2] *= -1.0                     # the last three heads see +inf in sequence 0
    qr64[1, 0, 1, 4], qr64[1, 0, 2, 4] = np.inf, np.nan
    qa64[1, 0, 0, 3, 9] = -np.inf
    (qr, qr64), (qa, qa64) = stored(qr64, "f32"), stored(qa64, "f32")
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau).double().cpu().numpy()
    bad = np.zeros((2, h), dtype=bool)
    bad[0, h - 3:], bad[1, 1:4] = True, True
    assert np.isnan(got[:, 0][bad]).all()
    with np.errstate(invalid="ignore"):
        ref, _ = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    assert np.isnan(ref[:, 0][bad]).all()
    assert max_rel_err(got[:, 0][~bad], ref[:, 0][~bad]) <= 1e-5


@pytest.mark.parametrize("n_blocks,d_cb,d_r,h", F32)
def test_the_largest_finite_numbers(n_blocks, d_cb, d_r, h):
    """Keys that round to an infinity in bf16, against queries of 1e-38."""
    lens, tau = [200, 70], 0.1
    hc, ((qa, qa64), (_, qr64), (wv, wv64)) = _f32(n_blocks, d_cb, d_r, h, lens, 43)
    rng = np.random.default_rng(44)
    for s, n in enumerate(lens):
        for t in range(n):
            _set_key(hc, s, t, 6, float(np.float32(rng.choice([-1.0, 1.0]) * rng.uniform(3.397e38, 3.4028e38))))
    # (bf16 numbers: lower terms of numbers this small would be denormal)
    qr64[..., 6] = stored(rng.uniform(1.2e-38, 6e-38, qr64[..., 6].shape), "bf16")[1]
    qr, qr64 = stored(qr64, "f32")
    hc.rope[np.isnan(hc.rope)] = 0.0                 # (spare slots: not to be converted with a warning)
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau).double().cpu().numpy()
    ref, _ = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    err = max_rel_err(got, ref)
    print(f"       max rel err {err:.3e}", flush=True)
    assert err <= 1e-5
