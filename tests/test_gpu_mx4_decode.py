"""Decode attention on a 4-bit latent cache against the fp64 oracle.

The cached values are exact, what is rounded is what a cache of the calls' type rounds, and the bars are those of its tests:
1e-2 (bf16) and 1e-5 (fp32) of the largest output.  bf16: the queries (with the softmax scale), the probabilities, a chunk's
row and the merged values are rounded by up to 2^-8 each; these errors are independent, 2^-8 / sqrt(3) in the mean, and sum up
over the same products as the values do, so that four of them give 4.5e-3 of the root mean square output and five times that,
2.3e-2, is less than 1e-2 of the largest one, which is three to four times as large.  fp32: sums of up to 10^4 terms of 2^-24."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as orc
from paper_2603_02188_amd import binding as mlra

from gpu_util import max_rel_err
from mx4_util import DT, HostCache, queries, stored

pytestmark = pytest.mark.gpu

# (fp32 outputs of a bf16 call are exact to fp32: cache, queries and weights are exact in bf16 as they are)
BAR = {"bf16": 1e-2, "f32": 1e-5}


def _check(lens, out=None, **kw):
    """bf16 calls with a bf16 output, on the bf16 kernels, without and with the log-sum-exp, and with both in fp32."""
    if out is None and kw.get("dtype", "bf16") == "bf16":
        _case(lens, out="bf16", with_lse=False, **kw)
        if kw.get("d_cb", 128) in (128, 512):
            _case(lens, out="bf16", **kw)
    _case(lens, out=out or "f32", **kw)


def _query_rest(rows, qa, tau, groups):
    """How far the scores of every query are off at most.  Units: the largest channel of a group of 32 lies in 3.75 .. 7.5.
    Three E2M3 numbers of units 1, 2^-4 and 2^-9 hold a bf16 number (8 bits) from 2^-5 on, whose steps are 2^-12 or more, the
    smallest that the third one has; smaller ones, below 2^-6 of the largest at any rate, are off by half of that, 2^-13, which
    is 2^-14.9 of the largest."""
    batch, q_len, n_blocks, hb, d_cb = qa.shape
    g = np.abs(qa).reshape(*qa.shape[:-1], d_cb // 32, 32)
    top = g.max(-1, keepdims=True)
    off = np.where(g < top / 64.0, top * 2.0 ** -14.9, 0.0).reshape(qa.shape)
    rest = np.zeros((batch, q_len, n_blocks, hb))
    for s in range(batch):
        for b in range(n_blocks):
            if len(rows[s]):
                c = np.abs(np.asarray(rows[s], dtype=np.float64).reshape(len(rows[s]), n_blocks, d_cb)[:, b])
                rest[s, :, b] = tau * (off[s, :, b] @ c.T).max(-1)
    return rest


def _case(lens, n_blocks=4, d_cb=128, d_r=64, h=128, d_h=128, groups=1, q_len=1, page=64, dtype="bf16", out="f32", gated=False,
          out_scale=1.0, max_pages=None, seed=1, single=False, with_lse=True):
    print(f"[case] lens={lens} nb={n_blocks} d_cb={d_cb} d_r={d_r} h={h} g={groups} q={q_len} page={page} {dtype}", flush=True)
    hc = HostCache(lens, n_blocks, d_cb, d_r, dtype, page, seed, max_pages)
    rng = np.random.default_rng([seed, 9])
    batch, hb, tau = len(lens), h // groups, 1.0 / np.sqrt(d_h + d_r)
    (qa, qa64), (qr, qr64), (wv, wv64) = queries(rng, batch, q_len, n_blocks, hb, groups, d_cb, d_r, d_h, dtype)
    gate, gate64 = stored(1.0 / (1.0 + np.exp(-rng.standard_normal((batch, q_len, h, d_h)))), dtype) if gated else (None, None)
    lse = torch.full((batch, q_len, n_blocks, hb), float("nan"), device="cuda")
    squeeze = (lambda t: None if t is None else t[:, 0]) if single else (lambda t: t)
    args = (hc.device(), squeeze(qa), squeeze(qr), wv, tau, out_scale)
    kw = dict(groups=groups, gate=squeeze(gate), out_dtype=DT[out])
    got = mlra.mlra_mx4_decode_attn(*args, lse=squeeze(lse) if with_lse else None, **kw)
    again = mlra.mlra_mx4_decode_attn(*args, lse=squeeze(torch.empty_like(lse)) if with_lse else None, **kw)
    torch.cuda.synchronize()
    assert torch.equal(got, again)                                # deterministic
    ref, ref_lse = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau, out_scale, groups, gate64)
    got = got.double().cpu().numpy().reshape(ref.shape)
    err = max_rel_err(got, ref)
    print(f"       max rel err {err:.3e} (bar {BAR[dtype]:g})", flush=True)
    assert err <= (BAR["bf16"] + 2.0 ** -8 if out == "bf16" else BAR["f32"])
    lse = lse.double().cpu().numpy()
    empty = np.isneginf(ref_lse)
    if with_lse:
        assert np.isneginf(lse[empty]).all()
    if with_lse and not empty.all():
        # a score is the sum of 3 d_cb + 6 d_r products (fp32: three terms a query, six a RoPE product), each addition off by up to
        # 2^-24 of a partial sum, which is about as large as the scores that count, and those are about the log-sum-exp:
        # independent errors of 2^-24 / sqrt(3) of it in the mean, five times the root of their number (8e-5 for 192 channels
        # and scores of 16).  The log-sum-exp of a bf16 call is exact to fp32 as well, but for what three E2M3 numbers leave of a
        # query beside a bf16 output (see _query_rest); a log-sum-exp moves by no more than the score that moves most.
        size = max(1.0, float(np.abs(ref_lse[~empty]).max()))
        bar = 5.0 * 2.0 ** -24 / np.sqrt(3.0) * np.sqrt(3.0 * d_cb + 6.0 * d_r) * size + 1e-6
        rest = _query_rest(hc.rows, qa64, tau, groups) if dtype == out == "bf16" and d_cb in (128, 512) else 0.0
        assert (np.abs(lse[~empty] - ref_lse[~empty]) <= (bar + rest * np.ones(lse.shape))[~empty]).all()
    for s, n in enumerate(lens):
        for j in range(q_len):
            if n - (q_len - 1 - j) <= 0:
                assert np.all(got[s, j] == 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [64, 16, 1, 7, 48, 80, 256])
def test_lengths_and_pages(dtype, page):
    _check([0, 1, 2, 63, 64, 65, 129, 300], page=page, dtype=dtype, h=32, n_blocks=2, d_h=32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_cb,d_r,n_blocks", [(32, 32, 1), (64, 32, 4), (96, 7, 2), (128, 64, 4), (160, 128, 1), (256, 64, 2),
                                               (288, 33, 1), (512, 64, 1), (512, 128, 2), (128, 1, 3)])
def test_channels(dtype, d_cb, d_r, n_blocks):
    _check([100, 5, 333], n_blocks=n_blocks, d_cb=d_cb, d_r=d_r, h=20, d_h=48, dtype=dtype, page=32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h", [1, 3, 16, 17, 31, 33, 64, 65, 127, 128, 200])
def test_heads(dtype, h):
    _check([70, 200], n_blocks=2, h=h, d_h=32 if h != 128 else 128, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups,n_blocks,d_cb,h", [(2, 4, 128, 128), (2, 2, 256, 128), (2, 4, 64, 6), (2, 2, 128, 2)])
def test_head_groups(dtype, groups, n_blocks, d_cb, h):
    _check([0, 300, 64, 1], groups=groups, n_blocks=n_blocks, d_cb=d_cb, h=h, dtype=dtype)


@pytest.mark.parametrize("dtype,h,groups,n_blocks,d_cb", [("bf16", 128, 1, 4, 128), ("f32", 128, 1, 4, 128), ("bf16", 64, 2, 2, 128),
                                                          ("bf16", 128, 1, 1, 512), ("f32", 12, 1, 2, 64)])
@pytest.mark.parametrize("q_len", [2, 3, 5])
def test_query_tokens(dtype, h, groups, n_blocks, d_cb, q_len):
    _check([0, 1, 2, 3, 4, 65, 400], q_len=q_len, h=h, groups=groups, n_blocks=n_blocks, d_cb=d_cb, dtype=dtype, gated=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gate_scale_and_output_types(dtype, out):
    _check([130, 64, 7], dtype=dtype, out=out, gated=True, out_scale=0.5, single=True)
    _check([130, 64, 7], dtype=dtype, out=out, h=40, d_h=20, gated=True, out_scale=2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,n_blocks,h", [([5000], 4, 128), ([3000, 1, 0, 2900], 1, 64), ([4097, 130], 2, 16)])
def test_long_contexts_in_chunks(dtype, lens, n_blocks, h):
    _check(lens, n_blocks=n_blocks, h=h, dtype=dtype, page=128)


# whole sequences as one chunk each: the pipelined kernels at every distance from the end of their prologue, stages and ring,
# last tiles full, of one token and of one short of full
@pytest.mark.parametrize("n_blocks,h,groups,page", [(2, 128, 1, 64), (4, 64, 1, 16), (4, 128, 2, 32), (1, 130, 1, 128), (1, 70, 1, 48), (2, 64, 1, 112)])
def test_tiles_of_the_pipelined_kernel(n_blocks, h, groups, page):
    lens = [64 * t + e for t in range(1, 14) for e in (0, 1, 63)] + [0, 1, 2, 3]
    lens += [5] * (260 // n_blocks)                       # (enough sequences for a chunk each)
    _check(lens, n_blocks=n_blocks, h=h, groups=groups, page=page, d_h=32)


@pytest.mark.parametrize("h,page", [(64, 32), (100, 64), (128, 96)])
def test_tiles_of_the_mla_kernel(h, page):
    lens = [32 * t + e for t in range(1, 12) for e in (0, 1, 31)] + [0, 1, 2, 700]
    lens += [5] * 260
    _check(lens, n_blocks=1, d_cb=512, h=h, page=page, d_h=32)


@pytest.mark.parametrize("n_blocks,d_cb,h", [(1, 512, 128), (4, 128, 128), (4, 128, 64), (1, 128, 128)])
def test_ragged_batches_in_chunks(n_blocks, d_cb, h):
    rng = np.random.default_rng(4)
    _check(rng.integers(0, 2500, size=20).tolist(), n_blocks=n_blocks, d_cb=d_cb, h=h, d_h=128)
    _check([9000, 100, 6500], n_blocks=n_blocks, d_cb=d_cb, h=h, d_h=128, max_pages=400)


def test_many_sequences():
    rng = np.random.default_rng(3)
    _check(rng.integers(0, 200, size=70).tolist(), n_blocks=2, h=64, d_h=32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_table_much_wider_than_the_lengths(dtype):
    _check([70, 3, 300], max_pages=5000, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_any_size(dtype):
    """One token far above the others (queries a thousand times as large), and a first token far below the rest."""
    lens, tau = [500, 65], 1.0 / np.sqrt(192)
    hc = HostCache(lens, 2, 128, 64, dtype, 64, 8)
    rng = np.random.default_rng(10)
    (qa, qa64), (qr, qr64), (wv, wv64) = queries(rng, 2, 1, 2, 32, 1, 128, 64, 128, dtype)
    big, big64 = stored(qa64 * 1024.0, dtype)
    got = mlra.mlra_mx4_decode_attn(hc.device(), big, qr, wv, tau).double().cpu().numpy()
    ref, _ = orc.attend(hc.rows, hc.ropes, lens, big64, qr64, wv64, tau)
    # the weights are those of the few largest scores; a score of 10^3 is off by up to 2^-8 (2^-24) of the root sum of
    # squares of its terms, which can move weight between tokens that are nearer to each other than that: fp32 1e-4 (a score
    # moved by 10^3 2^-24), bf16 not compared but finite and inside the values' range
    assert np.isfinite(got).all()
    if dtype == "f32":
        assert max_rel_err(got, ref) <= 1e-3
    else:
        assert np.abs(got).max() <= 4.0 * np.abs(ref).max()


# one query channel far above its group's others, against cached channels that are small there: what the others contribute is
# then most of a score, and has to keep its precision.  (Bars as above: 1e-2 of the largest output.  32 channels with the scale's
# power of two cut to 1/64 in one of them: scores stay as they are.)
@pytest.mark.parametrize("n_blocks,d_cb,h,factor", [(4, 128, 128, 12.0), (4, 128, 128, 64.0), (4, 128, 64, 200.0), (1, 512, 128, 64.0),
                                                    (1, 512, 20, 200.0), (2, 64, 16, 64.0)])
def test_query_channels_that_stand_out(n_blocks, d_cb, h, factor):
    lens, tau = [500, 65, 3], 1.0 / np.sqrt(192)
    hc = HostCache(lens, n_blocks, d_cb, 64, "bf16", 64, 21)
    hc.latent[:, :, :, 3::16] &= 0xF0                            # (the channel of the large query holds zeros)
    hc.rows = [np.where(np.arange(d_cb) % 32 == 6, 0.0, r) for r in hc.rows]
    rng = np.random.default_rng(22)
    (qa, qa64), (qr, qr64), (wv, wv64) = queries(rng, 3, 1, n_blocks, h, 1, d_cb, 64, 128, "bf16")
    qa64[..., 6::32] *= factor
    qa, qa64 = stored(qa64, "bf16")
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau).double().cpu().numpy()
    ref, _ = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    err = max_rel_err(got, ref)
    print(f"       max rel err {err:.3e}", flush=True)
    assert err <= 1e-2 + 2.0 ** -8


@pytest.mark.parametrize("n_blocks,d_cb,h", [(4, 128, 128), (4, 128, 64), (1, 512, 64)])
def test_nan_and_infinite_queries_and_rows_of_the_pipelined_kernels(n_blocks, d_cb, h):
    """A NaN or an infinity in a query reaches its head, one in a row its sequence, and neither another sequence.  (The row sums
    of heads 16 apart come from one matrix product over both, as on the wider caches, so that these two go together.)"""
    lens = [200, 130, 64]
    hc = HostCache(lens, n_blocks, d_cb, 64, "bf16", 64, 23)
    rng = np.random.default_rng(24)
    (qa, qa64), (qr, _), (wv, _) = queries(rng, 3, 1, n_blocks, h, 1, d_cb, 64, 128, "bf16")
    want = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, 0.07)
    bad = qa.clone()
    bad[0, 0, 0, 5, 40], bad[1, 0, 0, 7, 1] = float("nan"), float("inf")
    got = mlra.mlra_mx4_decode_attn(hc.device(), bad, qr, wv, 0.07)
    assert got[0, 0, 5].isnan().all() and got[1, 0, 7].isnan().all() and torch.equal(got[2], want[2])
    others = [i for i in range(h) if i % 32 not in (5, 21, 7, 23)]
    assert torch.equal(got[:, :, others], want[:, :, others])
    hc.scales[hc.table[1, 2], 0, 1, 2] = 255                     # the last row of sequence 1
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, 0.07)
    assert got[1].isnan().all() and torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("n_blocks,d_cb,dtype", [(4, 128, "bf16"), (1, 512, "bf16"), (4, 128, "f32")])
def test_pages_beyond_4_gib(n_blocks, d_cb, dtype):
    """The same rows in the first pages of a pool and in pages whose codes lie behind 2^32 bytes."""
    page, pages = 64, (1 << 32) // (64 * 256) + 40
    lens = torch.tensor([150, 64], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(30)
    (qa, _), (qr, _), (wv, _) = queries(rng, 2, 1, n_blocks, 64, 1, d_cb, 64, 32, dtype)
    g = torch.Generator("cuda").manual_seed(2)
    rows, rope = torch.randn((2, 150, 512), generator=g, device="cuda"), torch.randn((2, 150, 64), generator=g, device="cuda")
    cache = mlra.Mx4Cache.empty(pages, n_blocks, page, d_cb, 64, torch.zeros((2, 3), dtype=torch.int32, device="cuda"), lens,
                                torch.bfloat16 if dtype == "bf16" else torch.float32)
    outs = []
    for first in (0, pages - 6):
        cache.page_table = torch.arange(first, first + 6, dtype=torch.int32, device="cuda").view(2, 3)
        mlra.mlra_mx4_append_kv(cache, rows, rope, torch.zeros_like(lens), lens)
        outs.append(mlra.mlra_mx4_decode_attn(cache, qa, qr, wv, 0.07))
        cache.latent[:6], cache.scales[:6] = 0, 255
    assert outs[0].isfinite().all() and torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_rows_reach_their_sequence_only(dtype):
    lens = [100, 80]
    hc = HostCache(lens, 2, 64, 32, dtype, 32, 9)
    p, slot = hc.table[0, 50 // 32], 50 % 32
    hc.scales[p, 1, slot, 0] = 255
    rng = np.random.default_rng(11)
    (qa, _), (qr, _), (wv, _) = queries(rng, 2, 1, 2, 16, 1, 64, 32, 32, dtype)
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, 0.1)
    assert got[0].isnan().all() and got[1].isfinite().all()


def test_unaligned_queries():
    hc = HostCache([130, 64], 2, 64, 32, "bf16", 64, 14)
    rng = np.random.default_rng(15)
    (qa, _), (qr, _), (wv, _) = queries(rng, 2, 1, 2, 16, 1, 64, 32, 32, "bf16")
    want = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, 0.1)

    def shift(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:] = t.flatten()
        return flat[1:].view(t.shape)

    assert torch.equal(mlra.mlra_mx4_decode_attn(hc.device(), shift(qa), shift(qr), shift(wv), 0.1), want)


@pytest.mark.parametrize("which", ["scales", "q_abs", "q_rope", "w_uv"])
@pytest.mark.parametrize("n_blocks,d_cb,h", [(4, 128, 128), (4, 128, 64), (1, 512, 64)])
def test_tensors_that_start_anywhere(n_blocks, d_cb, h, which):
    """Each of scales, queries and weights one element behind an aligned address, at the pipelined kernels' shapes."""
    lens, tau = [130, 64, 0], 0.07
    hc = HostCache(lens, n_blocks, d_cb, 64, "bf16", 64, 14)
    rng = np.random.default_rng(15)
    (qa, qa64), (qr, qr64), (wv, wv64) = queries(rng, 3, 1, n_blocks, h, 1, d_cb, 64, 128, "bf16")
    cache, t = hc.device(), {"q_abs": qa, "q_rope": qr, "w_uv": wv}

    def shift(x):
        flat = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")
        flat[1:] = x.flatten()
        return flat[1:].view(x.shape)

    if which == "scales":
        cache.scales = shift(cache.scales)
    else:
        t[which] = shift(t[which])
    got = mlra.mlra_mx4_decode_attn(cache, t["q_abs"], t["q_rope"], t["w_uv"], tau).double().cpu().numpy()
    ref, _ = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    assert max_rel_err(got, ref) <= 1e-2 + 2.0 ** -8
