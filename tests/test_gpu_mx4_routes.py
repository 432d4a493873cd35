"""Decode attention on a 4-bit latent cache, form by form: each test asserts that the plan of its call is the one it is about, and
compares with the fp64 oracle as test_gpu_mx4_decode.py does (whose bars hold here as well)."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as orc
from paper_2603_02188_amd import binding as mlra

from gpu_util import max_rel_err
from mx4_util import DT, HostCache, queries, stored
from test_gpu_mx4_decode import _case

pytestmark = pytest.mark.gpu


def _info(lens, n_blocks=4, d_cb=128, h=128, d_h=128, groups=1, q_len=1, page=64, max_pages=None, out="bf16", with_lse=False):
    pages = max_pages or max(-(-n // page) for n in lens)
    return mlra.mlra_mx4_decode_plan_info(len(lens), h, d_h, groups, n_blocks, d_cb, 64, page, pages, torch.bfloat16, DT[out],
                                          with_lse, q_len)


_RAGGED = [9000, 100, 6500, 0, 2049, 2048, 4096, 1]


@pytest.mark.parametrize("with_lse", [False, True])
@pytest.mark.parametrize("kernel,kw", [
    ("mfma", dict(lens=_RAGGED, max_pages=512)),
    ("mfma", dict(lens=[5000] * 8, max_pages=512)),
    ("mfma", dict(lens=_RAGGED * 2, max_pages=1024, n_blocks=1)),
    ("mfma-paired", dict(lens=[9000, 3000, 0, 2100], max_pages=2048, groups=2)),
    ("mfma-mla", dict(lens=[4000, 1281, 1280, 1279, 0, 1, 700, 33] + [150] * 11 + [2600], max_pages=256, n_blocks=1, d_cb=512)),
    ("mfma-mla", dict(lens=[3000, 1300, 40, 0] * 10, max_pages=256, n_blocks=1, d_cb=512, h=70)),
    ("mfma", dict(lens=[5000, 0, 2, 1857, 1856], max_pages=256, q_len=3)),
    ("mfma-paired", dict(lens=[5000, 1, 1409, 1408, 300], max_pages=256, groups=2, q_len=2)),
])
def test_fitted_chunks(kernel, kw, with_lse):
    info = _info(with_lse=with_lse, **kw)
    assert info["kernel"] == kernel and info["fitted_from"] > 0 and max(kw["lens"]) > info["fitted_from"]
    _case(out="bf16", with_lse=with_lse, **kw)


@pytest.mark.parametrize("d_cb,d_r,n_blocks,h,page", [(32, 32, 1, 20, 32), (64, 64, 4, 128, 64), (64, 32, 2, 12, 16), (96, 7, 2, 20, 32),
                                                      (128, 32, 2, 64, 64), (160, 128, 1, 20, 48), (256, 64, 2, 64, 64), (288, 33, 1, 20, 32),
                                                      (512, 64, 1, 40, 48), (512, 128, 2, 20, 64)])
def test_log_sum_exp_beside_a_bf16_output_of_other_shapes(d_cb, d_r, n_blocks, h, page):
    """The kernel for every shape, probabilities of two terms."""
    lens = [100, 5, 333, 0]
    info = mlra.mlra_mx4_decode_plan_info(4, h, 128, 1, n_blocks, d_cb, d_r, page, -(-333 // page), torch.bfloat16, torch.bfloat16, True)
    assert info["kernel"] == "mx4" and info["precise"] and info["merge_mfma"]
    # (queries are bf16 as they come there: nothing is left of them, see _query_rest)
    hc = HostCache(lens, n_blocks, d_cb, d_r, "bf16", page, 61)
    rng = np.random.default_rng(62)
    (qa, qa64), (qr, qr64), (wv, wv64) = queries(rng, 4, 1, n_blocks, h, 1, d_cb, d_r, 128, "bf16")
    lse, tau = torch.empty((4, 1, n_blocks, h), device="cuda"), 1.0 / np.sqrt(192)
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau, lse=lse).double().cpu().numpy()
    ref, ref_lse = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau)
    assert max_rel_err(got, ref) <= 1e-2 + 2.0 ** -8 and not got[3].any()
    lse, some = lse.double().cpu().numpy(), ~np.isneginf(ref_lse)
    size = max(1.0, float(np.abs(ref_lse[some]).max()))
    bar = 5.0 * 2.0 ** -24 / np.sqrt(3.0) * np.sqrt(3.0 * d_cb + 6.0 * d_r) * size + 1e-6
    assert np.abs(lse[some] - ref_lse[some]).max() <= bar and np.isneginf(lse[~some]).all()


@pytest.mark.parametrize("n_blocks,d_cb,h,groups", [(4, 128, 128, 1), (4, 128, 64, 1), (4, 128, 128, 2), (1, 512, 64, 1)])
def test_query_channels_that_hardly_stand_out(n_blocks, d_cb, h, groups):
    """One channel of every group just below eight times the mean magnitude, against cached channels of zero there: the most that
    two rows are asked to hold.  They leave up to 2^-9 of that channel of every other one (2^-8 where the second is cut off, which a
    largest of 7.5 units and more is needed for), 2^-9 / sqrt(3) in the mean; a score is off by tau times the root sum of squares of
    that times its row, and the output's largest value, three to four times as large as its mean, by five times as much over 3.5,
    beside the bar's other roundings."""
    lens, tau, hb = [500, 65, 3], 1.0 / np.sqrt(192), h // groups
    info = _info(lens, n_blocks, d_cb, h, groups=groups)
    assert info["kernel"] != "mx4" and not info["precise"]
    hc = HostCache(lens, n_blocks, d_cb, 64, "bf16", 64, 71)
    hc.latent[:, :, :, 3::16] &= 0xF0
    hc.rows = [np.where(np.arange(d_cb) % 32 == 6, 0.0, r) for r in hc.rows]
    rng = np.random.default_rng(72)
    (qa, qa64), (qr, qr64), (wv, wv64) = queries(rng, 3, 1, n_blocks, hb, groups, d_cb, 64, 128, "bf16")
    groups_of = qa64.reshape(-1, 32)
    groups_of[:, 6] = 0.98 * np.abs(np.delete(groups_of, 6, axis=1)).sum(1) / 3.0 * rng.choice([-1.0, 1.0], len(groups_of))
    qa, qa64 = stored(qa64, "bf16")
    size = np.abs(qa64.reshape(-1, 32))
    top = size.max(1)
    assert (4.0 * top < 0.995 * size.sum(1)).all() and (4.0 * top > 0.95 * size.sum(1)).all()
    got = mlra.mlra_mx4_decode_attn(hc.device(), qa, qr, wv, tau, groups=groups).double().cpu().numpy()
    ref, _ = orc.attend(hc.rows, hc.ropes, lens, qa64, qr64, wv64, tau, 1.0, groups)
    off = 2.0 ** -9 / np.sqrt(3.0) * top.mean() * tau * max(np.sqrt((r ** 2).sum(-1)).max() for r in hc.rows)
    err = max_rel_err(got, ref)
    print(f"       max rel err {err:.3e}, scores off by {off:.2e}", flush=True)
    assert err <= 1e-2 + 2.0 ** -8 + 5.0 * off / 3.5


@pytest.mark.parametrize("kw", [dict(n_blocks=4, d_cb=128, h=128, batch=8, pages=512), dict(n_blocks=1, d_cb=512, h=128, batch=20, pages=256),
                                dict(n_blocks=4, d_cb=128, h=128, batch=5, pages=256, q_len=3), dict(n_blocks=4, d_cb=128, h=64, batch=100, pages=32)])
@pytest.mark.parametrize("with_lse", [False, True])
def test_captured_calls_with_other_lengths(kw, with_lse):
    """A decode call in a HIP graph, whose chunks follow the lengths on the device: replays with other lengths (longer and shorter than
    at the capture, zero among them) equal the eager call, with eager work in between."""
    n_blocks, d_cb, h, batch, pages, q_len = (kw.get(k, 1) for k in ("n_blocks", "d_cb", "h", "batch", "pages", "q_len"))
    info = mlra.mlra_mx4_decode_plan_info(batch, h, 128, 1, n_blocks, d_cb, 64, 64, pages, torch.bfloat16, torch.bfloat16, with_lse, q_len)
    assert info["kernel"] != "mx4" and (info["fitted_from"] > 0) == (batch <= 64)
    rng = np.random.default_rng(91)
    (qa, _), (qr, _), (wv, _) = queries(rng, batch, q_len, n_blocks, h, 1, d_cb, 64, 128, "bf16")
    g = torch.Generator("cuda").manual_seed(92)
    table = torch.randint(0, 64, (batch, pages), generator=g, device="cuda", dtype=torch.int32)       # (shared pages)
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    cache = mlra.Mx4Cache.empty(64, n_blocks, 64, d_cb, 64, table, lens)
    cache.latent.random_(0, 256, generator=g)
    cache.scales.random_(123, 129, generator=g)
    cache.rope.normal_(generator=g)
    ws = torch.empty(mlra.mlra_mx4_decode_workspace_bytes(batch, q_len, h, 1, n_blocks, d_cb, 64, pages), dtype=torch.uint8, device="cuda")
    out = torch.empty((batch, q_len, h, 128), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((batch, q_len, n_blocks, h), device="cuda") if with_lse else None
    call = lambda o, l, w: mlra.mlra_mx4_decode_attn(cache, qa, qr, wv, 0.07, out=o, lse=l, workspace=w)
    lens.fill_(1000)
    call(out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, ws)
    for i, most in enumerate((64 * pages, 100, 5000, 64 * pages, 1)):
        lens.copy_(torch.from_numpy(rng.integers(0, min(most, 64 * pages) + 1, batch).astype(np.int32)))
        lens[i % batch] = min(most, 64 * pages)
        want_lse = torch.empty_like(lse) if with_lse else None
        want = call(torch.empty_like(out), want_lse, torch.empty_like(ws))
        out.fill_(9.0)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and out.isfinite().all() and (not with_lse or torch.equal(lse, want_lse)), i
