"""The 4-bit latent cache without a GPU: the oracle's encoding against values worked out by hand, and what the entry points
refuse on the host."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as orc
from paper_2603_02188_amd import binding as mlra


@pytest.mark.parametrize("top,e", [(1.0, -2), (1.74, -2), (1.75, -1), (2.0, -1), (6.0, 0), (7.0, 1), (0.0, -125),
                                   (2.0 ** -126, -125), (2.0 ** -123, -125), (2.0 ** -122, -124), (2.0 ** 127, 125),
                                   (1.9 * 2.0 ** 127, 125)])
def test_oracle_scale(top, e):
    assert orc.scale_exponent(top) == e


def test_oracle_codes_ties_and_saturation():
    x = np.zeros(32)
    #        0.25 0.75 1.25 1.75 2.5 3.5 5.0: ties go to 0 1 1 2 2 4 4; then neighbours, signs, the largest
    x[:16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.26, -0.25, -0.75, -2.6, 4.9, 5.1, -6.0, 6.9, -0.0]
    codes, byte = orc.encode_group(x)
    assert byte == 127
    assert codes[:16].tolist() == [0, 2, 2, 4, 4, 6, 6, 1, 8, 8 + 2, 8 + 5, 6, 7, 15, 7, 8]
    packed, scales = orc.encode(x[None])
    want = [0, 1, 1, 2, 2, 4, 4, 0.5, 0, -1, -3, 4, 6, -6, 6, 0] + [0] * 16
    assert orc.decode(packed, scales)[0].tolist() == want
    assert orc.encode_group(np.where(np.arange(32) == 3, np.inf, x))[1] == 255
    assert np.isnan(orc.decode(*orc.encode(np.where(np.arange(32) == 3, np.nan, x)[None]))).all()


def test_oracle_attention_closed_forms():
    """One token: its own value row whatever the queries; equal scores: the mean; hidden tokens do not count."""
    rng = np.random.default_rng(0)
    w = np.eye(32)[None].repeat(2, 0)                                   # one head, d_h = d_cb: out = z_0 + z_1
    c, k = rng.standard_normal((5, 2, 32)), rng.standard_normal((5, 8))
    q, r = rng.standard_normal((1, 2, 2, 1, 32)), rng.standard_normal((1, 2, 1, 8))
    out, lse = orc.attend([c[:2]], [k[:2]], [2], q, r, w, 0.3)
    np.testing.assert_allclose(out[0, 0, 0], c[0].sum(0), rtol=1e-13)   # the first of two queries sees one token
    np.testing.assert_allclose(lse[0, 0, 1, 0], 0.3 * (q[0, 0, 1, 0] @ c[0, 1] + r[0, 0, 0] @ k[0]), rtol=1e-12)
    out, lse = orc.attend([c], [k], [5], 0 * q, 0 * r, w, 0.3, gate=np.full((1, 2, 1, 32), 0.5))
    np.testing.assert_allclose(out[0, 1, 0], 0.5 * c.mean(0).sum(0), rtol=1e-13)
    np.testing.assert_allclose(lse[0, 1], np.log(5.0))
    out, lse = orc.attend([c], [k], [1], q, r, w, 0.3)
    assert np.all(out[0, 0] == 0) and np.isneginf(lse[0, 0]).all() and np.isfinite(lse[0, 1]).all()


def _struct(**kw):
    d = dict(latent=256, scales=256, rope=256, page_table=256, seq_lens=256, num_pages=4, page_size=64, max_pages_per_seq=4,
             n_blocks=4, d_cb=64, d_r=32, dtype=1)
    d.update(kw)
    return mlra._Mx4CacheStruct(*d.values())


_ONE, _NULL = 256, None         # (never dereferenced: the checks come first)


def _decode(cs, batch=1, q_len=1, h=8, d_h=64, groups=1, q=_ONE, w=_ONE, out=_ONE, out_dtype=1, ws=_ONE, ws_bytes=1 << 40):
    return mlra.load_library().mlra_mx4_decode_attn(cs and ctypes.byref(cs), batch, q_len, h, d_h, groups, q, _ONE, w, _NULL,
                                                    0.1, 1.0, out, out_dtype, _NULL, ws, ws_bytes, _NULL)


_BAD_CACHE = [(dict(latent=0), -1), (dict(scales=0), -1), (dict(rope=0), -1), (dict(page_table=0), -1), (dict(dtype=2), -3),
              (dict(d_cb=0), -2), (dict(d_cb=48), -2), (dict(d_r=0), -2), (dict(n_blocks=0), -2), (dict(page_size=0), -2),
              (dict(num_pages=0), -2), (dict(max_pages_per_seq=0), -2), (dict(n_blocks=256), -2), (dict(latent=264), -2),
              (dict(rope=258), -2), (dict(max_pages_per_seq=1 << 25), -2)]


@pytest.mark.parametrize("kw,status", _BAD_CACHE)
def test_bad_caches_are_refused(kw, status):
    lib, cs = mlra.load_library(), _struct(**kw)
    assert lib.mlra_mx4_append_kv(ctypes.byref(cs), 1, 1, _ONE, _ONE, 1, _ONE, _NULL, _NULL) == status
    assert lib.mlra_mx4_read_kv(ctypes.byref(cs), 1, 1, _ONE, _NULL, _ONE, _ONE, 1, _NULL) == status
    assert _decode(cs) == status


def test_bad_rows_calls_are_refused():
    lib, cs = mlra.load_library(), _struct()
    for fn in (lambda b, n, c, k, t, p: lib.mlra_mx4_append_kv(ctypes.byref(cs), b, n, c, k, t, p, _NULL, _NULL),
               lambda b, n, c, k, t, p: lib.mlra_mx4_read_kv(ctypes.byref(cs), b, n, p, _NULL, c, k, t, _NULL)):
        assert fn(1, 1, _NULL, _ONE, 1, _ONE) == fn(1, 1, _ONE, _NULL, 1, _ONE) == fn(1, 1, _ONE, _ONE, 1, _NULL) == -1
        assert fn(1, 1, _ONE, _ONE, 2, _ONE) == fn(1, 1, _ONE, _ONE, -1, _ONE) == -3
        assert fn(0, 1, _ONE, _ONE, 1, _ONE) == fn(65536, 1, _ONE, _ONE, 1, _ONE) == fn(1, 0, _ONE, _ONE, 1, _ONE) == -2
        assert fn(1, -1, _ONE, _ONE, 1, _ONE) == fn(1, (1 << 26) + 1, _ONE, _ONE, 1, _ONE) == -2
    assert lib.mlra_mx4_append_kv(None, 1, 1, _ONE, _ONE, 1, _ONE, _NULL, _NULL) == -1
    assert lib.mlra_mx4_read_kv(None, 1, 1, _ONE, _NULL, _ONE, _ONE, 1, _NULL) == -1


def test_bad_decode_calls_are_refused():
    cs = _struct()
    assert _decode(None) == _decode(cs, q=_NULL) == _decode(cs, w=_NULL) == _decode(cs, out=_NULL) == -1
    assert _decode(_struct(seq_lens=0)) == -1
    assert _decode(cs, out_dtype=2) == -3
    for kw in (dict(batch=0), dict(q_len=0), dict(h=0), dict(d_h=0), dict(groups=0), dict(groups=3), dict(h=7, groups=2),
               dict(batch=40000, q_len=2), dict(h=70000)):
        assert _decode(cs, **kw) == -2, kw
    assert _decode(_struct(n_blocks=3), groups=2) == _decode(_struct(d_cb=544)) == _decode(_struct(d_r=129)) == -2
    need = mlra.mlra_mx4_decode_workspace_bytes(1, 1, 8, 1, 4, 64, 64, 4)
    assert need > 0 and need % 256 == 0
    assert _decode(cs, ws=_NULL) == _decode(cs, ws_bytes=need - 1) == _decode(cs, ws=264) == -4


def test_workspace_sizes():
    size = mlra.mlra_mx4_decode_workspace_bytes
    assert size(64, 1, 128, 1, 4, 128, 64, 128) >= 64 * 4 * 128 * 130 * 4
    assert size(2, 4, 128, 1, 4, 128, 64, 100) >= size(8, 1, 128, 1, 4, 128, 64, 100) + 8 * 4 + 800 * 4
    assert size(2, 1, 128, 2, 4, 128, 64, 100) < size(2, 1, 128, 1, 4, 128, 64, 100) * 2
    for bad in ((0, 1, 8, 1, 4, 64, 64, 4), (1, 1, 8, 1, 4, 63, 64, 4), (1, 1, 7, 2, 4, 64, 64, 4), (1, 1, 8, 4, 4, 64, 64, 4),
                (1, 1, 8, 1, 1, 544, 64, 4), (1, 1, 8, 1, 4, 64, 64, 1 << 25)):
        assert size(*bad) == 0, bad


def test_binding_checks_shapes():
    table, lens = torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    c = mlra.Mx4Cache.empty(7, 4, 16, 64, 32, table, lens)
    assert c.latent.shape == (7, 4, 16, 32) and c.scales.shape == (7, 4, 16, 2) and c.rope.dtype == torch.bfloat16
    assert c.max_seq_len == 48
    with pytest.raises(ValueError):                              # host tensors
        c.struct()
    for bad in (dict(scales=c.scales[:, :, :, :1]), dict(rope=c.rope[:, :8]), dict(latent=c.latent.view(torch.int8)),
                dict(page_table=table.long())):
        args = dict(latent=c.latent, scales=c.scales, rope=c.rope, page_table=table, seq_lens=lens)
        args.update(bad)
        with pytest.raises((AssertionError, ValueError)):
            mlra.Mx4Cache(**args).struct()


def test_bad_pre_attention_calls_are_refused():
    lib, cs = mlra.load_library(), _struct()
    pw = lambda **kw: mlra._PreWeightsStruct(*{**dict(w_dq=256, w_dkv=256, w_kr=256, w_uq=256, w_qr=256, gain_q=None, gain_kv=None, d=96,
                                                      d_cq=40, h=8, d_h=64, dtype=1, alpha_q=1.0, alpha_kv=1.0, eps=1e-6,
                                                      rope_base=1e4), **kw}.values())

    def call(c, w, batch=2, hidden=_ONE, pos=_ONE, ws=_ONE, ws_bytes=1 << 30):
        return lib.mlra_mx4_pre_attention(c and ctypes.byref(c), w and ctypes.byref(w), batch, hidden, pos, _ONE, _ONE, ws, ws_bytes,
                                          _NULL)

    assert call(None, pw()) == call(cs, None) == call(cs, pw(), hidden=_NULL) == call(cs, pw(), pos=_NULL) == -1
    assert call(cs, pw(w_dq=None)) == -1
    assert call(cs, pw(dtype=9)) == -3
    assert call(cs, pw(), batch=0) == call(cs, pw(d=0)) == call(cs, pw(d_h=63)) == call(_struct(d_r=31), pw()) == -2
    assert call(cs, pw(), ws=_NULL) == call(cs, pw(), ws_bytes=16) == call(cs, pw(), ws=264) == -4
    size = mlra.mlra_mx4_pre_attention_workspace_bytes
    assert size(2, 96, 40, 4, 64, 32, 8, 64, torch.float32) >= 2 * (256 + 32) * 4
    assert size(2, 96, 40, 4, 48, 32, 8, 64, torch.float32) == size(0, 96, 40, 4, 64, 32, 8, 64, torch.float32) == 0
    for kw, status in _BAD_CACHE:
        assert call(_struct(**kw), pw()) == status, kw
