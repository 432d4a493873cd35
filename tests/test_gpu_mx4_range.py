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
