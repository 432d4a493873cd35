"""Head groups of an odd number of 128-channel blocks: the kernel that takes two neighbouring blocks per workgroup must not
run there, since its two blocks would belong to different groups, which have RoPE queries of their own."""
import numpy as np
import pytest
import torch

from oracle import mlra_oracle as orc
from oracle import mx4_oracle
from paper_2603_02188_amd import binding as mlra
from paper_2603_02188_amd import inputs as gen

from gpu_util import device_cache, device_queries_weights, max_rel_err, oracle_views

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_blocks,h", [(2, 128), (6, 128), (2, 2), (6, 40)])
def test_odd_number_of_blocks_in_a_group(n_blocks, h):
    wl = gen.WORKLOADS["M2"].scaled(name="odd-groups", batch=3, n_blocks=n_blocks, h=h, n_min=70, n_max=300)
    inp = gen.make_decode_inputs(wl, poison=True)
    q_nope, q_rope, w_uk, w_uv = device_queries_weights(inp)
    q_abs = mlra.mlra2_absorb_q(q_nope, w_uk)
    out = mlra.mlra2_decode_attn(device_cache(inp), q_abs, q_rope, w_uv, wl.tau, out_dtype=torch.float32)
    v = oracle_views(inp)
    rows = [orc.gather_sequence(v["latent_pool"], v["rope_pool"], v["page_table"][s], int(v["seq_lens"][s])) for s in range(3)]
    latent = [c.reshape(len(c), n_blocks, wl.d_cb) for c, _ in rows]
    ref, _ = mx4_oracle.attend(latent, [k for _, k in rows], v["seq_lens"], q_abs.double().cpu().numpy()[:, None],
                               v["q_rope"][:, None], v["w_uv"], wl.tau, groups=2)
    assert max_rel_err(out.double().cpu().numpy(), ref[:, 0]) <= 1e-2
