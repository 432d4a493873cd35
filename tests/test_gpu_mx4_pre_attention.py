"""mlra_mx4_pre_attention: the queries are those of mlra_pre_attention, and the cache holds what mlra_mx4_append_kv makes of the
rows that mlra_pre_attention leaves in an fp32 cache, bit for bit; then a decode step on it."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle
from paper_2603_02188_amd import binding as mlra
from paper_2603_02188_amd import inputs as gen

from gpu_util import max_rel_err, to_device

pytestmark = pytest.mark.gpu


def _weights(wl, d, d_cq):
    pre, tag = gen.make_pre_inputs(wl, d, d_cq), wl.dtype
    W = mlra.PreWeights(*(to_device(x, tag) for x in (pre.w_dq, pre.w_dkv, pre.w_kr, pre.w_uq, pre.w_qr)), wl.h, pre.alpha_q,
                        pre.alpha_kv, to_device(pre.gain_q, tag), to_device(pre.gain_kv, tag), pre.eps, pre.rope_base)
    return W, to_device(pre.hidden, tag)


@pytest.mark.parametrize("dtype,n_blocks,d_cb,d_r,h,d_h", [("bf16", 4, 128, 64, 128, 128), ("f32", 4, 64, 32, 8, 64),
                                                           ("bf16", 1, 512, 64, 17, 128), ("bf16", 3, 96, 14, 6, 24)])
@pytest.mark.parametrize("rope_dtype", [torch.bfloat16, torch.float32])
def test_rows_and_queries(dtype, n_blocks, d_cb, d_r, h, d_h, rope_dtype):
    page, pages, batch = 16, 5, 7
    wl = gen.WORKLOADS["C1"].scaled(name="mx4-pre", batch=batch, n_blocks=n_blocks, d_cb=d_cb, d_r=d_r, h=h, d_h=d_h, dtype=dtype)
    W, hidden = _weights(wl, 256, 96)
    rng = np.random.default_rng(5)
    table = torch.from_numpy(rng.permutation(batch * pages).astype(np.int32).reshape(batch, pages)).cuda()
    pos = torch.tensor([0, 15, 16, 79, -1, 40, 63], dtype=torch.int32, device="cuda")
    wide = mlra.Cache(torch.zeros((batch * pages, n_blocks, page, d_cb), device="cuda"),
                      torch.zeros((batch * pages, page, d_r), device="cuda"), table, pos)
    qn, qr = mlra.mlra_pre_attention(wide, W, hidden, pos)
    caches = []
    for _ in range(2):
        c = mlra.Mx4Cache.empty(batch * pages, n_blocks, page, d_cb, d_r, table, pos, rope_dtype)
        c.latent.fill_(0x5A), c.scales.fill_(0x33), c.rope.fill_(7.0)
        caches.append(c)
    qn4, qr4 = mlra.mlra_mx4_pre_attention(caches[0], W, hidden, pos)
    assert torch.equal(qn, qn4) and torch.equal(qr, qr4)
    p = pos.clamp_min(0).long()
    at = table[torch.arange(batch, device="cuda"), p // page].long(), p % page
    rows = wide.latent[at[0], :, at[1]].reshape(batch, 1, n_blocks * d_cb).contiguous()
    mlra.mlra_mx4_append_kv(caches[1], rows, wide.rope[at[0], at[1]][:, None].contiguous(), pos)
    for name in ("latent", "scales", "rope"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name
    assert (caches[0].scales != 0x33).any() and (caches[0].scales == 0x33).any()


def test_captured_step_from_hidden_states():
    """Pre-attention, absorb and decode in a HIP graph, against the eager step, replayed over changing hidden states."""
    wl = gen.WORKLOADS["C3"].scaled(name="mx4-pre-step", batch=3)
    W, hidden = _weights(wl, 512, 128)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    lens, pos = torch.tensor([100, 1, 65], dtype=torch.int32, device="cuda"), torch.tensor([99, 0, 64], dtype=torch.int32, device="cuda")
    c = mlra.Mx4Cache.empty(6, 4, 64, 128, 64, table, lens)
    g = torch.Generator("cuda").manual_seed(1)
    mlra.mlra_mx4_append_kv(c, torch.randn((3, 128, 512), generator=g, device="cuda"), torch.randn((3, 128, 64), generator=g, device="cuda"),
                            torch.zeros(3, dtype=torch.int32, device="cuda"))
    w_uk = (torch.randn((4, 128, 128 * 128), generator=g, device="cuda") / 128 ** 0.5).bfloat16()
    w_uv = (torch.randn((4, 128, 128 * 128), generator=g, device="cuda") / 128 ** 0.5).bfloat16()
    qn, qr = torch.empty((3, 128, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 128, 64), dtype=torch.bfloat16, device="cuda")
    pre_ws = torch.empty(mlra.mlra_mx4_pre_attention_workspace_bytes(3, 512, 128, 4, 128, 64, 128, 128, torch.bfloat16),
                         dtype=torch.uint8, device="cuda")
    qa, ws = torch.empty((3, 4, 128, 128), dtype=torch.bfloat16, device="cuda"), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    out = torch.empty((3, 128, 128), dtype=torch.bfloat16, device="cuda")

    def step():
        mlra.mlra_mx4_pre_attention(c, W, hidden, pos, qn, qr, pre_ws)
        mlra.mlra_absorb_q(qn, w_uk, qa)
        mlra.mlra_mx4_decode_attn(c, qa, qr, w_uv, wl.tau, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        hidden.copy_(torch.randn(hidden.shape, generator=g, device="cuda"))
        step()
        want = out.clone()
        out.fill_(float("nan")), ws.fill_(255), pre_ws.fill_(255)
        c.latent[1, :, 35], c.latent[2, :, 0] = 0, 0                  # (two of the rows that the step writes)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
    rows, ropes = torch.zeros((3, 128, 512), device="cuda"), torch.zeros((3, 128, 64), device="cuda")
    mlra.mlra_mx4_read_kv(c, torch.zeros(3, dtype=torch.int32, device="cuda"), lens, rows, ropes)
    host = lambda t: t.double().cpu().numpy()
    ref, _ = mx4_oracle.attend([host(r).reshape(128, 4, 128) for r in rows], list(host(ropes)), lens.tolist(), host(qa)[:, None],
                               host(qr)[:, None], host(w_uv), wl.tau)
    assert max_rel_err(host(out), ref[:, 0]) <= 1e-2 + 2.0 ** -8
