"""The operators of the 4-bit cache together, as a serving loop runs them: prompts written in pieces, steps of append, absorb
and decode, eager, captured and on other streams."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as orc
from paper_2603_02188_amd import binding as mlra

from gpu_util import max_rel_err
from mx4_util import stored

pytestmark = pytest.mark.gpu


class _Loop:
    """Three prompts, written in pieces of up to 50 tokens, then decode steps."""

    def __init__(self, dtype, groups=1):
        self.rng = np.random.default_rng([17, groups])
        self.nb, self.d_cb, self.d_r, self.h, self.d_h, self.groups, self.dtype = 4, 128, 64, 128, 128, groups, dtype
        self.hb, self.tau, self.lens = self.h // groups, 1.0 / np.sqrt(192), [130, 1, 63]
        pages = 4
        table = torch.from_numpy(self.rng.permutation(3 * pages).astype(np.int32).reshape(3, pages)).cuda()
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.cache = mlra.Mx4Cache.empty(3 * pages, self.nb, 64, self.d_cb, self.d_r, table,
                                         torch.tensor(self.lens, dtype=torch.int32, device="cuda"), dt)
        for t in (self.cache.latent, self.cache.scales):
            t.fill_(255)                                             # NaN wherever nothing is written
        self.cache.rope.fill_(float("nan"))
        self.rows = [np.zeros((0, self.nb, self.d_cb)) for _ in range(3)]
        self.ropes = [np.zeros((0, self.d_r)) for _ in range(3)]
        self.w_uk, self.w_uk64 = stored(self.rng.standard_normal((self.nb, self.d_cb, self.hb * self.d_h)) / np.sqrt(self.d_cb), dtype)
        self.w_uv, self.w_uv64 = stored(self.rng.standard_normal((self.nb, self.d_cb, self.hb * self.d_h)) / np.sqrt(self.d_cb), dtype)
        for at in range(0, 130, 50):
            left = [max(0, min(50, n - at)) for n in self.lens]
            c, k = self.new_rows(50, left)
            mlra.mlra_mx4_append_kv(self.cache, c, k, torch.full((3,), at, dtype=torch.int32, device="cuda"),
                                    torch.tensor(left, dtype=torch.int32, device="cuda"))

    def new_rows(self, n, lens):
        c, c64 = stored(self.rng.standard_normal((3, n, self.nb * self.d_cb)), self.dtype)
        k, k64 = stored(self.rng.standard_normal((3, n, self.d_r)), self.dtype)
        for s, m in enumerate(lens):
            got = orc.decode(*orc.encode(c64[s, :m].reshape(m, self.nb, self.d_cb)))
            self.rows[s], self.ropes[s] = np.concatenate((self.rows[s], got)), np.concatenate((self.ropes[s], k64[s, :m]))
        return c, k

    def queries(self):
        qn, self.qn64 = stored(self.rng.standard_normal((3, self.h, self.d_h)), self.dtype)
        qr, self.qr64 = stored(self.rng.standard_normal((3, self.h, self.d_r)), self.dtype)
        return qn, qr

    def reference(self):
        w = self.w_uk64.reshape(self.nb, self.d_cb, self.hb, self.d_h)
        q_abs = np.zeros((3, 1, self.nb, self.hb, self.d_cb))
        for b in range(self.nb):
            first = b // (self.nb // self.groups) * self.hb
            q_abs[:, 0, b] = np.einsum("sip,cip->sic", self.qn64[:, first:first + self.hb], w[b])
        lens = [len(r) for r in self.rows]
        return orc.attend(self.rows, self.ropes, lens, q_abs, self.qr64[:, None], self.w_uv64, self.tau, 1.0, self.groups)[0][:, 0]


@pytest.mark.parametrize("dtype,groups", [("bf16", 1), ("bf16", 2), ("f32", 1)])
@pytest.mark.parametrize("folded", [False, True])
def test_prompts_and_steps(dtype, groups, folded):
    loop = _Loop(dtype, groups)
    absorb = mlra.mlra2_absorb_q if groups == 2 else mlra.mlra_absorb_q
    absorb_folded = mlra.mlra2_absorb_q_folded if groups == 2 else mlra.mlra_absorb_q_folded
    for _ in range(3):
        c, k = loop.new_rows(1, [1, 1, 1])
        qn, qr = loop.queries()
        mlra.mlra_mx4_append_kv(loop.cache, c, k, loop.cache.seq_lens)        # the slot behind the last token
        loop.cache.seq_lens += 1
        if folded:
            qa, qr = absorb_folded(qn, loop.w_uk, qr, loop.tau)
        else:
            qa = absorb(qn, loop.w_uk)
        out = mlra.mlra_mx4_decode_attn(loop.cache, qa, qr, loop.w_uv, mlra.SCALE_FOLDED if folded else loop.tau,
                                        groups=groups)
        assert max_rel_err(out.double().cpu().numpy(), loop.reference()) <= (1e-2 + 2.0 ** -8 if dtype == "bf16" else 1e-5)
    # the prompts come back as what they stand for
    n = max(len(r) for r in loop.rows)
    c, k = (torch.zeros((3, n, w), dtype=loop.cache.rope.dtype, device="cuda") for w in (512, 64))
    mlra.mlra_mx4_read_kv(loop.cache, torch.zeros(3, dtype=torch.int32, device="cuda"), loop.cache.seq_lens, c, k)
    for s, r in enumerate(loop.rows):
        assert np.array_equal(c[s, :len(r)].double().cpu().numpy(), r.reshape(len(r), 512)) and not c[s, len(r):].any()
        assert np.array_equal(k[s, :len(r)].double().cpu().numpy(), loop.ropes[s])


@pytest.mark.parametrize("dtype,q_len", [("bf16", 1), ("bf16", 3), ("f32", 1)])
def test_captured_steps(dtype, q_len):
    """A step in a HIP graph: every replay with new rows, queries and lengths equals the eager step."""
    loop = _Loop(dtype)
    dt, c = loop.cache.rope.dtype, loop.cache
    mk = lambda *shape: torch.randn(shape, device="cuda").to(dt)
    c_new, k_new, qn, qr = mk(3, q_len, 512), mk(3, q_len, 64), mk(3 * q_len, 128, 128), mk(3, q_len, 128, 64)
    qa = torch.empty((3 * q_len, 4, 128, 128), dtype=dt, device="cuda")
    pos, out = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.empty((3, q_len, 128, 128), dtype=dt, device="cuda")
    c_out, k_out = torch.zeros((3, 256, 512), dtype=dt, device="cuda"), torch.zeros((3, 256, 64), dtype=dt, device="cuda")
    zero = torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(mlra.mlra_mx4_decode_workspace_bytes(3, q_len, 128, 1, 4, 128, 64, 4), dtype=torch.uint8, device="cuda")

    def step():
        mlra.mlra_mx4_append_kv(c, c_new, k_new, pos)
        mlra.mlra_absorb_q(qn, loop.w_uk, qa)
        mlra.mlra_mx4_decode_attn(c, qa.view(3, q_len, 4, 128, 128), qr, loop.w_uv, loop.tau, out=out, workspace=ws)
        mlra.mlra_mx4_read_kv(c, zero, c.seq_lens, c_out, k_out)

    start = [t.clone() for t in (c.latent, c.scales, c.rope, c.seq_lens)]

    def restore(i):
        for t, v in zip((c.latent, c.scales, c.rope), start):
            t.copy_(v)
        pos.copy_(start[3] + i)
        c.seq_lens.copy_(start[3] + i + q_len)
        g = torch.Generator("cuda").manual_seed(i)
        for t in (c_new, k_new, qn, qr):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        for t in (out, c_out, k_out):
            t.zero_()

    graph = torch.cuda.CUDAGraph()
    restore(0)
    step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        restore(i)
        if i:                                                        # (rows between the prompt and the new ones)
            fill = torch.randn((3, i, 512), generator=torch.Generator("cuda").manual_seed(99), device="cuda").to(dt)
            mlra.mlra_mx4_append_kv(c, fill, fill[..., :64].contiguous(), start[3])
            torch.cuda.synchronize()
        state = [t.clone() for t in (c.latent, c.scales, c.rope)]
        step()
        want = [t.clone() for t in (out, c_out, k_out, c.latent, c.scales, c.rope)]
        for t, v in zip((c.latent, c.scales, c.rope), state):
            t.copy_(v)
        for t in (out, c_out, k_out):
            t.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert out.isfinite().all()
        for a, b in zip((out, c_out, k_out, c.latent, c.scales), want):
            assert torch.equal(a, b), i
        assert torch.equal(c.rope.nan_to_num(9.0), want[5].nan_to_num(9.0))


def test_steps_on_two_streams_with_workspaces_of_their_own():
    """Two loops at once, each on a stream of its own, give what they give alone."""
    results = []
    for together in (False, True):
        loops, streams = [_Loop("bf16"), _Loop("bf16", 2)], [torch.cuda.Stream(), torch.cuda.Stream()]
        qs = []
        for loop in loops:
            qn, qr = loop.queries()
            absorb = mlra.mlra2_absorb_q if loop.groups == 2 else mlra.mlra_absorb_q
            qs.append((absorb(qn, loop.w_uk), qr))
        torch.cuda.synchronize()
        outs = []
        for loop, stream, (qa, qr) in zip(loops, streams, qs):
            with torch.cuda.stream(stream):
                for _ in range(5):
                    out = mlra.mlra_mx4_decode_attn(loop.cache, qa, qr, loop.w_uv, loop.tau, groups=loop.groups)
            if not together:
                torch.cuda.synchronize()
            outs.append(out)
        torch.cuda.synchronize()
        results.append(outs)
    assert all(torch.equal(a, b) for a, b in zip(*results))
