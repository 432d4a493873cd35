"""Caches in 4 bits for the GPU tests: built on the host with the oracle's format, poisoned where no sequence owns a slot."""
from __future__ import annotations

import numpy as np
import torch

from oracle import mx4_oracle as orc
from paper_2603_02188_amd import binding as mlra
from paper_2603_02188_amd import inputs as gen

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def stored(x, dtype):
    """float values -> (device tensor of dtype, the float64 values that it holds)."""
    bits = gen.to_storage(np.asarray(x, dtype=np.float32), dtype)
    t = torch.from_numpy(bits)
    if dtype == "bf16":
        t = t.view(torch.bfloat16)
    return t.cuda(), gen.to_f64(bits, dtype)


def random_groups(rng, shape):
    """Codes and scale bytes of random rows (scales over six binades): every code occurs."""
    packed = rng.integers(0, 256, size=shape[:-1] + (shape[-1] // 2,), dtype=np.uint8)
    scales = rng.integers(123, 129, size=shape[:-1] + (shape[-1] // 32,)).astype(np.uint8)
    return packed, scales


class HostCache:
    """Pools of a paged cache; slots that no sequence owns hold NaN."""

    def __init__(self, lens, n_blocks, d_cb, d_r, dtype, page, seed, max_pages=None, spare=3):
        rng = np.random.default_rng([seed, 4])
        self.lens, self.n_blocks, self.d_cb, self.d_r, self.dtype, self.page = list(lens), n_blocks, d_cb, d_r, dtype, page
        need = [-(-n // page) for n in self.lens]
        width = max_pages or max(1, max(need))
        total = sum(need) + spare
        order = rng.permutation(total)
        self.table = np.full((len(self.lens), width), order[-1], dtype=np.int32)
        at = 0
        for s, k in enumerate(need):
            self.table[s, :k] = order[at:at + k]
            at += k
        self.latent = rng.integers(0, 256, size=(total, n_blocks, page, d_cb // 2), dtype=np.uint8)
        self.scales = np.full((total, n_blocks, page, d_cb // 32), 255, dtype=np.uint8)
        self.rope = np.full((total, page, d_r), np.nan)
        self.rows, self.ropes = [], []
        for s, n in enumerate(self.lens):
            packed, scales = random_groups(rng, (n, n_blocks, d_cb))
            rope = gen.to_f64(gen.to_storage(rng.standard_normal((n, d_r)).astype(np.float32), dtype), dtype)
            for t in range(0, n, page):
                p, k = self.table[s, t // page], min(page, n - t)
                self.latent[p, :, :k] = packed[t:t + k].transpose(1, 0, 2)
                self.scales[p, :, :k] = scales[t:t + k].transpose(1, 0, 2)
                self.rope[p, :k] = rope[t:t + k]
            self.rows.append(orc.decode(packed, scales))
            self.ropes.append(rope)

    def device(self, lens=None):
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        return mlra.Mx4Cache(up(self.latent), up(self.scales), stored(self.rope, self.dtype)[0], up(self.table),
                             up(np.array(self.lens if lens is None else lens, dtype=np.int32)))


def queries(rng, batch, q_len, n_blocks, hb, groups, d_cb, d_r, d_h, dtype):
    q_abs = stored(rng.standard_normal((batch, q_len, n_blocks, hb, d_cb)), dtype)
    q_rope = stored(rng.standard_normal((batch, q_len, groups * hb, d_r)), dtype)
    w_uv = stored(rng.standard_normal((n_blocks, d_cb, hb * d_h)) / np.sqrt(d_cb), dtype)
    return q_abs, q_rope, w_uv
