"""The operators of the 4-bit latent cache: what is timed, on which inputs, and what they compute.

The cache holds the latent C^KV of every token in 4 bits: groups of 32 channels share a power of two (one byte, E8M0), and
each channel is one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times it (E2M1).  The RoPE key stays in the cache's 16- or 32-bit
type.  Three operators work on it:

  write    rows of new tokens are quantised as they go into their pages
  read     rows are gathered from their pages and given back as the values they stand for
  decode   the attention of MLRA-4 / MLRA-2 / MLA on such a cache, up-projection and block sum included

A "write" case writes a piece of every sequence and then reads the sequence back up to its end, as a prompt that comes in
pieces is handled: the attention of the next piece works on what the cache stands for.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_GROUP = 32
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases ------------------------------------------------------------------------------------------------------------
def _rows(kind, batch, n_min, n_max, **kw):
    """kind "write": the last `new` tokens of every sequence (all of them if it is shorter) are written, then the sequence
    is read; kind "read": only read."""
    case = {"kind": kind, "batch": batch, "n_min": n_min, "n_max": n_max, "new": n_max, "n_blocks": 4, "d_cb": 128,
            "d_r": 64, "dtype": "bf16", "src": "bf16", "page": 64, "shuffle": False}
    case.update(kw)
    return case


def _decode(batch, n_min, n_max, **kw):
    case = {"kind": "decode", "batch": batch, "n_min": n_min, "n_max": n_max, "groups": 1, "n_blocks": 4, "d_cb": 128,
            "d_r": 64, "h": 128, "d_h": 128, "dtype": "bf16", "out": "bf16", "page": 64, "shuffle": False, "q_len": 1,
            "gated": False, "lse": False}
    case.update(kw)
    return case


def listed():
    return [
        # the newest row of every sequence of a serving batch, as a decode step writes it, and the sequence's first rows with
        # it: all launches
        dict(_rows("write", 64, 1, 16, new=1, src="f32", shuffle=True), name="write-step-64"),
        # a piece of 512 tokens of four long prompts, shuffled pages
        dict(_rows("write", 4, 2000, 8192, new=512, shuffle=True), name="write-piece-4x512"),
        # whole prompts of a batch, from fp32 rows
        dict(_rows("write", 64, 1024, 8192, src="f32"), name="write-prompts-64"),
        # one short context of the small fp32 model
        dict(_rows("read", 1, 333, 333, d_cb=64, d_r=32, dtype="f32", src="f32", page=16), name="read-333-f32"),
        # the whole cache of the headline workload, handed to another server
        dict(_rows("read", 64, 8192, 8192, shuffle=True), name="read-64x8k"),
        # one user's request, small pages
        dict(_decode(1, 1501, 1501, page=16, shuffle=True), name="decode-single-1501"),
        # the headline workload: MLRA-4, 64 sequences of 8K
        dict(_decode(64, 8192, 8192), name="decode-64x8k"),
        # a serving batch: mixed lengths, shuffled pages, gated output, log-sum-exp
        dict(_decode(128, 512, 8192, shuffle=True, gated=True, lse=True), name="decode-128-mixed"),
        # few users, very long contexts, MLRA-2
        dict(_decode(4, 65536, 131072, groups=2), name="decode-mlra2-4x128k"),
        # drafts of four tokens, ragged
        dict(_decode(16, 1000, 4093, q_len=4, shuffle=True, out="f32"), name="decode-draft-16x4"),
        # MLA: one latent of 512 channels
        dict(_decode(64, 512, 4096, n_blocks=1, d_cb=512, shuffle=True), name="decode-mla-64-mixed"),
        # the full-size layer in fp32 (reference runs)
        dict(_decode(8, 300, 2048, dtype="f32", out="f32", lse=True), name="decode-f32-8x2k"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "decode", "decode", "multi", "mlra2", "mla", "f32", "small"])
    opt = {"page": rng.choice([16, 32, 64, 64, 128, 48]), "shuffle": rng.random() < 0.5}
    total = {"write": 300000, "read": 400000, "decode": 500000, "mlra2": 500000, "multi": 40000, "mla": 150000, "f32": 9000,
             "small": 60000}[kind]
    most = {"decode": 131072, "mlra2": 131072, "multi": 16384, "f32": 2048}.get(kind, 32768)
    batch = _log(rng, 1, {"f32": 16, "multi": 32}.get(kind, 128))
    n_max = _log(rng, 32, max(33, min(most, total // batch)))
    n_min = n_max if rng.random() < 0.3 else max(1, int(n_max * rng.uniform(0.02, 1.0)))
    if kind in ("write", "read"):
        opt.update(n_blocks=rng.choice([1, 4]), d_cb=rng.choice([64, 128, 128, 256]), d_r=rng.choice([32, 64]),
                   dtype=rng.choice(["bf16", "bf16", "f32"]), src=rng.choice(["bf16", "f32"]))
        return _rows(kind, batch, n_min, n_max, new=_log(rng, 1, n_max), **opt)
    opt.update(lse=rng.random() < 0.4, out=rng.choice(["bf16", "f32"]))
    if kind == "decode":
        return _decode(batch, n_min, n_max, n_blocks=rng.choice([1, 4, 4]), h=rng.choice([16, 64, 128, 128]),
                       gated=rng.random() < 0.3, **opt)
    if kind == "multi":
        return _decode(batch, n_min, n_max, q_len=rng.choice([2, 3, 4]), **opt)
    if kind == "mlra2":
        return _decode(batch, n_min, n_max, groups=2, **opt)
    if kind == "mla":
        return _decode(batch, n_min, n_max, n_blocks=1, d_cb=512, h=rng.choice([16, 64, 128]), **opt)
    if kind == "f32":
        return _decode(batch, n_min, n_max, h=rng.choice([16, 64, 128]), dtype="f32", **dict(opt, out="f32"))
    return _decode(batch, n_min, n_max, n_blocks=rng.choice([2, 4]), d_cb=64, d_r=32, d_h=64, h=rng.choice([8, 12, 16]),
                   dtype=rng.choice(["bf16", "f32"]), **opt)


# ---- inputs -----------------------------------------------------------------------------------------------------------
class _State:
    pass


def _lens(case):
    """Spread evenly from n_min to n_max, so that the work does not depend on the seed."""
    b, lo, hi = case["batch"], case["n_min"], case["n_max"]
    return [hi if b == 1 else lo + round((hi - lo) * i / (b - 1)) for i in range(b)]


def _quantise(x):
    """x [..., channels], fp32 -> codes (0..15) and scale bytes [..., channels / 32]."""
    g = x.unflatten(-1, (-1, _GROUP))
    bits = g.abs().amax(-1).view(torch.int32)
    # the power of two of the largest channel as one mantissa bit rounds it, two lower: 1.75 .. 2 counts as 2
    byte = (((bits + 0x200000) >> 23) - 2).clamp(2, 252)
    finite = (bits & 0x7F800000) != 0x7F800000
    y = g.abs() * torch.ldexp(torch.ones((), device=x.device), 127 - byte)[..., None]
    code = (y > 0.25).to(torch.uint8)
    for at, tie_up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (y >= at) if tie_up else (y > at)                       # ties go to the even mantissa
    code += torch.signbit(g).to(torch.uint8) * 8
    code = torch.where(finite[..., None], code, torch.zeros_like(code))
    return code.flatten(-2), torch.where(finite, byte, torch.full_like(byte, 255)).to(torch.uint8)


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _values(packed, scales):
    """The fp32 values that packed codes [..., channels / 2] and scale bytes [..., channels / 32] stand for."""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=packed.device)
    v = torch.stack((table[(packed & 15).long()], table[(packed >> 4).long()]), dim=-1).flatten(-2)
    scale = torch.ldexp(torch.ones((), device=packed.device), scales.int() - 127)
    scale = torch.where(scales == 255, torch.full_like(scale, math.nan), scale)
    return (v.unflatten(-1, (-1, _GROUP)) * scale[..., None]).flatten(-2)


def _paging(case, gen):
    """Lengths in an order drawn from the seed; a page table over the pages that they need and one that nobody owns."""
    lens = torch.tensor(_lens(case), dtype=torch.int32)
    lens = lens[torch.randperm(len(lens), generator=gen, device="cuda").cpu()].contiguous()
    pages = (lens + case["page"] - 1) // case["page"]
    total, width = int(pages.sum()), int(pages.max())
    order = torch.randperm(total + 1, generator=gen, device="cuda").int().cpu() if case["shuffle"] else torch.arange(total + 1).int()
    table, at = torch.full((len(pages), width), int(order[total]), dtype=torch.int32), 0
    for b, k in enumerate(pages.tolist()):
        table[b, :k] = order[at:at + k]
        at += k
    return lens, table, total + 1


def _slots(case, table, first, count):
    """(page, slot) of tokens first .. first + count of a sequence, whose pages `table` lists."""
    t = torch.arange(first, first + count, device=table.device)
    return table.long()[t // case["page"]], t % case["page"]


def _new_rows(case, gen, shape):
    """Latents as they leave a norm with learned gains: channels of different size, a few much larger than the rest."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    gain = torch.exp(0.3 * torch.randn(shape[-1], generator=gen, device="cuda"))
    gain[torch.rand(shape[-1], generator=gen, device="cuda") < 0.01] *= 4.0
    return x.mul_(gain / gain.square().mean().sqrt())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = _State()
    s.case, dt, b = case, _DT[case["dtype"]], case["batch"]
    nb, d_cb, d_r, page = case["n_blocks"], case["d_cb"], case["d_r"], case["page"]
    lens, table, total = _paging(case, gen)
    s.lens_host, s.lens, s.table = lens.tolist(), lens.cuda(), table.cuda()
    # slots that no sequence owns hold NaN, whatever their codes
    s.latent = torch.randint(0, 256, (total, nb, page, d_cb // 2), generator=gen, device="cuda", dtype=torch.uint8)
    s.scales = torch.full((total, nb, page, d_cb // _GROUP), 255, dtype=torch.uint8, device="cuda")
    s.rope = torch.full((total, page, d_r), math.nan, dtype=dt, device="cuda")
    for i, n in enumerate(s.lens_host):
        at = _slots(case, s.table[i], 0, n)
        code, byte = _quantise(_new_rows(case, gen, (n, nb * d_cb)))
        s.latent[at[0], :, at[1]] = _pack(code).view(n, nb, d_cb // 2)
        s.scales[at[0], :, at[1]] = byte.view(n, nb, -1)
        s.rope[at[0], at[1]] = torch.randn((n, d_r), generator=gen, device="cuda").to(dt)
    if case["kind"] != "decode":
        src, new = _DT[case["src"]], case["new"]
        if case["kind"] == "write":
            s.c_new = _new_rows(case, gen, (b, new, nb * d_cb)).to(src)
            s.k_new = torch.randn((b, new, d_r), generator=gen, device="cuda").to(src)
            s.new_lens_host = [min(n, new) for n in s.lens_host]
            s.first = torch.tensor([n - k for n, k in zip(s.lens_host, s.new_lens_host)], dtype=torch.int32, device="cuda")
            s.new_lens = torch.tensor(s.new_lens_host, dtype=torch.int32, device="cuda")
        s.start = torch.zeros(b, dtype=torch.int32, device="cuda")
        s.c_out = torch.zeros((b, max(s.lens_host), nb * d_cb), dtype=src, device="cuda")
        s.k_out = torch.zeros((b, max(s.lens_host), d_r), dtype=src, device="cuda")
    else:
        h, d_h, hb, lead = case["h"], case["d_h"], case["h"] // case["groups"], (b, case["q_len"])
        s.scale = 1.0 / math.sqrt(d_h + d_r)
        s.q_abs = torch.randn(lead + (nb, hb, d_cb), generator=gen, device="cuda").to(dt)
        s.q_rope = torch.randn(lead + (h, d_r), generator=gen, device="cuda").to(dt)
        s.w_uv = (torch.randn((nb, d_cb, hb * d_h), generator=gen, device="cuda") / math.sqrt(d_cb)).to(dt)
        s.gate = torch.sigmoid(torch.randn(lead + (h, d_h), generator=gen, device="cuda")).to(dt) if case["gated"] else None
        s.out = torch.empty(lead + (h, d_h), dtype=_DT[case["out"]], device="cuda")
        s.lse = torch.empty(lead + (nb, hb), device="cuda") if case["lse"] else None
    if own:
        from paper_2603_02188_amd import binding as mlra
        s.cache = mlra.Mx4Cache(s.latent, s.scales, s.rope, s.table, s.lens)
        if case["kind"] == "decode":
            s.workspace = torch.empty(mlra.mlra_mx4_decode_workspace_bytes(b, case["q_len"], case["h"], case["groups"], nb, d_cb,
                                                                           page, s.table.shape[1]),
                                      dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2603_02188_amd import binding as mlra
    case = s.case
    if case["kind"] == "decode":
        mlra.mlra_mx4_decode_attn(s.cache, s.q_abs, s.q_rope, s.w_uv, s.scale, groups=case["groups"], gate=s.gate, out=s.out,
                                  lse=s.lse, workspace=s.workspace)
        return {"out": s.out} if s.lse is None else {"out": s.out, "lse": s.lse}
    if case["kind"] == "write":
        mlra.mlra_mx4_append_kv(s.cache, s.c_new, s.k_new, s.first, new_lens=s.new_lens)
    mlra.mlra_mx4_read_kv(s.cache, s.start, s.lens, s.c_out, s.k_out)
    return {"c_kv": s.c_out, "k_rope": s.k_out}


def _run_plain(s):
    case = s.case
    nb, d_cb = case["n_blocks"], case["d_cb"]
    if case["kind"] == "decode":
        return _attend_plain(s)
    if case["kind"] == "write":
        for i, k in enumerate(s.new_lens_host):
            at = _slots(case, s.table[i], s.lens_host[i] - k, k)
            code, byte = _quantise(s.c_new[i, :k].float())
            s.latent[at[0], :, at[1]] = _pack(code).view(k, nb, d_cb // 2)
            s.scales[at[0], :, at[1]] = byte.view(k, nb, -1)
            s.rope[at[0], at[1]] = s.k_new[i, :k].to(s.rope.dtype)
    for i, n in enumerate(s.lens_host):
        at = _slots(case, s.table[i], 0, n)
        s.c_out[i, :n] = _values(s.latent[at[0], :, at[1]], s.scales[at[0], :, at[1]]).view(n, nb * d_cb).to(s.c_out.dtype)
        s.k_out[i, :n] = s.rope[at[0], at[1]].to(s.k_out.dtype)
    return {"c_kv": s.c_out, "k_rope": s.k_out}


def _attend_plain(s):
    case = s.case
    b, q_len, nb, hb, d_cb = s.q_abs.shape
    groups, d_h = case["groups"], case["d_h"]
    bpg = nb // groups
    q_abs, q_rope, w_uv = s.q_abs.float(), s.q_rope.float(), s.w_uv.float().view(nb, d_cb, hb, d_h)
    z = torch.zeros((b, q_len, nb, hb, d_cb), device=q_abs.device)
    lse = torch.full((b, q_len, nb, hb), -math.inf, device=q_abs.device)
    for i, n in enumerate(s.lens_host):
        at = _slots(case, s.table[i], 0, n)
        c = _values(s.latent[at[0], :, at[1]], s.scales[at[0], :, at[1]])                 # [n][blocks][channels]
        k_rope = s.rope[at[0], at[1]].float()
        # query j stands at token n - q_len + j and sees the tokens up to itself
        seen = torch.arange(n, device=c.device)[None, :] <= n - q_len + torch.arange(q_len, device=c.device)[:, None]
        for blk in range(nb):
            first = (blk // bpg) * hb
            c_b = c[:, blk].contiguous()
            score = q_abs[i, :, blk].reshape(q_len * hb, d_cb) @ c_b.t()
            score += q_rope[i, :, first:first + hb].reshape(q_len * hb, -1) @ k_rope.t()
            score = (score * s.scale).view(q_len, hb, n)
            score = torch.where(seen[:, None], score, torch.full_like(score, -math.inf))
            top = score.amax(-1, keepdim=True).clamp_min(-3.0e38)
            p = torch.exp(score - top)
            total = p.sum(-1, keepdim=True)
            z[i, :, blk] = ((p.view(q_len * hb, n) @ c_b).view(q_len, hb, d_cb) / total.clamp_min(1e-38))
            lse[i, :, blk] = (top + torch.log(total)).squeeze(-1)
    out = torch.zeros((b * q_len, case["h"], d_h), device=z.device)
    z = z.view(b * q_len, nb, hb, d_cb)
    for blk in range(nb):
        for i in range(hb):
            out[:, (blk // bpg) * hb + i] += z[:, blk, i] @ w_uv[blk, :, i]
    out = out.view(s.out.shape)
    if s.gate is not None:
        out = out * s.gate.float()
    out = out.to(s.out.dtype)
    return {"out": out} if s.lse is None else {"out": out, "lse": lse}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    nb, d_cb, d_r, e = case["n_blocks"], case["d_cb"], case["d_r"], _SIZE[case["dtype"]]
    lens = _lens(case)
    tokens, row = sum(lens), nb * (d_cb // 2 + d_cb // _GROUP) + d_r * e             # cached bytes of one token
    if case["kind"] != "decode":
        src = (nb * d_cb + d_r) * _SIZE[case["src"]]
        new = sum(min(n, case["new"]) for n in lens) if case["kind"] == "write" else 0
        # rows that were just written need not be read from the cache again to be given back
        return {"bytes": new * (src + row) + (tokens - new) * row + tokens * src, "flops": tokens * nb * d_cb}
    b, q_len, h, hb, d_h = case["batch"], case["q_len"], case["h"], case["h"] // case["groups"], case["d_h"]
    rows, w = b * q_len, nb * d_cb * hb * d_h
    moved = tokens * row + rows * (nb * hb * d_cb + h * d_r) * e + w * e + rows * h * d_h * _SIZE[case["out"]]
    moved += rows * h * d_h * e if case["gated"] else 0
    moved += rows * nb * hb * 4 if case["lse"] else 0
    pairs = sum(max(0, n - j) for n in lens for j in range(q_len))                   # (query, token) pairs
    return {"bytes": moved, "flops": 2 * pairs * nb * hb * (2 * d_cb + d_r) + 2 * rows * w}


# ---- the same in 64 bits, from the definition -------------------------------------------------------------------------
def _e2m1(x):
    """x [rows, channels] in 64 bits -> the values that the cache stands for after x was written."""
    g = x.reshape(x.shape[0], -1, _GROUP)
    top = g.abs().max(dim=-1).values
    m, e = torch.frexp(top)                                              # top = m 2^e, m in [0.5, 1)
    e = e + (m >= 0.875).to(e.dtype) - 3                                 # 2^e: the group's power of two
    unit = torch.ldexp(torch.ones_like(top), e.clamp(-125, 125))[..., None]
    y = g / unit
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y.abs()).exponent.clamp(1, 3) - 2)    # 0.5 below 2, 1 below 4, 2 above
    v = (torch.round(y / step) * step).clamp(-6.0, 6.0) * unit           # round: ties to even
    return torch.where(torch.isfinite(top)[..., None], v, torch.full_like(v, math.nan)).reshape(x.shape)


def _stored(packed, scales):
    """The 64-bit values of stored rows: sign, two exponent bits and one mantissa bit, times 2^(byte - 127)."""
    n = torch.stack((packed % 16, packed // 16), dim=-1).flatten(-2).to(torch.int64)
    exponent, mantissa = (n % 8) // 2, (n % 2).double()
    size = torch.where(exponent == 0, 0.5 * mantissa, (1.0 + 0.5 * mantissa) * 2.0 ** (exponent - 1).double())
    size = torch.where(n >= 8, -size, size).unflatten(-1, (-1, _GROUP))
    return (size * (2.0 ** (scales.double() - 127.0))[..., None]).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    nb, d_cb, d_r, page, b = case["n_blocks"], case["d_cb"], case["d_r"], case["page"], case["batch"]
    f64 = dict(dtype=torch.float64, device="cuda")

    def pages_of(i):
        return s.table[i, : -(-s.lens_host[i] // page)].long()

    def latent_of(i, blk):
        p = pages_of(i)
        return _stored(s.latent[p, blk], s.scales[p, blk]).reshape(-1, d_cb)[:s.lens_host[i]]

    def rope_of(i):
        return s.rope[pages_of(i)].reshape(-1, d_r)[:s.lens_host[i]].double()

    if case["kind"] != "decode":
        c, k = torch.zeros(s.c_out.shape, **f64), torch.zeros(s.k_out.shape, **f64)
        for i, n in enumerate(s.lens_host):
            for blk in range(nb):
                c[i, :n, blk * d_cb:(blk + 1) * d_cb] = latent_of(i, blk)
            k[i, :n] = rope_of(i)
            if case["kind"] == "write":
                m = s.new_lens_host[i]
                c[i, n - m:n] = _e2m1(s.c_new[i, :m].double())
                k[i, n - m:n] = s.k_new[i, :m].to(s.rope.dtype).double()
        return {"c_kv": c, "k_rope": k}
    h, d_h, groups, q_len = case["h"], case["d_h"], case["groups"], case["q_len"]
    hb, bpg = h // groups, nb // groups
    out, lse = torch.zeros((b, q_len, h, d_h), **f64), torch.full((b, q_len, nb, hb), -math.inf, **f64)
    w = s.w_uv.double().view(nb, d_cb, hb, d_h).permute(0, 2, 1, 3).contiguous()
    for i, n in enumerate(s.lens_host):
        k_rope = rope_of(i)
        for blk in range(nb):
            c, g = latent_of(i, blk), blk // bpg
            for j in range(q_len):
                m = n - (q_len - 1 - j)
                if m <= 0:
                    continue
                q = torch.cat((s.q_abs[i, j, blk], s.q_rope[i, j, g * hb:(g + 1) * hb]), dim=-1).double() * s.scale
                t = q @ torch.cat((c[:m], k_rope[:m]), dim=-1).t()
                lse[i, j, blk] = torch.logsumexp(t, dim=-1)
                z = torch.exp(t - lse[i, j, blk][:, None]) @ c[:m]
                out[i, j, g * hb:(g + 1) * hb] += torch.matmul(z[:, None, :], w[blk]).squeeze(1)
    if s.gate is not None:
        out *= s.gate.double()
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
