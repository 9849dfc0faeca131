"""Operators on a caller's own tensors, what they compute and how long they take.

Three operators that belong together when a program keeps the keys and values of a
prompt and of finished blocks instead of recomputing them:

* rotary positions (``wino_rope``), and the same fused with the write of the rotated
  keys and of the values into a paged cache (``wino_rope_append``)
* attention of a chunk of new tokens over that cache (``wino_paged_attention``)
* attention over whole prompts of different lengths, packed one after the other
  (``wino_packed_attention``)

Each has a plain form here (elementary torch operations in 32 bits, angles in 64) and
the call of the framework; ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------ cases
def _rope(name, op, tokens, hq, hk, hd, **kw):
    c = dict(name=name, op=op, tokens=tokens, hq=hq, hk=hk, hd=hd, rot=hd, layout="half", start=0, page=16,
             theta=500000.0, factor=1.0, dtype="bf16")
    c.update(kw)
    return c


def _attn(name, op, seqs, hq, hk, hd, **kw):
    c = dict(name=name, op=op, seqs=seqs, hq=hq, hk=hk, hd=hd, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, mask="full", block=0,
             page=16, order="token", dtype="bf16", lens=1)
    c.update(kw)
    return c


def listed():
    return [
        # one new token of the tiny model: a launch and its latency
        _rope("append_one", "append", 1, 4, 4, 64, start=95, theta=10000.0),
        # one step of 16 cached sequences at the 8B shape: 32 block rows and 32 shadow rows each
        _rope("append_blocks", "append", 16 * 64, 32, 32, 128, start=512, page=64),
        # a long prompt entering the cache: grouped heads, interleaved pairs over half of each head, frequencies
        # scaled by parts for a context far beyond the trained one
        _rope("append_prompt", "append", 6007, 32, 8, 128, rot=64, layout="inter", start=1000003, theta=10000.0,
              factor=32.0, dtype="fp16", page=32),
        # gradients of the queries of 4 x 2112 rows, taken back through the rotation inside a fused QKV gradient
        _rope("rope_inverse", "inverse", 4 * 2112, 32, 32, 128),
        # one token against a short cache of the tiny model
        _attn("paged_one", "paged", 1, 4, 4, 64, kv_lo=97, kv_hi=97),
        # a serving batch of single tokens, ragged caches, grouped heads, small pages
        _attn("paged_tokens", "paged", 64, 32, 8, 128, kv_lo=1, kv_hi=8192),
        # a WINO step over 16 cached sequences at the 8B shape: block rows and shadow rows, the shadow mask
        _attn("paged_shadow", "paged", 16, 32, 32, 128, q_lo=64, q_hi=64, kv_lo=300, kv_hi=544, mask="shadow", block=32,
              page=64),
        # chunks of new prompt tokens behind long caches
        _attn("paged_chunks", "paged", 4, 32, 4, 128, q_lo=200, q_hi=500, kv_lo=3000, kv_hi=16000, mask="causal", page=32,
              order="head", dtype="fp16"),
        # a few short prompts of the tiny model
        _attn("packed_short", "packed", 3, 4, 4, 64, q_lo=1, q_hi=40, mask="causal", dtype="fp16"),
        # 16 prompts of different lengths with their responses at the 8B shape, every row sees every key
        _attn("packed_full", "packed", 16, 32, 32, 128, q_lo=200, q_hi=544),
        # many prompts, 64-wide grouped heads, empty ones among them
        _attn("packed_many", "packed", 24, 16, 2, 64, q_lo=0, q_hi=700, mask="causal", dtype="fp16", lens=3),
        # one long prompt: the matrix cores' share
        _attn("packed_long", "packed", 1, 32, 8, 128, q_lo=8192, q_hi=8192, mask="causal"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "inverse", "paged", "paged", "packed", "packed"])
    hd = rng.choice([64, 128])
    hk = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
    hq = hk * rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8) if g * hk <= 40])
    dtype = rng.choice(["bf16", "fp16"])
    if op in ("append", "inverse"):
        return dict(op=op, tokens=_log(rng, 1, 12000), hq=hq, hk=hk, hd=hd, rot=rng.choice([hd, hd, hd // 2, 16, 48]),
                    layout=rng.choice(["half", "inter"]), start=rng.choice([0, _log(rng, 1, 2000000)]),
                    page=rng.choice([16, 32, 64, 128]), theta=rng.choice([10000.0, 500000.0]),
                    factor=rng.choice([1.0, 4.0, 16.0]), dtype=dtype)
    c = dict(op=op, seqs=_log(rng, 1, 64), hq=hq, hk=hk, hd=hd, q_lo=1, q_hi=1, kv_lo=1, kv_hi=1, mask="full", block=0,
             page=rng.choice([16, 32, 64, 128]), order=rng.choice(["token", "head"]), dtype=dtype,
             lens=rng.randrange(1 << 30))
    if op == "packed":
        c["q_hi"] = _log(rng, 1, 8192)
        c["q_lo"] = rng.choice([0, 1, c["q_hi"]])
        c["mask"] = rng.choice(["full", "causal"])
        while c["seqs"] * hq * c["q_hi"] ** 2 > 1 << 30 and c["seqs"] > 1:
            c["seqs"] = (c["seqs"] + 1) // 2
    else:
        kind = rng.choice(["token", "chunk", "shadow"])
        c["kv_hi"] = _log(rng, 1, 16384)
        if kind == "shadow":
            c["block"] = rng.choice([4, 16, 24, 32, 64])
            c["q_lo"] = c["q_hi"] = 2 * c["block"]
            c["kv_hi"] += 2 * c["block"]
            c["mask"] = "shadow"
        elif kind == "chunk":
            c["q_hi"] = _log(rng, 1, 1000)
            c["mask"] = rng.choice(["full", "causal"])
        c["kv_lo"] = max(1, c["kv_hi"] // rng.choice([1, 2, 64]))
        while c["seqs"] > 1 and (c["seqs"] * hq * c["q_hi"] * c["kv_hi"] > 1 << 30 or
                                 c["seqs"] * hk * hd * c["kv_hi"] > 1 << 29):
            c["seqs"] = (c["seqs"] + 1) // 2
    return c


def _lens(c):
    """Rows and keys of each sequence, from the case alone."""
    r = random.Random(c["lens"])
    q = [r.randint(c["q_lo"], c["q_hi"]) for _ in range(c["seqs"])]
    q[r.randrange(c["seqs"])] = c["q_hi"]
    if c["op"] == "packed":
        return q, q
    least = c["block"] if c["mask"] == "shadow" else 0
    kv = [max(r.randint(c["kv_lo"], c["kv_hi"]), n + least) for n in q]
    kv[r.randrange(c["seqs"])] = max(c["kv_hi"], max(q) + least)
    return q, kv


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, dt, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dt)


def frequencies(rot, theta, factor, orig=4096, fast=32.0, slow=1.0):
    """Radians per position of each pair; with factor > 1 interpolated by parts: pairs that turn fewer than `slow` times
    over the trained context are slowed by the factor, pairs that turn over `fast` times keep theirs."""
    f = torch.tensor([theta ** (-2.0 * j / rot) for j in range(rot // 2)], dtype=torch.float64)
    if factor == 1.0:
        return f, 1.0
    turns = orig * f / (2 * math.pi)
    keep = ((turns - slow) / (fast - slow)).clamp(0, 1)
    return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = DT[c["dtype"]]
    hq, hk, hd = c["hq"], c["hk"], c["hd"]
    if c["op"] in ("append", "inverse"):
        n = c["tokens"]
        freq, mag = frequencies(c["rot"], c["theta"], c["factor"])
        # the rows of a fused QKV product; the positions of a block and of its shadow are the same ones
        qkv = _randn(g, (n, (hq + 2 * hk) * hd), dt)
        s = dict(case=c, freq=freq.to(DEV), magnitude=mag,
                 pos=(c["start"] + torch.arange(n, device=DEV) // (2 if n % 64 == 0 else 1)).to(torch.int32),
                 q=qkv[:, :hq * hd].view(n, hq, hd), k=qkv[:, hq * hd:(hq + hk) * hd].view(n, hk, hd),
                 v=qkv[:, (hq + hk) * hd:].view(n, hk, hd), q_out=torch.empty(n, hq, hd, dtype=dt, device=DEV))
        if c["op"] == "append":
            pages = -(-n // c["page"]) + 3
            s["k_cache"] = _randn(g, (pages, c["page"], hk, hd), dt)
            s["v_cache"] = _randn(g, (pages, c["page"], hk, hd), dt)
            slot = torch.randperm(pages * c["page"], generator=g, device=DEV)[:n]
            if n >= 8:
                slot[n - 2:] = -1  # padding rows of a batch are not written
            s["slot"] = slot
        return s
    q_len, kv_len = _lens(c)
    i32 = dict(dtype=torch.int32, device=DEV)
    total = sum(q_len)
    cu_q = torch.tensor([sum(q_len[:i]) for i in range(len(q_len) + 1)], **i32)
    s = dict(case=c, max_q=max(q_len), max_kv=max(kv_len), cu_q=cu_q, scale=1.0 / math.sqrt(hd),
             q=_randn(g, (total, hq, hd), dt, 1.5), out=torch.empty(total, hq, hd, dtype=dt, device=DEV),
             lse=torch.empty(total, hq, dtype=torch.float32, device=DEV), cur_start=None)
    if c["op"] == "packed":
        kv = _randn(g, (total, 2, hk, hd), dt)  # keys and values side by side, as a fused product leaves them
        s.update(k=kv[:, 0], v=kv[:, 1], cu_k=cu_q)
        return s
    page = c["page"]
    width = -(-max(kv_len) // page)
    used = [-(-n // page) for n in kv_len]
    pages = sum(used) + 5
    shape = (pages, page, hk, hd) if c["order"] == "token" else (pages, hk, page, hd)
    k, v = _randn(g, shape, dt), _randn(g, shape, dt)
    if c["order"] == "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    ids = torch.randperm(pages, generator=g, device=DEV)[:sum(used)].to(torch.int32)
    table = torch.zeros(len(used), width, **i32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = ids[at:at + n]
        at += n
    s.update(k_cache=k, v_cache=v, table=table, kv_len=torch.tensor(kv_len, **i32))
    if c["mask"] == "shadow":
        room = torch.tensor(kv_len, **i32) - 2 * c["block"]
        u = torch.rand(len(kv_len), generator=g, device=DEV)
        s["cur_start"] = (u * (room + 1).float()).to(torch.int32).minimum(room).clamp(min=0)
    return s


# ------------------------------------------------------------------ plain forms
def _rotate(x, s, sign):
    """x [tokens, heads, hd] in 32 bits, the first `rot` values of each head rotated by sign * position * frequency."""
    c = s["case"]
    rot = c["rot"]
    angle = s["pos"].double()[:, None] * s["freq"][None, :]
    cos = (torch.cos(angle) * s["magnitude"]).float()[:, None, :]
    sin = (torch.sin(angle) * (sign * s["magnitude"])).float()[:, None, :]
    x = x.float()
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_append(s):
    c, dt = s["case"], DT[s["case"]["dtype"]]
    page, last = c["page"], s["k_cache"].shape[0] * c["page"]
    slot = torch.where(s["slot"] < 0, last, s["slot"])  # one row more takes what is not written
    out = [_rotate(s["q"], s, 1.0).to(dt)]
    for cache, rows in ((s["k_cache"], _rotate(s["k"], s, 1.0).to(dt)), (s["v_cache"], s["v"])):
        flat = torch.cat([cache.flatten(0, 1), cache[0, :1]])
        flat[slot] = rows
        cache.copy_(flat[:last].view_as(cache))
        out.append(cache)
    return out


def _plain_attention(s):
    c = s["case"]
    hq, hk, hd, B = c["hq"], c["hk"], c["hd"], c["seqs"]
    q0, n_q = s["cu_q"][:-1].long(), (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    i = torch.arange(s["max_q"], device=DEV)
    j = torch.arange(s["max_kv"], device=DEV)
    rows = (q0[:, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float()
    if c["op"] == "packed":
        n_kv = n_q
        keys = (s["cu_k"][:-1].long()[:, None] + j).clamp(max=s["k"].shape[0] - 1)
        k, v = s["k"][keys].float(), s["v"][keys].float()
    else:
        n_kv = s["kv_len"].long()
        pages = s["table"].long()[:, j // c["page"]]
        off = (j % c["page"]).expand_as(pages)
        k, v = s["k_cache"][pages, off].float(), s["v_cache"][pages, off].float()
    # [B, hk, group * rows, hd] times [B, hk, hd, keys]: the query heads of a group share their keys
    qh = q.view(B, -1, hk, hq // hk, hd).permute(0, 2, 3, 1, 4).reshape(B, hk, -1, hd).contiguous()
    kh, vh = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()
    z = torch.matmul(qh, kh).view(B, hk, hq // hk, s["max_q"], s["max_kv"])
    z *= s["scale"]
    if c["mask"] == "full":
        sees = (j < n_kv[:, None])[:, None, :].expand(B, s["max_q"], s["max_kv"])
    elif c["mask"] == "causal":
        sees = j <= (n_kv - n_q)[:, None, None] + i[:, None]
    else:
        at = i - (n_q - c["block"])[:, None]  # which shadow row, below zero for the others
        shadow = (at >= 0)[:, :, None]
        sees = j < torch.where(shadow, n_kv[:, None, None], (n_kv - c["block"])[:, None, None])
        sees = sees & ~(shadow & (j == (s["cur_start"].long()[:, None] + at)[:, :, None]))
    z.masked_fill_(~sees[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top)[..., 0]
    o = torch.matmul(p.view(B, hk, -1, s["max_kv"]), vh).view(B, hk, hq // hk, s["max_q"], hd)
    o = torch.where(total > 0, o / total, 0.0)
    t = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(s["cu_q"][1:].long(), t, right=True)
    at = t - q0[b]
    o = o.permute(0, 3, 1, 2, 4).reshape(B, s["max_q"], hq, hd)[b, at]
    return o.to(DT[c["dtype"]]), lse.permute(0, 3, 1, 2).reshape(B, s["max_q"], hq)[b, at]


# ------------------------------------------------------------------ the framework's calls
def _kept(s):
    """What a user's program makes once and keeps beside its tensors: parameters, the cache's description, a workspace."""
    if "kept" in s:
        return s["kept"]
    import paper_2605_16941_amd as P
    c = s["case"]
    act = P.ACT_BF16 if c["dtype"] == "bf16" else P.ACT_FP16
    kept = {"P": P}
    if "k_cache" in s:
        kept["cache"] = P.make_kv_cache(s["k_cache"], s["v_cache"])
    if c["op"] in ("append", "inverse"):
        kept["p"] = P.make_rope_params(c["hd"], c["rot"], P.ROPE_HALF if c["layout"] == "half" else P.ROPE_INTERLEAVED,
                                       dtype=act, magnitude=s["magnitude"], inverse=c["op"] == "inverse")
    else:
        mask = {"full": P.MASK_FULL, "causal": P.MASK_CAUSAL, "shadow": P.MASK_SHADOW}[c["mask"]]
        kept["p"] = P.make_attn_params(c["hq"], c["hk"], c["hd"], dtype=act, mask=mask, block_len=c["block"],
                                       scale=s["scale"])
        n = P.wino_attention_workspace_bytes(kept["p"], c["seqs"], s["q"].shape[0], s["max_kv"])
        kept["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    s["kept"] = kept
    return kept


def _own(s):
    kept, op = _kept(s), s["case"]["op"]
    P = kept["P"]
    if op == "append":
        P.wino_rope_append(kept["p"], kept["cache"], s["freq"], s["pos"], s["slot"], s["q"], s["k"], s["v"], s["q_out"])
        return [s["q_out"], s["k_cache"], s["v_cache"]]
    if op == "inverse":
        P.wino_rope(kept["p"], s["freq"], s["pos"], s["q"], s["q_out"])
        return [s["q_out"]]
    if op == "paged":
        P.wino_paged_attention(kept["p"], kept["cache"], s["q"], s["out"], s["cu_q"], s["kv_len"], s["table"], s["max_kv"],
                               cur_start=s["cur_start"], lse=s["lse"], workspace=kept["workspace"])
    else:
        P.wino_packed_attention(kept["p"], s["q"], s["k"], s["v"], s["out"], s["cu_q"], s["cu_k"], s["max_kv"],
                                cur_start=s["cur_start"], lse=s["lse"], workspace=kept["workspace"])
    return [s["out"], s["lse"]]


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    if op == "append":
        return _plain_append(s)
    if op == "inverse":
        return [_rotate(s["q"], s, -1.0).to(DT[s["case"]["dtype"]])]
    return list(_plain_attention(s))


# ------------------------------------------------------------------ work and exact results
def _pairs(c):
    """(query, key) pairs of one head, and the keys read."""
    q, kv = _lens(c)
    pairs = 0
    for n, m in zip(q, kv):
        if c["mask"] == "full":
            pairs += n * m
        elif c["mask"] == "causal":
            pairs += sum(max(0, m - n + i + 1) for i in range(n))
        else:
            pairs += (n - c["block"]) * (m - c["block"]) + c["block"] * (m - 1)
    return pairs, sum(m for n, m in zip(q, kv) if n), sum(q)


def work(case):
    c = case
    if c["op"] in ("append", "inverse"):
        n = c["tokens"]
        values = n * c["hd"] * (c["hq"] + (2 * c["hk"] if c["op"] == "append" else 0))
        return {"bytes": 2 * 2 * values + n * (4 + (8 if c["op"] == "append" else 0)) + 4 * c["rot"],
                "flops": 6 * n * c["rot"] // 2 * (c["hq"] + (c["hk"] if c["op"] == "append" else 0))}
    pairs, keys, rows = _pairs(c)
    return {"bytes": 2 * c["hd"] * (2 * rows * c["hq"] + 2 * keys * c["hk"]) + 4 * rows * c["hq"],
            "flops": 4 * c["hd"] * c["hq"] * pairs}


def _exact_rotate(x, s, sign):
    c, rot = s["case"], s["case"]["rot"]
    x = x.double()
    turn = torch.polar(torch.full_like(s["freq"], s["magnitude"]).expand(x.shape[0], -1).contiguous(),
                       sign * s["pos"].double()[:, None] * s["freq"])[:, None, :]
    y = x.clone()
    if c["layout"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.complex(x[..., 0:rot:2].contiguous(), x[..., 1:rot:2].contiguous()) * turn
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "inverse":
        return [_exact_rotate(s["q"], s, -1.0)]
    if c["op"] == "append":
        out = [_exact_rotate(s["q"], s, 1.0)]
        write = s["slot"] >= 0
        at = s["slot"][write]
        for cache, rows in ((s["k_cache"], _exact_rotate(s["k"], s, 1.0)), (s["v_cache"], s["v"].double())):
            flat = cache.double().flatten(0, 1)
            flat[at] = rows[write]
            out.append(flat.view(cache.shape))
        return out
    q_len, kv_len = _lens(c)
    hq, hk = c["hq"], c["hk"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, m) in enumerate(zip(q_len, kv_len)):
        if n and m:
            if c["op"] == "packed":
                k, v = s["k"][first:first + m].double(), s["v"][first:first + m].double()
            else:
                pages = s["table"][b, :-(-m // c["page"])].long()
                k = s["k_cache"][pages].flatten(0, 1)[:m].double()
                v = s["v_cache"][pages].flatten(0, 1)[:m].double()
            row, key = torch.arange(n, device=DEV)[:, None], torch.arange(m, device=DEV)[None, :]
            hide = torch.zeros(n, m, dtype=torch.bool, device=DEV)
            if c["mask"] == "causal":
                hide = key - row > m - n
            elif c["mask"] == "shadow":
                lb = c["block"]
                j = row - (n - lb)
                hide = ((j < 0) & (key >= m - lb)) | ((j >= 0) & (key == s["cur_start"][b].long() + j))
            for h in range(hq):
                z = s["q"][first:first + n, h].double() @ k[:, h // (hq // hk)].T.contiguous() * s["scale"]
                z.masked_fill_(hide, -math.inf)
                l = torch.logsumexp(z, -1)
                w = torch.exp(z - torch.where(torch.isfinite(l), l, 0.0)[:, None])
                out[first:first + n, h] = w @ v[:, h // (hq // hk)].contiguous()
                lse[first:first + n, h] = l
        first += n
    return [out, lse]
