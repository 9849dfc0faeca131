"""Attention of packed rows over a paged cache or over packed keys against the float64 oracle.

Tolerances, from arithmetic, with eps/2 half a step of the type, a = sum_j w_j |v_j| and d the largest
scale sum_e |q_e k_e| of a row: the weights are rounded to the type before they meet the values (eps/2 a; for fp16 also
2^-25 each where they are subnormal, next to a sum of at least one: n 2^-25 max|v|), the output once (eps/2 |o|); the
scores, taken in fp32, are off by at most (hd + 4) 2^-24 d, which moves weights and their sum by twice that each (4 a
times it), and sums over n keys by at most (n + 64) 2^-24 (2 a times it).  lse: the scores' error, the sum's, and two
roundings of itself."""
import numpy as np
import pytest
import torch

from oracle import operators as oo

pytestmark = pytest.mark.gpu

DT = {0: torch.bfloat16, 1: torch.float16}
HALF = {0: 2.0 ** -8, 1: 2.0 ** -11}
MASK = {"full": 0, "causal": 1, "shadow": 2}


@pytest.fixture(scope="module")
def P():
    import paper_2605_16941_amd as pkg
    return pkg


class Problem:
    """Sequences of (rows, keys), their tensors on the host, and the oracle's answer."""

    def __init__(self, seqs, hq, hk, hd, act, mask="full", block=0, seed=0, std=1.5):
        rng = np.random.default_rng(seed)
        self.seqs, self.hq, self.hk, self.hd, self.act, self.mask, self.block = seqs, hq, hk, hd, act, mask, block
        t = lambda n, h, s=1.0: torch.from_numpy(rng.standard_normal((n, h, hd)) * s).to(DT[act])  # noqa: E731
        self.q = [t(n, hq, std) for n, _ in seqs]
        self.k, self.v = [t(m, hk) for _, m in seqs], [t(m, hk) for _, m in seqs]
        self.cur = [int(rng.integers(-1, max(1, m - 2 * block) + 1)) for _, m in seqs]
        self.scale = float(np.float32(hd ** -0.5))
        self.hidden = [np.zeros((n, m), bool) for n, m in seqs]  # keys that no mask hides but the test does

    def visible(self, b):
        n, m = self.seqs[b]
        return oo.sees(self.mask, n, m, self.block, self.cur[b]) & ~self.hidden[b]

    def params(self, P, **kw):
        return P.make_attn_params(self.hq, self.hk, self.hd, dtype=self.act, mask=MASK[self.mask], block_len=self.block,
                                  scale=self.scale, **kw)

    def i32(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def cu(self, which):
        return np.concatenate([[0], np.cumsum([s[which] for s in self.seqs])]).tolist()

    def cur_start(self):
        return self.i32(self.cur) if self.mask == "shadow" else None

    def workspace(self, P, p, total, max_kv):
        n = P.wino_attention_workspace_bytes(p, len(self.seqs), total, max_kv)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None

    def paged(self, P, page=16, order="token", extra=0, seed=0, tail=float("nan"), max_kv=None, stream=None):
        """The call with keys in shuffled pages, everything that is not a key being `tail`, and `extra` rows behind the
        last sequence."""
        rng = np.random.default_rng(seed + 100)
        used = [-(-m // page) for _, m in self.seqs]
        pages = sum(used) + 3
        ids = rng.permutation(pages)
        kc = torch.full((pages, page, self.hk, self.hd), tail, dtype=DT[self.act])
        vc = kc.clone()
        width = max(max(used), 1)
        table = np.full((len(used), width), 1 << 30)
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = ids[at:at + n]
            at += n
            for c, x in ((kc, self.k[b]), (vc, self.v[b])):
                m = x.shape[0]
                j = np.arange(m)
                c[table[b, j // page], j % page] = x
        self.table = table
        kc, vc = kc.cuda(), vc.cuda()
        if order == "head":
            kc, vc = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc))
        self.cache_tensors = kc, vc
        return self.call_paged(P, extra, max_kv, stream)

    def call_paged(self, P, extra=0, max_kv=None, stream=None):
        p = self.params(P)
        total = self.cu(0)[-1] + extra
        q = torch.full((total, self.hq, self.hd), float("nan"), dtype=DT[self.act])
        q[:total - extra] = torch.cat(self.q)
        out = torch.full((total, self.hq, self.hd), 3.0, dtype=DT[self.act], device="cuda")
        lse = torch.full((total, self.hq), 5.0, device="cuda")
        max_kv = max(m for _, m in self.seqs) if max_kv is None else max_kv
        ws = self.workspace(P, p, total, max_kv)
        args = (p, P.make_kv_cache(*self.cache_tensors), q.cuda(), out, self.i32(self.cu(0)),
                self.i32([m for _, m in self.seqs]), self.i32(self.table), max_kv)
        self.last = args, ws
        P.wino_paged_attention(*args, cur_start=self.cur_start(), lse=lse, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        if extra:
            assert (out[-extra:] == 3).all() and (lse[-extra:] == 5).all()
        return out[:total - extra], lse[:total - extra]

    def packed(self, P, extra=0):
        p = self.params(P)
        total, keys = self.cu(0)[-1] + extra, self.cu(1)[-1]
        # queries, keys and values as slices of fused products, NaN around them; the output in [heads, tokens] order
        fq = torch.full((total, self.hq + 1, self.hd), float("nan"), dtype=DT[self.act])
        fq[:total - extra, 1:] = torch.cat(self.q)
        fkv = torch.full((keys + 2, 2 * self.hk + 1, self.hd), float("nan"), dtype=DT[self.act])
        fkv[:keys, :self.hk], fkv[:keys, self.hk + 1:] = torch.cat(self.k), torch.cat(self.v)
        fq, fkv = fq.cuda(), fkv.cuda()
        out = torch.full((self.hq, total, self.hd), 3.0, dtype=DT[self.act], device="cuda").transpose(0, 1)
        lse = torch.full((total, self.hq), 5.0, device="cuda")
        max_kv = max(m for _, m in self.seqs)
        P.wino_packed_attention(p, fq[:, 1:], fkv[:, :self.hk], fkv[:, self.hk + 1:], out, self.i32(self.cu(0)),
                                self.i32(self.cu(1)), max_kv, cur_start=self.cur_start(), lse=lse,
                                workspace=self.workspace(P, p, total, max_kv))
        torch.cuda.synchronize()
        if extra:
            assert (out[-extra:] == 3).all() and (lse[-extra:] == 5).all()
        return out[:total - extra], lse[:total - extra]

    def check(self, got, only=None):
        out, lse = got[0].double().cpu().numpy(), got[1].double().cpu().numpy()
        at = 0
        for b, (n, m) in enumerate(self.seqs):
            if n and (only is None or b in only):
                vis = self.visible(b)
                q, k, v = (x[b].double().numpy() for x in (self.q, self.k, self.v))
                o, l, a, d = oo.attention(q, k, v, self.scale, vis)
                half = HALF[self.act]
                fp32 = (4 * (self.hd + 4) * d[..., None] + 2 * (m + 64)) * 2.0 ** -24
                vmax = np.abs(np.where(np.isfinite(v), v, 0)).max() if m else 0.0
                tol = half * (np.abs(o) + a) * 1.01 + fp32 * a + (m * 2.0 ** -25 * vmax + 2.0 ** -25 if self.act else 0)
                g, gl = out[at:at + n], lse[at:at + n]
                fin = np.isfinite(o)
                assert np.array_equal(np.isnan(g), np.isnan(o)), f"sequence {b}: NaN elsewhere"
                assert np.array_equal(g[np.isinf(o)], o[np.isinf(o)]) and np.isfinite(g[fin]).all()
                err = np.abs(g[fin] - o[fin]) - tol[fin]
                assert (err <= 0).all(), f"sequence {b} ({n} rows, {m} keys): {err.max()} over, at {np.argwhere(fin)[err.argmax()]}"
                empty = ~vis.any(1)
                assert (g[empty] == 0).all() and np.isneginf(gl[empty]).all()
                ltol = (2 * (self.hd + 4) * d + m + 64) * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(l))
                assert (np.abs(gl[~empty] - l[~empty]) <= ltol[~empty]).all(), f"sequence {b}: lse"
            at += n


HEADS = [(4, 4, 64, 0), (8, 2, 128, 1), (3, 1, 128, 0), (14, 2, 64, 1)]
TOKENS = [[(1, 1)], [(1, 97)], [(1, 0), (1, 63), (0, 40), (1, 64), (1, 65), (1, 1), (1, 700)],
          [(1, 2500), (1, 16), (1, 1025)]]
CHUNKS = [[(5, 5), (0, 0), (17, 33), (1, 64)], [(31, 200), (32, 129), (33, 128)], [(64, 700), (2, 500)],
          [(130, 130), (3, 900), (0, 77), (70, 64)], [(9, 2), (40, 0), (129, 127)]]


@pytest.mark.parametrize("hq,hk,hd,act", HEADS)
@pytest.mark.parametrize("seqs", TOKENS)
@pytest.mark.parametrize("page,order", [(16, "token"), (64, "head")])
def test_single_tokens_over_pages(P, hq, hk, hd, act, seqs, page, order):
    for mask in ("full", "causal"):
        pr = Problem(seqs, hq, hk, hd, act, mask, seed=len(seqs))
        pr.check(pr.paged(P, page, order, extra=2))


@pytest.mark.parametrize("hq,hk,hd,act", HEADS)
@pytest.mark.parametrize("seqs", CHUNKS)
@pytest.mark.parametrize("mask", ["full", "causal"])
def test_chunks(P, hq, hk, hd, act, seqs, mask):
    pr = Problem(seqs, hq, hk, hd, act, mask, seed=len(seqs))
    pr.check(pr.paged(P, 32, "head", extra=1))
    pr.check(pr.packed(P, extra=3))


@pytest.mark.parametrize("hq,hk,hd,act", HEADS)
@pytest.mark.parametrize("block,seqs", [(1, [(2, 2), (2, 70)]), (4, [(8, 8), (8, 131), (6, 40), (3, 9), (8, 3)]),
                                        (32, [(64, 64), (64, 300), (64, 97), (32, 64)]), (64, [(128, 600), (200, 200)])])
def test_shadow_mask(P, hq, hk, hd, act, block, seqs):
    pr = Problem(seqs, hq, hk, hd, act, "shadow", block, seed=block)
    pr.check(pr.paged(P, 16, extra=1))
    pr.check(pr.packed(P))


@pytest.mark.parametrize("hq,hk,hd,act,page", [(2, 1, 128, 0, 1024), (1, 1, 64, 1, 128)])
def test_long(P, hq, hk, hd, act, page):
    for seqs, mask in (([(700, 1500)], "causal"), ([(1, 20000), (3, 9000)], "full"), ([(1030, 1030)], "causal")):
        pr = Problem(seqs, hq, hk, hd, act, mask, seed=5)
        pr.check(pr.paged(P, page))


@pytest.mark.parametrize("batch", [64, 65, 200, 4200])
def test_many_sequences(P, batch):
    """More sequences than a wave has lanes (and more than 64 per lane), empty ones among them, in every position."""
    rng = np.random.default_rng(batch)
    seqs = [(int(n), int(m)) for n, m in zip(rng.integers(0, 3, batch), rng.integers(0, 30, batch))]
    seqs[-1] = (3, 300)
    pr = Problem(seqs, 2, 1, 64, 0, "causal")
    pr.check(pr.paged(P, 16, extra=1))
    pr.check(pr.packed(P))


def test_no_keys_at_all(P):
    pr = Problem([(3, 0), (70, 0)], 4, 2, 128, 1, "full")
    pr.check(pr.paged(P, 16, max_kv=0))
    pr.check(pr.packed(P))


def test_a_loose_bound_of_the_lengths(P):
    """max_kv_len far above every length: more chunks than there are, for few rows and for many."""
    for seqs in ([(1, 700), (1, 3)], [(40, 300), (5, 5)], [(200, 260)]):
        pr = Problem(seqs, 4, 2, 64, 0, "causal")
        pr.paged(P, 16)
        wide = np.full((len(seqs), 1 << 14), -1)
        wide[:, :pr.table.shape[1]] = pr.table
        pr.table = wide
        pr.check(pr.call_paged(P, max_kv=1 << 18))


def test_one_key_heavier_than_all(P):
    """A late key far above the others (the running maximum moves by more than any exponent's range) and scores of
    hundreds in both directions."""
    pr = Problem([(40, 500), (1, 500)], 4, 2, 64, 0, std=1.0)
    for b in range(2):
        pr.k[b][450] = (pr.q[b][-1, 0::2] * 40).to(pr.k[b].dtype)
        pr.k[b][3] = (pr.q[b][-1, 0::2] * -40).to(pr.k[b].dtype)
    pr.check(pr.paged(P))
    pr.check(pr.packed(P))


@pytest.mark.parametrize("mask", ["causal", "shadow", "full"])
@pytest.mark.parametrize("act,hd", [(0, 128), (1, 64)])
def test_values_of_unseen_keys_do_not_reach_a_row(P, mask, act, hd):
    """Infinities and NaN among the values at keys that later rows (causal) or other rows (shadow) see, and rows see
    them exactly where they see the key."""
    pr = Problem([(140, 150), (64, 90), (6, 300), (2, 70)], 4, 2, hd, act, mask, block=2 if mask == "shadow" else 0)
    if mask == "full":
        pr.seqs = pr.seqs[:]
    pr.cur = [100, 30, 250, 60]
    for b, (n, m) in enumerate(pr.seqs):
        j = {"causal": m - 2, "shadow": pr.cur[b] + 1, "full": m - 1}[mask]
        pr.v[b][j, 0, 3], pr.v[b][j, 1, 7], pr.v[b][j, 0, 40] = float("inf"), float("nan"), -float("inf")
        if mask == "shadow":
            pr.v[b][m - 1, 0, 5] = float("inf")  # a shadow key: the other rows do not see it
    pr.check(pr.paged(P, 16))
    pr.check(pr.packed(P))


def test_a_nan_key_stays_with_the_rows_that_see_it(P):
    pr = Problem([(70, 80), (3, 40)], 4, 2, 64, 0, "causal")
    good = Problem([(70, 80), (3, 40)], 4, 2, 64, 0, "causal")
    pr.k[0][60], pr.q[0][69] = float("nan"), float("inf")
    for call in (lambda p: p.paged(P, 32), lambda p: p.packed(P)):
        bad, ok = call(pr), call(good)
        first = 60 - 10  # the first row that sees key 60
        assert torch.equal(bad[0][:first], ok[0][:first]) and torch.equal(bad[0][70:], ok[0][70:])
        assert bad[0][first:70].isnan().all() and torch.equal(bad[1][:first], ok[1][:first])


@pytest.mark.parametrize("page", [16, 64])
def test_pages_with_bad_ids_are_not_seen(P, page):
    """Page ids outside the cache among a sequence's pages: their keys are skipped (ids just outside and far outside)."""
    for seqs in ([(1, 500), (1, 300)], [(40, 260), (100, 200)]):
        pr = Problem(seqs, 4, 2, 64, 0, "causal")
        pr.paged(P, page)
        pages = pr.cache_tensors[0].shape[0]
        for b, (n, m) in enumerate(seqs):
            for at, bad in ((1, -1), (2, pages), (3, -(1 << 31))):
                pr.table[b, at] = bad
                pr.hidden[b][:, at * page:(at + 1) * page] = True
        pr.check(pr.call_paged(P))


def test_lengths_are_cut_to_what_the_host_knows(P):
    """Keys past max_kv_len are not read (causal rows are then the last of the cut length), and lengths below zero or
    row offsets past total_q hold no memory outside the tensors."""
    pr = Problem([(2, 100), (1, 60)], 4, 4, 64, 0)
    pr.paged(P, 16)
    for b in range(2):
        pr.hidden[b][:, 50:] = True
    pr.check(pr.call_paged(P, max_kv=50))
    args, ws = pr.last
    out = torch.full_like(args[3], 3.0)
    args = args[:3] + (out, pr.i32([0, 2, 1 << 20]), pr.i32([-5, 60])) + args[6:]
    P.wino_paged_attention(*args, workspace=ws)
    torch.cuda.synchronize()
    assert (out[:2] == 0).all() and torch.isfinite(out[2:]).all()


def test_first_sequence_may_start_late(P):
    pr = Problem([(4, 40), (40, 50)], 4, 2, 64, 1, "causal")
    want = pr.paged(P, 16)
    args, ws = pr.last
    q = torch.cat([torch.full_like(args[2][:5], float("nan")), args[2]])
    out = torch.full_like(q, 3.0)
    P.wino_paged_attention(*args[:2], q, out, args[4] + 5, *args[5:], workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out[5:], want[0]) and (out[:5] == 3).all()


def test_repeated_inputs_and_broadcast_keys(P):
    """Every key and head the same row (strides of 0): any weighting gives the value back."""
    n, hd = 70, 64
    q = torch.randn(n, 4, hd, device="cuda").bfloat16()
    row = torch.randn(1, 1, hd, device="cuda").bfloat16()
    kv = row.expand(n, 2, hd)
    out = torch.empty_like(q)
    cu = torch.tensor([0, 30, n], dtype=torch.int32, device="cuda")
    p = P.make_attn_params(4, 2, hd, mask=P.MASK_CAUSAL)
    need = P.wino_attention_workspace_bytes(p, 2, n, n)
    P.wino_packed_attention(p, q, kv, kv, out, cu, cu, n,
                            workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    assert torch.allclose(out.float(), row.float().expand_as(out), rtol=2.0 ** -7, atol=0)


def test_same_bits_again_on_other_streams_and_in_a_graph(P):
    """The same call twice at once on two streams with workspaces of their own, and captured and replayed with lengths
    and pages that change between the replays: all the bits of an eager call."""
    pr = Problem([(1, 1800), (1, 300), (1, 5)], 8, 2, 128, 0)
    want = pr.paged(P, 16)
    args, ws = pr.last
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(args[3]) for _ in streams]
    spaces = [None if ws is None else torch.empty_like(ws) for _ in streams]
    torch.cuda.synchronize()
    for st, o, w in zip(streams, outs, spaces):
        with torch.cuda.stream(st):
            P.wino_paged_attention(*args[:3], o, *args[4:], workspace=w)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) for o in outs)

    q, out, kv_len = args[2].clone(), torch.empty_like(args[3]), args[5].clone()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st), torch.cuda.graph(graph, stream=st):
        P.wino_paged_attention(*args[:2], q, out, args[4], kv_len, *args[6:], workspace=ws)
    for lens in ([1800, 300, 5], [17, 299, 0], [1024, 1, 3], [1800, 300, 5]):
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(torch.randn_like(q.float()).to(q.dtype))
        out.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(out)
        P.wino_paged_attention(*args[:2], q, eager, args[4], kv_len, *args[6:],
                               workspace=None if ws is None else torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_two_graphs_with_one_workspace(P):
    """Two captured calls share a workspace; replayed one after the other in both orders they equal the eager calls."""
    problems = [Problem([(1, 3000), (1, 900)], 8, 2, 64, 1, seed=1), Problem([(2, 2500), (1, 40)], 4, 1, 128, 0, seed=2)]
    wants = [pr.paged(P, 32)[0].clone() for pr in problems]
    calls = [pr.last for pr in problems]
    need = max(0 if ws is None else ws.numel() for _, ws in calls)
    assert need  # both are split
    shared = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    st, graphs = torch.cuda.Stream(), []
    for (args, ws), pr in zip(calls, problems):
        assert ws is not None
        g = torch.cuda.CUDAGraph()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st), torch.cuda.graph(g, stream=st):
            P.wino_paged_attention(*args, workspace=shared)
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for i in order:
            calls[i][0][3].fill_(7)
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in set(order):
            assert torch.equal(calls[i][0][3], wants[i])


def test_cache_beyond_32_bits(P):
    """Pages past element 2^32 of the cache."""
    hk, hd, page = 2, 64, 128
    pages = (1 << 32) // (page * hk * hd) + 3
    pr = Problem([(1, 300), (40, 200)], 4, hk, hd, 1, "causal")
    pr.paged(P, page)
    small = pr.cache_tensors
    pr.cache_tensors = tuple(torch.empty(pages, page, hk, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    for big, c in zip(pr.cache_tensors, small):
        big[-c.shape[0]:] = c
    pr.table = np.where(pr.table < (1 << 30), pr.table + pages - small[0].shape[0], pr.table)
    pr.check(pr.call_paged(P))


def test_prompt_then_blocks_then_tokens(P):
    """The operators together, as a program with a cache uses them: ragged prompts are rotated and written to pages while
    they attend to themselves packed; then chunks and single tokens are appended and attend over the cache.  Every
    output equals one oracle attention over the whole sequence; the keys it is given are the rotated rows rounded to
    the type, as the cache holds them."""
    hq, hk, hd, act, page = 6, 2, 64, 1, 16
    lens, steps = [37, 5, 80], [9, 1, 1]
    rng = np.random.default_rng(9)
    t = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, hd))).to(DT[act])  # noqa: E731
    B, total = len(lens), sum(lens)
    freq, mag = P.wino_rope_frequencies(32, 10000.0, P.ROPE_SCALE_PARTS, 4.0, orig_len=64, turns_fast=8)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda")
    rp = P.make_rope_params(hd, 32, P.ROPE_INTERLEAVED, dtype=act, magnitude=mag)
    width = -(-(max(lens) + sum(steps)) // page)
    table = torch.from_numpy(rng.permutation(B * width).reshape(B, width)).to(torch.int32)
    kc = torch.full((B * width, page, hk, hd), float("nan"), dtype=DT[act], device="cuda")
    vc = kc.clone()
    cache = P.make_kv_cache(kc, vc)
    keys, values, done = [t(0, hk) for _ in lens], [t(0, hk) for _ in lens], [0] * B
    for step, new in enumerate([lens] + [[s] * B for s in steps]):
        n = sum(new)
        q, k, v = t(n, hq), t(n, hk), t(n, hk)
        pos = np.concatenate([done[b] + np.arange(m) for b, m in enumerate(new)])
        seq = np.repeat(np.arange(B), new)
        slot = torch.from_numpy(table.numpy()[seq, pos // page].astype(np.int64) * page + pos % page).cuda()
        q_out = torch.empty(n, hq, hd, dtype=DT[act], device="cuda")
        vd = v.cuda()
        P.wino_rope_append(rp, cache, fd, torch.from_numpy(pos).to(torch.int32).cuda(), slot, q.cuda(), k.cuda(), vd,
                           q_out)
        rk = kc.flatten(0, 1)[slot]
        qr = oo.rope(q.double().numpy(), pos, freq, 32, True, mag)
        assert (np.abs(q_out.double().cpu().numpy() - qr) <= 2.0 ** -10 * (np.abs(qr) + 0.01)).all()
        cu = np.concatenate([[0], np.cumsum(new)])
        done = [d + m for d, m in zip(done, new)]
        pr = Problem([(m, d) for m, d in zip(new, done)], hq, hk, hd, act, "causal")
        for b in range(B):
            keys[b] = torch.cat([keys[b], rk.cpu()[cu[b]:cu[b + 1]]])
            values[b] = torch.cat([values[b], v[cu[b]:cu[b + 1]]])
        pr.q = [q_out.cpu()[cu[b]:cu[b + 1]] for b in range(B)]
        pr.k, pr.v = keys, values
        p = pr.params(P)
        out, lse = torch.empty_like(q_out), torch.empty(n, hq, device="cuda")
        ws = pr.workspace(P, p, n, max(done))
        cud = pr.i32(cu.tolist())
        P.wino_paged_attention(p, cache, q_out, out, cud, pr.i32(done), table.cuda(), max(done), lse=lse, workspace=ws)
        pr.check((out, lse))
        if step == 0:
            out2 = torch.empty_like(out)
            P.wino_packed_attention(p, q_out, rk, vd, out2, cud, cud, max(lens), lse=lse, workspace=ws)
            pr.check((out2, lse))


def split(pr):
    """Whether the last paged call cut the keys into chunks: partial outputs are in its workspace."""
    ws = pr.last[1]
    return ws is not None and bool((ws != 0xFF).any())


@pytest.mark.parametrize("act,hd", [(0, 128), (1, 64)])
@pytest.mark.parametrize("n", [1, 20, 100])
def test_nan_at_a_key_far_below_the_maximum_in_another_chunk(P, n, act, hd):
    """A row's output is over all keys it sees: NaN among the values of a key whose weight is far below the smallest
    fp32 number (scores of 300 and more between them) reaches the row from another chunk than the heavy key's, in tiles
    of 32, 64 and 128 rows."""
    pr = Problem([(n, 1100)], 4, 2, hd, act, "causal", seed=n)
    pr.q[0][..., 0] = 16
    pr.k[0][30, :, 0] = 256
    pr.v[0][700, 0, 3], pr.v[0][600, 1, 7] = float("nan"), float("nan")
    pr.check(pr.paged(P, 16))
    assert split(pr)
    pr.check(pr.packed(P))


@pytest.mark.parametrize("mask", ["causal", "shadow", "full"])
@pytest.mark.parametrize("act,hd", [(0, 128), (1, 64)])
@pytest.mark.parametrize("n", [2, 20, 200])
def test_unseen_values_stay_out_of_chunks(P, n, act, hd, mask):
    """Infinities and NaN among the values where a sequence is cut into chunks, in tiles of 32, 64 and 128 rows: at keys
    that every row sees, that some rows see, in a chunk that whole tiles do not see, and at the last key."""
    m, block = 1100, {2: 1, 20: 8, 200: 64}[n]
    pr = Problem([(n, m)], 4, 2, hd, act, mask, block=block if mask == "shadow" else 0, seed=n)
    pr.cur = [500]
    inf, nan = float("inf"), float("nan")
    for j, e in ((300, 1), (m - 2, 3), (m - n // 2, 5), (m - 1 - n // 8, 7), (500 + block // 2, 9), (m - 1, 11)):
        pr.v[0][j, 0, e], pr.v[0][j, 0, e + 40], pr.v[0][j, 1, e + 1] = inf, nan, -inf
    pr.check(pr.paged(P, 16))
    assert split(pr)
    pr.check(pr.packed(P))


@pytest.mark.parametrize("n", [1, 20, 200])
@pytest.mark.parametrize("page", [16, 64])
def test_chunks_of_pages_with_bad_ids(P, n, page):
    """Pages with ids outside the cache, where a sequence is cut into chunks: one, all of a chunk's, all of the table."""
    pr = Problem([(n, 1100)], 4, 2, 64, 0, "causal", seed=n)
    pr.paged(P, page)
    pages = pr.cache_tensors[0].shape[0]
    for lo, hi, bad in ((900 // page, 900 // page + 1, pages), (256 // page, 512 // page, -1), (0, 1100, (1 << 31) - 1)):
        pr.table[:, lo:hi] = bad
        pr.hidden[0][:, lo * page:hi * page] = True
        pr.check(pr.call_paged(P))
        assert split(pr)


@pytest.mark.parametrize("n", [1, 20, 200])
def test_one_key_heavier_than_all_in_its_chunk(P, n):
    """A key far above the others in one chunk, and far below them in another: the join's weights span all exponents."""
    pr = Problem([(n, 1100)], 4, 2, 64, 1, "causal", seed=n)
    pr.k[0][700] = (pr.q[0][-1, 0::2] * 40).to(pr.k[0].dtype)
    pr.k[0][100] = (pr.q[0][-1, 0::2] * -40).to(pr.k[0].dtype)
    pr.check(pr.paged(P))
    assert split(pr)
    pr.check(pr.packed(P))


def test_one_workspace_for_the_largest_sizes(P):
    """Memory for a program's largest sizes, which are not split, serves smaller calls, which are, and nothing behind it
    is written."""
    heads, hd, batch, total, keys = (4, 2), 128, 64, 4096, 1500
    need = P.wino_attention_workspace_bytes(P.make_attn_params(*heads, hd), batch, total, keys)
    memory = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    ran_split = 0
    for n, m in ((1, 1500), (1, 1100), (3, 900), (33, 1400), (130, 1200), (9, 300)):
        pr = Problem([(n, m), (1, 7)], *heads, hd, 0, "causal", seed=n)
        pr.workspace = lambda P, p, total, max_kv: memory[:need]
        memory.fill_(0xFF)
        pr.check(pr.paged(P, 32))
        ran_split += split(pr)
        assert (memory[need:] == 0xFF).all()
    assert ran_split >= 4


def test_a_bound_of_the_lengths_beyond_32_bits_is_refused(P):
    pr = Problem([(2, 100)], 4, 4, 64, 0)
    pr.paged(P, 16)
    args, ws = pr.last
    for bound in ((1 << 32) + 50, 1 << 40, (1 << 63) + 100):
        with pytest.raises(P.WinoError) as e:
            P.wino_paged_attention(*args[:7], bound, workspace=ws)
        assert e.value.status == -2
        with pytest.raises(P.WinoError) as e:
            P.wino_packed_attention(args[0], args[2], args[2], args[2], args[3], args[4], args[4], bound, workspace=ws)
        assert e.value.status == -2


def test_page_tables_inside_a_wider_one(P):
    """The entries in use of a table with room for more, rows of a larger table, a table of one column."""
    pr = Problem([(2, 100), (40, 61), (1, 9)], 4, 2, 64, 0, "causal")
    want = pr.paged(P, 16)
    args, ws = pr.last
    table, out = args[6], torch.empty_like(args[3])
    wide = torch.full((7, table.shape[1] + 9), -1, dtype=torch.int32, device="cuda")
    for rows, first in ((slice(0, 3), 0), (slice(1, 7, 2), 5)):
        wide.fill_(-1)
        view = wide[rows, first:first + table.shape[1]]
        view.copy_(table)
        out.fill_(3)
        P.wino_paged_attention(*args[:3], out, *args[4:6], view, args[7], workspace=ws)
        assert torch.equal(out, want[0])
    for view in (wide.t()[:3, :7], wide[:3, ::2], wide[:1, :7].expand(3, 7)[:, None, :]):
        with pytest.raises(ValueError):
            P.wino_paged_attention(*args[:3], out, *args[4:6], view, args[7], workspace=ws)
    pr = Problem([(2, 16), (3, 5)], 4, 2, 64, 0, "causal")
    want = pr.paged(P, 16)
    args, ws = pr.last
    P.wino_paged_attention(*args[:6], args[6].expand(-1, 1).t().contiguous().t(), args[7], workspace=ws)
    wide[:2, 4:5] = args[6]
    out = torch.empty_like(args[3])
    P.wino_paged_attention(*args[:3], out, *args[4:6], wide[:2, 4:5], args[7], workspace=ws)
    assert torch.equal(out, want[0]) and torch.equal(args[3], want[0])


@pytest.mark.parametrize("n,m", [(130, 200), (3, 1100), (130, 1100)])
def test_offsets_in_any_order_stay_inside(P, n, m):
    """Offsets that do not ascend and lengths of any sign: rows may be anything, but nothing around the outputs and the
    workspace is written, and a later call is right."""
    pr = Problem([(n, m), (1, 9), (7, m // 2)], 4, 2, 64, 0, "causal", seed=n)
    want = pr.paged(P, 16)
    args, _ = pr.last
    total = args[2].shape[0]
    need = P.wino_attention_workspace_bytes(args[0], 3, total, m)
    memory = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    ws = memory[:need] if need else None
    rng = np.random.default_rng(n)
    for _ in range(6):
        cu = pr.i32(rng.integers(-5, total + 50, 4).tolist())
        lens = pr.i32(rng.integers(-5, m + 50, 3).tolist())
        space = torch.full((total + 2, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((total + 2, 4), 5.0, device="cuda")
        P.wino_paged_attention(*args[:3], space[1:-1], cu, lens, *args[6:], lse=lse[1:-1], workspace=ws)
        P.wino_packed_attention(args[0], args[2], args[2][:, :2], args[2][:, 2:], space[1:-1], cu, cu.flip(0), m,
                                lse=lse[1:-1], workspace=ws)
        torch.cuda.synchronize()
        assert (space[0] == 3).all() and (space[-1] == 3).all() and (lse[0] == 5).all() and (lse[-1] == 5).all()
        assert (memory[need:] == 0xFF).all()
    out = torch.empty_like(args[3])
    P.wino_paged_attention(*args[:3], out, *args[4:], workspace=ws)
    assert torch.equal(out, want[0])


@pytest.mark.parametrize("seqs", [[(300, 300), (70, 70)], [(600, 600)], [(1, 400), (1, 300)]])
def test_calls_that_are_not_split_need_no_workspace(P, seqs):
    """Where keys are not cut into chunks a call runs without memory, though smaller calls of the same program need some."""
    pr = Problem(seqs, 4, 2, 64, 0, "causal")
    assert P.wino_attention_workspace_bytes(pr.params(P), len(seqs), pr.cu(0)[-1], pr.seqs[0][1]) > 0
    pr.check(pr.paged(P, 16))
    assert not split(pr)
    pr.workspace = lambda *a: None
    pr.check(pr.paged(P, 16))
    pr.check(pr.packed(P))
