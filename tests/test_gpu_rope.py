"""Rotary positions and the cache write against the float64 oracle.

Tolerance, from arithmetic: y = m (x_a cos - x_b sin) is formed in fp32 and rounded once, so it is off by at most half a
step of the type (eps/2 |y|, or half the smallest step near zero) plus the fp32 error of the sine and cosine (a fraction
of a turn rounded to 2^-25, and two steps of the function: below 2^-21) times m (|x_a| + |x_b|), and two fp32 roundings
of the products, below 2^-22 of the same."""
import numpy as np
import pytest
import torch

from oracle import operators as oo

pytestmark = pytest.mark.gpu

DT = {0: torch.bfloat16, 1: torch.float16}
STEP = {0: 2.0 ** -8, 1: 2.0 ** -11}
LEAST = {0: 0.0, 1: 2.0 ** -25}


@pytest.fixture(scope="module")
def P():
    import paper_2605_16941_amd as pkg
    return pkg


def rows(rng, n, h, hd, act):
    return torch.from_numpy(rng.standard_normal((n, h, hd))).to(DT[act])


def check(got, x, pos, freq, rot, act, mag=1.0, **kw):
    ref = oo.rope(x.double().numpy(), pos.numpy(), freq, rot, magnitude=mag, **kw)
    near = np.abs(x.double().numpy()).max(-1, keepdims=True) * 2 * abs(mag)
    tol = STEP[act] * np.abs(ref) * (1 + STEP[act]) + LEAST[act] + 2.0 ** -20 * near
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("inter", [0, 1])
@pytest.mark.parametrize("n,h,hd,rot", [(1, 1, 64, 64), (3, 4, 64, 16), (5, 7, 128, 128), (131, 3, 128, 48), (67, 33, 64, 32),
                                        (2500, 5, 128, 112)])
def test_rope_forward_inverse_in_place(P, act, inter, n, h, hd, rot):
    rng = np.random.default_rng(n + rot)
    x = rows(rng, n, h, hd, act)
    freq, _ = P.wino_rope_frequencies(rot, 10000.0)
    far = 2 ** 31 - 1
    pos = torch.from_numpy(rng.integers(-far - 1, far, n)).to(torch.int32)
    pos[0] = far
    if n > 2:
        pos[1], pos[2] = 0, -far - 1
    fd, pd = torch.tensor(freq, dtype=torch.float64, device="cuda"), pos.cuda()
    for inverse in (False, True):
        p = P.make_rope_params(hd, rot, inter, dtype=act, magnitude=1.25, inverse=inverse)
        # a slice of a fused product, and an output in [heads, tokens] order inside a larger tensor
        fused = torch.zeros(n, h + 2, hd, dtype=DT[act], device="cuda")
        fused[:, 1:h + 1] = x.cuda()
        out = torch.full((h + 1, n, hd), 7.0, dtype=DT[act], device="cuda")
        P.wino_rope(p, fd, pd, fused[:, 1:h + 1], out[:h].transpose(0, 1))
        check(out[:h].transpose(0, 1), x, pos, freq, rot, act, 1.25, interleaved=bool(inter), inverse=inverse)
        assert (out[h] == 7).all() and (fused[:, 0] == 0).all() and (fused[:, h + 1] == 0).all()
        y = x.cuda()
        P.wino_rope(p, fd, pd, y, y)
        assert torch.equal(y, out[:h].transpose(0, 1))


def test_rope_is_the_gradient_of_itself(P):
    """<rope(x), g> = <x, inverse(g)>, and the directional difference of rope at x along d is rope(d): both to the sum of
    the roundings, half a step of each product's term."""
    rng = np.random.default_rng(3)
    n, h, hd = 40, 3, 64
    x, g, d = (rows(rng, n, h, hd, 1).cuda() for _ in range(3))
    freq = torch.tensor(P.wino_rope_frequencies(48, 10000.0)[0], dtype=torch.float64, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 31
    fwd, back = (P.make_rope_params(hd, 48, dtype=1, inverse=i) for i in (False, True))

    def rope(p, t):
        o = torch.empty_like(t)
        P.wino_rope(p, freq, pos, t, o)
        return o.double()

    y, gx = rope(fwd, x), rope(back, g)
    lhs, rhs = (y * g.double()).sum(), (x.double() * gx).sum()
    tol = 2.0 ** -10 * ((y * g.double()).abs().sum() + (x.double() * gx).abs().sum())
    assert abs(lhs - rhs) <= tol
    step = 0.25  # exact in the type for d and for x + step d up to its own rounding
    xp = (x.double() + step * d.double()).to(torch.float16)
    diff = (rope(fwd, xp) - y) / step
    moved = (xp.double() - x.double()) / step
    want = torch.from_numpy(oo.rope(moved.cpu().numpy(), pos.cpu().numpy(), freq.cpu().numpy(), 48)).cuda()
    assert ((diff - want).abs() <= 2.0 ** -10 / step * 1.01 * torch.maximum(y.abs(), rope(fwd, xp).abs()) + 1e-4).all()


@pytest.mark.parametrize("act,hd,hq,hk,page,order", [(0, 64, 4, 4, 16, "token"), (1, 128, 8, 2, 64, "head"),
                                                     (0, 128, 5, 5, 32, "head"), (1, 64, 9, 3, 1024, "token")])
@pytest.mark.parametrize("n", [1, 19, 300])
def test_append_writes_its_slots_and_nothing_else(P, act, hd, hq, hk, page, order, n):
    rng = np.random.default_rng(n)
    pages = -(-n // page) + 3
    shape = (pages, page, hk, hd) if order == "token" else (pages, hk, page, hd)
    kc, vc = (torch.from_numpy(rng.standard_normal(shape)).to(DT[act]).cuda() for _ in range(2))
    view = (lambda t: t) if order == "token" else (lambda t: t.transpose(1, 2))
    before = view(kc).clone(), view(vc).clone()
    qkv = rows(rng, n, hq + 2 * hk, hd, act)
    dev = qkv.cuda()
    slot = torch.from_numpy(rng.permutation(pages * page)[:n])
    if n > 3:  # rows that are not written: padding, and slots behind the cache
        slot[0], slot[1], slot[2] = -1, pages * page, 1 << 40
    freq, _ = P.wino_rope_frequencies(hd, 500000.0)
    pos = torch.from_numpy(rng.integers(0, 5000, n)).to(torch.int32)
    q_out = torch.empty(n, hq, hd, dtype=DT[act], device="cuda")
    p = P.make_rope_params(hd, dtype=act)
    P.wino_rope_append(p, P.make_kv_cache(view(kc), view(vc)), torch.tensor(freq, dtype=torch.float64, device="cuda"),
                       pos.cuda(), slot.cuda(), dev[:, :hq], dev[:, hq:hq + hk], dev[:, hq + hk:], q_out)
    check(q_out, qkv[:, :hq], pos, freq, hd, act)
    ok = (slot >= 0) & (slot < pages * page)
    s = slot[ok]
    k, v = view(kc).cpu(), view(vc).cpu()
    check(k[s // page, s % page], qkv[ok, hq:hq + hk], pos[ok], freq, hd, act)
    assert torch.equal(v[s // page, s % page], qkv[ok, hq + hk:])
    kb, vb = before[0].cpu(), before[1].cpu()
    kb[s // page, s % page], vb[s // page, s % page] = k[s // page, s % page], v[s // page, s % page]
    assert torch.equal(k, kb) and torch.equal(v, vb)


def test_append_in_place_of_the_queries(P):
    """q_out = q, on a stream given by argument, inside a fused product whose keys and values stay as they are."""
    n, hq, hk, hd = 37, 6, 2, 64
    rng = np.random.default_rng(4)
    qkv = rows(rng, n, hq + 2 * hk, hd, 1)
    dev = qkv.cuda()
    kc, vc = (torch.zeros(4, 16, hk, hd, dtype=torch.float16, device="cuda") for _ in range(2))
    freq, _ = P.wino_rope_frequencies(hd, 1e4, P.ROPE_SCALE_BASE, 4.0)
    pos = torch.arange(n, dtype=torch.int32)
    st = torch.cuda.Stream()
    slot = torch.arange(n, device="cuda") + 5
    fd, pd = torch.tensor(freq, dtype=torch.float64, device="cuda"), pos.cuda()
    torch.cuda.synchronize()
    P.wino_rope_append(P.make_rope_params(hd, dtype=1), P.make_kv_cache(kc, vc), fd, pd, slot, dev[:, :hq],
                       dev[:, hq:hq + hk], dev[:, hq + hk:], dev[:, :hq], stream=st)
    torch.cuda.synchronize()
    check(dev[:, :hq], qkv[:, :hq], pos, freq, hd, 1)
    assert torch.equal(dev[:, hq:].cpu(), qkv[:, hq:])
    check(kc.flatten(0, 1)[5:5 + n].cpu(), qkv[:, hq:hq + hk], pos, freq, hd, 1)
    assert torch.equal(vc.flatten(0, 1)[5:5 + n].cpu(), qkv[:, hq + hk:])


def test_append_beyond_32_bits(P):
    """A cache of more than 2^32 elements: the last page's rows are where they belong."""
    hk, hd, page = 2, 128, 64
    pages = (1 << 32) // (page * hk * hd) + 2
    kc = torch.empty(pages, page, hk, hd, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    kc[-1], vc[-1], kc[1], vc[1] = 0, 0, 0, 0
    x = torch.randn(2, 3 * hk, hd, device="cuda").bfloat16()
    slot = torch.tensor([pages * page - 1, pages * page - page], device="cuda")
    freq = torch.tensor(P.wino_rope_frequencies(hd, 1e4)[0], dtype=torch.float64, device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    P.wino_rope_append(P.make_rope_params(hd), P.make_kv_cache(kc, vc), freq, pos, slot, x[:, :hk], x[:, hk:2 * hk],
                       x[:, 2 * hk:], torch.empty(2, hk, hd, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(kc[-1, -1], x[0, hk:2 * hk]) and torch.equal(vc[-1, -1], x[0, 2 * hk:])
    assert torch.equal(kc[-1, 0], x[1, hk:2 * hk]) and torch.equal(vc[-1, 0], x[1, 2 * hk:])
    assert not kc[1].any() and not vc[1].any() and not kc[-1, 1:-1].any()
