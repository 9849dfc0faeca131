"""Operators on a caller's own tensors, without a GPU: every refusal happens on the host before any GPU work, the
rotary frequencies equal their formulas, and the oracle agrees with independent forms of itself."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import operators as oo

PTR = 0x10000  # never dereferenced: each call below is refused first


@pytest.fixture(scope="module")
def abi():
    from paper_2605_16941_amd import _abi
    return _abi


def heads(abi, data=PTR, ts=512, hs=64):
    return abi.wino_heads(data, ts, hs)


def cache(abi, **kw):
    base = dict(k=PTR, v=PTR, page_stride=16 * 256, token_stride=256, head_stride=64, n_pages=8, page_size=16,
                n_kv_heads=4, head_dim=64, dtype=0)
    base.update(kw)
    return abi.wino_kv_cache(*base.values())


def test_struct_sizes_match_header_layout(abi):
    assert C.sizeof(abi.wino_heads) == 24 and C.sizeof(abi.wino_kv_cache) == 64
    assert C.sizeof(abi.wino_rope_params) == 24 and C.sizeof(abi.wino_rope_config) == 48
    assert C.sizeof(abi.wino_attn_params) == 28


ROPE = dict(head_dim=64, rotary_dim=64, layout=0, dtype=0, inverse=0, magnitude=1.0)


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=96), -6), (dict(rotary_dim=0), -2), (dict(rotary_dim=80), -2), (dict(rotary_dim=24), -6),
    (dict(layout=2), -1), (dict(dtype=2), -1), (dict(magnitude=math.inf), -1), (dict(n=-1), -2), (dict(n=1 << 26), -2),
    (dict(h=0), -2), (dict(freq=None), -1), (dict(pos=None), -1), (dict(x=None), -1), (dict(x=(None, 512, 64)), -1),
    (dict(x=(PTR + 2, 512, 64)), -6), (dict(x=(PTR, 511, 64)), -6), (dict(x=(PTR, -512, 64)), -6),
    (dict(x=(PTR, 512, 65)), -6), (dict(out=(PTR, 56, 64)), -2), (dict(out=(PTR, 512, 0)), -2)])
def test_rope_refusals(abi, change, status):
    a = dict(n=5, h=4, freq=PTR, pos=PTR, x=(PTR, 512, 64), out=(PTR, 512, 64))
    p = dict(ROPE)
    for key, val in change.items():
        (a if key in a else p)[key] = val
    prm = abi.wino_rope_params(*p.values())
    x, out = (C.byref(heads(abi, *t)) if t else None for t in (a["x"], a["out"]))
    assert abi.lib.wino_rope(C.byref(prm), a["n"], a["h"], a["freq"], a["pos"], x, out, None) == status


def append(abi, cache_args=None, p=None, q=None, k=None, slot=PTR, n=5):
    prm = abi.wino_rope_params(*{**ROPE, **(p or {})}.values())
    c = cache(abi, **(cache_args or {}))
    hq, hk = heads(abi, *(q or (PTR, 512, 64))), heads(abi, *(k or (PTR, 512, 64)))
    return abi.lib.wino_rope_append(C.byref(prm), C.byref(c), n, 4, PTR, PTR, slot, C.byref(hq), C.byref(hk),
                                    C.byref(hk), C.byref(hq), None)


@pytest.mark.parametrize("kw,status", [
    (dict(p=dict(inverse=1)), -1), (dict(slot=None), -1), (dict(cache_args=dict(k=None)), -1),
    (dict(cache_args=dict(dtype=1)), -1), (dict(cache_args=dict(dtype=7)), -1), (dict(cache_args=dict(n_pages=0)), -2),
    (dict(cache_args=dict(page_size=24)), -6), (dict(cache_args=dict(page_size=8)), -6),
    (dict(cache_args=dict(page_size=2048)), -6), (dict(cache_args=dict(head_dim=128, head_stride=128)), -2),
    (dict(cache_args=dict(n_kv_heads=0)), -2), (dict(cache_args=dict(head_stride=0)), -2),
    (dict(cache_args=dict(token_stride=8)), -2), (dict(cache_args=dict(page_stride=0)), -2),
    (dict(cache_args=dict(page_stride=-4096)), -6), (dict(cache_args=dict(v=PTR + 8)), -6),
    (dict(k=(PTR, 510, 64)), -6), (dict(q=(PTR, 0, 64)), -2)])
def test_append_refusals(abi, kw, status):
    assert append(abi, **kw) == status


def test_no_rows_is_no_work(abi):
    """Calls without rows return before any GPU work (which has no device here)."""
    assert append(abi, n=0) == 0
    assert paged(abi, total_q=0) == 0
    assert packed(abi, total_q=0) == 0


ATTN = dict(n_heads=8, n_kv_heads=4, head_dim=64, dtype=0, mask=0, block_len=0, scale=0.125)


def attn_params(abi, kw):
    p = {**ATTN, **{k: v for k, v in kw.items() if k in ATTN}}
    return abi.wino_attn_params(*p.values()), {k: v for k, v in kw.items() if k not in ATTN}


def paged(abi, **kw):
    p, kw = attn_params(abi, kw)
    a = dict(batch=2, total_q=7, max_kv=96, cu_q=PTR, kv_len=PTR, table=PTR, table_stride=6, width=6, cur=None,
             q=(PTR, 512, 64), out=(PTR, 512, 64), ws=PTR, ws_bytes=1 << 40, cache={})
    a.update(kw)
    c, q, out = cache(abi, **a["cache"]), heads(abi, *a["q"]), heads(abi, *a["out"])
    return abi.lib.wino_paged_attention(C.byref(p), C.byref(c), a["batch"], a["total_q"], a["max_kv"], a["cu_q"],
                                        a["kv_len"], a["table"], a["table_stride"], a["width"], a["cur"], C.byref(q),
                                        C.byref(out), None, a["ws"], a["ws_bytes"], None)


def packed(abi, **kw):
    p, kw = attn_params(abi, kw)
    a = dict(batch=2, total_q=7, total_k=7, max_kv=7, cu_q=PTR, cu_k=PTR, cur=None, q=(PTR, 512, 64), k=(PTR, 512, 64),
             out=(PTR, 512, 64), ws=PTR, ws_bytes=1 << 40)
    a.update(kw)
    q, k, out = heads(abi, *a["q"]), heads(abi, *a["k"]), heads(abi, *a["out"])
    return abi.lib.wino_packed_attention(C.byref(p), a["batch"], a["total_q"], a["total_k"], a["max_kv"], a["cu_q"],
                                         a["cu_k"], a["cur"], C.byref(q), C.byref(k), C.byref(k), C.byref(out), None,
                                         a["ws"], a["ws_bytes"], None)


BOTH = [(dict(n_heads=7), -2), (dict(n_heads=0), -2), (dict(n_kv_heads=0), -2), (dict(head_dim=96), -6),
        (dict(dtype=3), -1), (dict(mask=3), -1), (dict(mask=2, block_len=0, cur=PTR), -2),
        (dict(mask=2, block_len=4), -1), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(scale=1e9), -1),
        (dict(batch=0), -2), (dict(total_q=-1), -2), (dict(max_kv=-1), -2), (dict(cu_q=None), -1),
        (dict(q=(PTR + 4, 512, 64)), -6), (dict(q=(PTR, 500, 64)), -6), (dict(out=(PTR, 512, 32)), -2),
        (dict(out=(None, 512, 64)), -1), (dict(total_q=1 << 30), -2), (dict(batch=1 << 21), -2),
        (dict(max_kv=(1 << 30) + 1), -2)]


@pytest.mark.parametrize("call", [paged, packed])
@pytest.mark.parametrize("kw,status", BOTH)
def test_attention_refusals(abi, call, kw, status):
    assert call(abi, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(kv_len=None), -1), (dict(table=None), -1), (dict(cache=dict(dtype=1)), -1), (dict(cache=dict(v=None)), -1),
    (dict(cache=dict(n_kv_heads=8)), -2), (dict(cache=dict(page_size=48)), -6), (dict(max_kv=97), -2),
    (dict(width=-1), -2), (dict(table_stride=5), -2), (dict(cache=dict(token_stride=12)), -6),
    (dict(cache=dict(token_stride=1 << 26)), -6)])
def test_paged_attention_refusals(abi, kw, status):
    assert paged(abi, **kw) == status


@pytest.mark.parametrize("kw,status", [(dict(cu_k=None), -1), (dict(total_k=-1), -2), (dict(k=(PTR, 512, 60)), -6),
                                       (dict(k=(PTR, -8, 64)), -6),
                                       (dict(k=(PTR, 1 << 26, 64)), -6)])
def test_packed_attention_refusals(abi, kw, status):
    assert packed(abi, **kw) == status


def test_workspace_is_checked(abi):
    """A call whose rows are few and whose keys are many needs a workspace, and refuses one that is short."""
    p, _ = attn_params(abi, {})
    need = abi.wino_attention_workspace_bytes(p, 1, 1, 1 << 16)
    kw = dict(batch=1, total_q=1, max_kv=1 << 16, width=1 << 12, table_stride=1 << 12)
    if need:
        assert paged(abi, **kw, ws=None) == -1
        assert paged(abi, **kw, ws_bytes=need - 1) == -2
        assert paged(abi, **kw, ws=PTR + 8) == -6
    assert abi.wino_attention_workspace_bytes(p, 0, 1, 100) == 0
    bad, _ = attn_params(abi, dict(head_dim=80))
    assert abi.wino_attention_workspace_bytes(bad, 1, 1, 100) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes(abi):
    import torch
    k = torch.zeros(2, 16, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        abi.make_kv_cache(k, k)
    with pytest.raises(TypeError):
        abi.make_kv_cache(k.float(), k.float())
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        abi.wino_rope(abi.make_rope_params(64), x, x, x, x)
    with pytest.raises(TypeError):
        abi.wino_rope(abi.make_rope_params(64, dtype=abi.ACT_FP16), x, x, x, x)
    with pytest.raises(ValueError):
        abi.wino_packed_attention(abi.make_attn_params(4, 4, 64), x, x, x, x, torch.zeros(2, dtype=torch.int32),
                                  torch.zeros(2, dtype=torch.int32), 3)


def test_frequencies_are_their_formulas(abi):
    r, th, s = 64, 10000.0, 8.0
    f, m = abi.wino_rope_frequencies(r, th)
    base = [th ** (-2 * j / r) for j in range(r // 2)]
    assert np.allclose(f, base, rtol=1e-13) and m == 1.0
    f, m = abi.wino_rope_frequencies(r, th, abi.ROPE_SCALE_LINEAR, s)
    assert np.allclose(f, [x / s for x in base], rtol=1e-13) and m == 1.0
    f, _ = abi.wino_rope_frequencies(r, th, abi.ROPE_SCALE_BASE, s)
    assert f[0] == 1.0 and math.isclose(f[-1], base[-1] / s, rel_tol=1e-12)
    f, m = abi.wino_rope_frequencies(r, th, abi.ROPE_SCALE_PARTS, s, orig_len=4096, turns_fast=32, turns_slow=1)
    turns = [4096 * x / (2 * math.pi) for x in base]
    for x, b, t in zip(f, base, turns):
        if t >= 32:
            assert x == b
        elif t <= 1:
            assert math.isclose(x, b / s, rel_tol=1e-15)
        else:
            g = (t - 1) / 31
            assert math.isclose(x, g * b + (1 - g) * b / s, rel_tol=1e-13)
    assert any(1 < t < 32 for t in turns) and math.isclose(m, 0.1 * math.log(s) + 1, rel_tol=1e-7)


@pytest.mark.parametrize("kw,status", [
    (dict(theta=1.0), -1), (dict(theta=math.inf), -1), (dict(scaling=4), -1), (dict(scaling=1, factor=0.5), -1),
    (dict(rotary_dim=3), -2), (dict(rotary_dim=0), -2), (dict(scaling=2, rotary_dim=2), -2),
    (dict(scaling=3, orig_len=0.0), -1), (dict(scaling=3, turns_fast=1.0), -1)])
def test_frequency_refusals(abi, kw, status):
    a = dict(rotary_dim=64, theta=1e4, scaling=0, factor=2.0)
    a.update(kw)
    with pytest.raises(abi.WinoError) as e:
        abi.wino_rope_frequencies(**a)
    assert e.value.status == status


def test_oracle_rope_is_a_rotation():
    """Interleaved pairs are complex numbers; the inverse with m = 1 undoes it; scores depend on differences only."""
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((5, 2, 64)), 10000.0 ** (-np.arange(16) / 16)
    pos = np.array([0, 1, 7, 100, 1000])
    y = oo.rope(x, pos, f, 32, interleaved=True)
    z = (x[..., 0:32:2] + 1j * x[..., 1:32:2]) * np.exp(1j * pos[:, None] * f)[:, None]
    assert np.allclose(y[..., 0:32:2], z.real) and np.allclose(y[..., 1:32:2], z.imag)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    assert np.allclose(oo.rope(y, pos, f, 32, interleaved=True, inverse=True), x)
    a, b = oo.rope(x, pos, f, 32), oo.rope(x, pos + 13, f, 32)
    assert np.allclose(np.einsum("thd,shd->hts", a, a), np.einsum("thd,shd->hts", b, b))


def test_oracle_attention_closed_forms():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    q = np.zeros((4, 4, 64))
    vis = oo.sees("causal", 4, 9)
    o, lse, a, _ = oo.attention(q, k, v, 1.0, vis)
    for i in range(4):
        assert np.allclose(o[i, 3], v[:6 + i, 1].mean(0)) and np.allclose(lse[i], math.log(6 + i))
    assert not oo.sees("causal", 5, 2)[:3].any() and oo.sees("causal", 5, 2)[3].tolist() == [True, False]
    s = oo.sees("shadow", 5, 9, block_len=2, cur_start=3)
    assert s[:3].tolist() == [[True] * 7 + [False] * 2] * 3
    assert [int(x) for x in (~s[3:]).nonzero()[1]] == [3, 4] and (~s[3:]).sum() == 2


@pytest.mark.parametrize("heads", [(1, 1), (8, 4), (32, 8), (32, 32), (40, 5)])
@pytest.mark.parametrize("hd", [64, 128])
def test_workspace_of_the_largest_sizes_serves_smaller_ones(abi, heads, hd):
    """A workspace is never larger for fewer sequences, rows or keys, so that a program may allocate one for its largest."""
    p = abi.make_attn_params(*heads, hd)
    rng = np.random.default_rng(hd + heads[0])
    sizes = [[int(x) for x in np.exp(rng.uniform(0, np.log((512, 16384, 262144))))] for _ in range(300)]
    sizes += [[4, 4, 4096], [4, 4, 2048], [64, 64, 1024], [4, 4, 1024], [1, 32, 8192], [1, 33, 8192], [1, 361, 1024],
              [1, 362, 1024]]
    need = np.array([abi.wino_attention_workspace_bytes(p, *s) for s in sizes])
    sizes = np.array(sizes)
    for s, n in zip(sizes, need):
        assert n >= need[(sizes <= s).all(1)].max(), s


def test_workspace_of_split_keys(abi):
    """The refusals of a missing, short or misaligned workspace, at sizes that have one."""
    p, _ = attn_params(abi, {})
    need = abi.wino_attention_workspace_bytes(p, 1, 1, 1 << 16)
    assert need > 0
    kw = dict(batch=1, total_q=1, max_kv=1 << 16, width=1 << 12, table_stride=1 << 12)
    assert paged(abi, **kw, ws=None) == -1 and paged(abi, **kw, ws_bytes=need - 1) == -2
    assert paged(abi, **kw, ws=PTR + 8) == -6


@pytest.mark.parametrize("n,status", [((1 << 26) - 3, -2), ((1 << 26) - 1, -2), ((1 << 26) - 4, -6)])
def test_most_rotary_tokens(abi, n, status):
    """A launch of 2^32 threads (64 a token, tokens rounded up to four) does not start: it is refused before; one token
    fewer passes the sizes' check (and is refused here for its stride)."""
    prm, x = abi.wino_rope_params(*ROPE.values()), heads(abi, PTR, 511, 64)
    assert abi.lib.wino_rope(C.byref(prm), n, 4, PTR, PTR, C.byref(x), C.byref(x), None) == status
    assert append(abi, n=n, q=(PTR, 511, 64)) == status


@pytest.mark.parametrize("call", [paged, packed])
def test_documented_limits_of_attention(abi, call):
    """Each limit is accepted (the calls go on to the missing offsets) and the next value refused."""
    one = dict(n_heads=1, n_kv_heads=1, cu_q=None, cache=dict(n_kv_heads=1)) if call is paged else \
        dict(n_heads=1, n_kv_heads=1, cu_q=None)
    assert call(abi, **one, batch=65535) == -1 and call(abi, **one, batch=65536) == -2
    many = dict(n_heads=65535, n_kv_heads=1)
    assert call(abi, **{**one, **many}) == -1 and call(abi, **{**one, **many, "n_heads": 65536}) == -2
    sh = dict(mask=2, cur=PTR)
    assert call(abi, **one, **sh, block_len=1 << 20) == -1 and call(abi, **one, **sh, block_len=(1 << 20) + 1) == -2
    assert call(abi, **one, batch=65535, total_q=1 << 28) == -1
    assert call(abi, **one, total_q=(1 << 28) + 1) == -2


def test_documented_limits_of_rope(abi):
    x = heads(abi, PTR, 1 << 23, 65)  # a head stride that is refused after the sizes
    for n_heads, status in ((65535, -6), (65536, -2)):
        prm = abi.wino_rope_params(*ROPE.values())
        assert abi.lib.wino_rope(C.byref(prm), 5, n_heads, PTR, PTR, C.byref(x), C.byref(x), None) == status
    big = dict(token_stride=1 << 23, page_stride=1 << 27)
    assert append(abi, cache_args=dict(n_kv_heads=65535, **big), k=(PTR, 511, 64)) == -6
    assert append(abi, cache_args=dict(n_kv_heads=65536, **big), k=(PTR, 511, 64)) == -2
    assert len(abi.wino_rope_frequencies(65536, 1e4)[0]) == 32768
    with pytest.raises(abi.WinoError) as e:
        abi.wino_rope_frequencies(65538, 1e4)
    assert e.value.status == -2


def test_integers_beyond_32_bits_are_refused(abi):
    """The binding does not hand on the lower bits of a size that no 32-bit argument holds."""
    p = abi.make_attn_params(8, 4, 64)
    some = abi.wino_attention_workspace_bytes(p, 1, 1, 5000)
    assert some > 0
    for b, n, m in ((1, 1, (1 << 32) + 5000), (1, (1 << 32) + 1, 5000), ((1 << 32) + 1, 1, 5000), (1, 1, 5000 - (1 << 32))):
        assert abi.wino_attention_workspace_bytes(p, b, n, m) == 0
    for rotary_dim in ((1 << 32) + 64, 64 - (1 << 32), (1 << 40) + 64):
        with pytest.raises(abi.WinoError) as e:
            abi.wino_rope_frequencies(rotary_dim, 1e4)
        assert e.value.status == -2
    with pytest.raises(abi.WinoError):
        abi.wino_rope_frequencies(64, 1e4, scaling=1 << 32)
    assert abi.wino_attention_workspace_bytes(abi.make_attn_params((1 << 32) + 8, 4, 64), 1, 1, 5000) == 0
    assert abi.wino_attention_workspace_bytes(abi.make_attn_params(8, 4, 64, mask=1 << 32), 1, 1, 5000) == 0
    assert abi.make_rope_params(64, inverse=1 << 32).inverse == 1
    assert abi.make_rope_params((1 << 32) + 64).head_dim == (1 << 31) - 1


def test_current_device_without_the_private_call(abi, monkeypatch):
    """torch's public call stands in where the private one does not exist."""
    import torch
    monkeypatch.setattr(abi, "_get_device", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert abi._current_device() == 3
    k = torch.zeros(1, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="must be a device tensor"):
        abi._op_ptr(k, None, "k", abi._current_device())


@pytest.mark.parametrize("rotary_dim,theta,factor", [(4, 1e4, 1e160), (64, 1e300, 1e10), (64, 1.7e308, 2.0)])
def test_a_base_that_overflows_is_refused(abi, rotary_dim, theta, factor):
    """theta times factor^(r/(r-2)) past the largest number: frequencies of zero are not the formula's."""
    with pytest.raises(abi.WinoError) as e:
        abi.wino_rope_frequencies(rotary_dim, theta, abi.ROPE_SCALE_BASE, factor)
    assert e.value.status == -1
