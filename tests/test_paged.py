"""Rows turned by their positions, new rows into the pages of a cache, attention over the pages: against the definitions in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2602_02159_amd import binding as fb

DEV = "cuda:0"
HALF = {torch.bfloat16: 2.0 ** -8}


# ---- plain forms ------------------------------------------------------------------------------------------------------------
def bf16_bits(x):
    """float32 array -> bf16 bits, to the nearest, ties to even."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def pairs(d, rot, interleaved):
    j = np.arange(rot // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)


def turned32(x, pos, freq, interleaved, scale=1.0):
    """float32 rows [n, heads, d] turned as the header says: angles in 64 bits, factors, products and sums rounded to 32."""
    angle = pos.astype(np.float64)[:, None] * freq
    c, s = ((scale * f(angle)).astype(np.float32)[:, None] for f in (np.cos, np.sin))
    a, b = pairs(x.shape[-1], 2 * freq.size, interleaved)
    y = x.astype(np.float32).copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def turned64(x, pos, freq, interleaved, scale=1.0):
    w = scale * np.exp(1j * (pos.astype(np.float64)[:, None] * freq))[:, None]
    a, b = pairs(x.shape[-1], 2 * freq.size, interleaved)
    y = x.astype(np.float64).copy()
    t = (y[..., a] + 1j * y[..., b]) * w
    y[..., a], y[..., b] = t.real, t.imag
    return y


def e4m3_rows(x):
    """float32 rows -> (codes, exponent bytes): the smallest 2^E that holds the largest finite magnitude within 448 of it."""
    a = np.abs(np.where(np.isfinite(x), x, 0)).max(-1).astype(np.float64)
    m, b = np.frexp(a)
    e = np.clip(np.where(a == 0, -110, np.where(m <= 0.875, b - 9, b - 8)), -110, 119)
    y = np.clip(np.ldexp(x.astype(np.float64), -e[..., None]), -448, 448).astype(np.float32)
    y = np.where(np.isfinite(x), y, np.nan).astype(np.float32)
    return torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), (e + 127).astype(np.uint8)


def values(codes, exps):
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(exps.double() - 127)[..., None]


def attend64(q, k, v, seen):
    """[rows, d], [keys, d], [keys, d], [rows, keys] -> out, lse, and what the tolerances need: sum p |v|, max sum |q k|."""
    x = (q @ k.T) / math.sqrt(q.shape[1])
    x = torch.where(seen, x, -math.inf)
    lse = torch.logsumexp(x, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    v = torch.where(seen.any(0)[:, None], v, 0.0)
    size = (q.abs() @ k.abs().T).where(seen, torch.zeros(())).amax(1) / math.sqrt(q.shape[1]) if k.shape[0] else torch.zeros(q.shape[0], dtype=torch.float64)
    return p @ v, lse, p @ v.abs(), size


def check_attention(out, lse, exact):
    """A result is rounded once to bf16.  Before that: a logit's 128 products are added in 32 bits, 2^-17 of their sizes' sum and as much again from
    the normalisation; exp2 and p = hi + lo, whose rest is 2^-17, and the sums: 2^-15 of sum p |v|.  lse likewise, with 2^-20 of itself."""
    ref, ref_lse, mass, size = exact
    err, tol = (out.double() - ref).abs(), 2.0 ** -8 * ref.abs() + (2.0 ** -15 + 2.0 ** -16 * size[:, None]) * mass + 1e-38
    assert bool((err <= tol).all()), f"{(err / tol).max()} times the tolerance"
    empty = ref_lse == -math.inf
    assert bool((lse[empty] == -math.inf).all()) and bool((out[empty] == 0).all())
    far = (lse.double() - ref_lse).abs()[~empty]
    assert bool((far <= 2.0 ** -17 * size[~empty] + 2.0 ** -20 * (1 + ref_lse[~empty].abs())).all()), far.max()


def freqs(rot, base=10000.0):
    return base ** (-2.0 * np.arange(rot // 2) / rot)


def rotation(rot, interleaved=False, scale=1.0, freq=None):
    return fb.make_rotation(torch.from_numpy(freqs(rot) if freq is None else freq).to(DEV), interleaved, scale)


# ---- arguments, on the host ---------------------------------------------------------------------------------------------------
P = C.c_void_p(1 << 20)


def _rot(**kw):
    r = fb.Rotation(1 << 20, 64, 0, 1.0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _cache(**kw):
    c = fb.PagedCache()
    c.k = c.v = 1 << 20
    c.n_pages, c.page, c.n_heads, c.head_dim = 8, 16, 4, 64
    c.k_stride_p = c.v_stride_p = 16 * 4 * 64
    c.k_stride_h = c.v_stride_h = 16 * 64
    c.k_stride_n = c.v_stride_n = 64
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(**kw):
    b = fb.PagedBatch(1 << 20, 1 << 20, None, None, 4, 4, 2, 1, 2)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


ROT_BAD = [dict(freq=None), dict(freq=(1 << 20) + 4), dict(rot_dim=8), dict(rot_dim=24), dict(rot_dim=80), dict(scale=0.0), dict(scale=math.inf), dict(scale=math.nan)]


@pytest.mark.parametrize("bad", ROT_BAD)
def test_rotation_refused(bad):
    L = fb.lib()
    r = _rot(**bad)
    status = fb.FOCUS_EUNSUPPORTED if "rot_dim" in bad else fb.FOCUS_EINVAL
    assert L.focus_rotary(P, 64, 256, P, 64, 256, 4, 4, 64, None, 0, C.byref(r), None) == status
    assert L.focus_paged_append(C.byref(_cache()), C.byref(_batch()), P, P, 64, 256, C.byref(r), None, 0, 0, None, 0, 0, 0, None) == status


@pytest.mark.parametrize("args,status", [
    (dict(X=None), -1), (dict(out=None), -1), (dict(X=C.c_void_p(8)), -1), (dict(xh=4), -1), (dict(on=12), -1), (dict(rows=0), -1), (dict(heads=0), -1),
    (dict(heads=65536), -1), (dict(rows=(1 << 25) + 1), -1), (dict(d=96), -2), (dict(d=256), -2), (dict(on=0), -1), (dict(oh=0), -1), (dict(xn=-256), -1), (dict(on=512), -1)])
def test_rotary_refused(args, status):
    a = dict(X=P, xh=64, xn=256, out=P, oh=64, on=256, rows=4, heads=4, d=64)
    a.update(args)
    rc = fb.lib().focus_rotary(a["X"], a["xh"], a["xn"], a["out"], a["oh"], a["on"], a["rows"], a["heads"], a["d"], None, 0, C.byref(_rot()), None)
    assert rc == status and fb.last_error()


CACHE_BAD = [dict(k=None), dict(v=None), dict(k=8), dict(k_exp=1 << 20), dict(head_dim=32), dict(n_pages=0), dict(page=0), dict(page=65537), dict(n_heads=0),
             dict(n_heads=1025), dict(k_stride_n=32), dict(v_stride_n=68), dict(k_stride_n=1 << 24), dict(k_stride_h=4), dict(v_stride_p=-64),
             dict(k_exp=1 << 20, v_exp=1 << 20, k_stride_n=72), dict(k_exp=1 << 20, v_exp=1 << 20)]
BATCH_BAD = [dict(seq_len=None), dict(page_table=None), dict(n_req=0), dict(n_req=65536), dict(max_rows=0), dict(n_rows=0), dict(n_rows=1), dict(max_rows=2),
             dict(table_width=0), dict(table_width=1 << 28), dict(table_stride=3)]


@pytest.mark.parametrize("cache,batch", [(c, {}) for c in CACHE_BAD] + [({}, b) for b in BATCH_BAD])
def test_paged_refused(cache, batch):
    L, c, b = fb.lib(), _cache(**cache), _batch(**batch)
    status = fb.FOCUS_EUNSUPPORTED if "head_dim" in cache else fb.FOCUS_EINVAL
    assert L.focus_paged_append(C.byref(c), C.byref(b), P, P, 64, 256, None, None, 0, 0, None, 0, 0, 0, None) == status
    assert L.focus_paged_attn(P, 64, 256, 4, C.byref(c), C.byref(b), 0, P, 64, 256, None, P, 1 << 40, None) == status


def test_paged_calls_refused():
    L, c, b = fb.lib(), C.byref(_cache()), C.byref(_batch())
    attn = lambda q=P, heads=4, out=P, oh=64, ws=P, size=1 << 40, cc=c, bb=b: L.focus_paged_attn(q, 64, 256, heads, cc, bb, 0, out, oh, 256, None, ws, size, None)
    assert attn(q=None) == attn(out=None) == attn(heads=6) == attn(heads=0) == attn(oh=0) == attn(cc=None) == attn(bb=None) == fb.FOCUS_EINVAL
    need = L.focus_paged_attn_workspace(c, b, 4)
    assert need > 0 and attn(size=need - 1) == attn(ws=None) == attn(ws=C.c_void_p((1 << 20) + 8)) == fb.FOCUS_EWORKSPACE
    assert L.focus_paged_attn_workspace(c, b, 6) == 0 and L.focus_paged_attn_workspace(C.byref(_cache(head_dim=80)), b, 4) == 0
    many = C.byref(_batch(row_start=1 << 20, n_req=60000, max_rows=4096, n_rows=1 << 20, table_width=1 << 20, table_stride=1 << 20))
    assert L.focus_paged_attn_workspace(c, many, 4) == 0 and attn(bb=many) == fb.FOCUS_EUNSUPPORTED
    wide = C.byref(_batch(row_start=1 << 20, n_req=30000, max_rows=5000, n_rows=1 << 20))
    assert attn(bb=wide) == fb.FOCUS_EUNSUPPORTED and L.focus_paged_append(c, wide, P, P, 64, 256, None, None, 0, 0, None, 0, 0, 0, None) == fb.FOCUS_EUNSUPPORTED
    append = lambda k=P, v=P, q=None, qo=None, heads=0, h=64, qoh=64: L.focus_paged_append(c, b, k, v, h, 256, None, q, 64, 256, qo, qoh, 256, heads, None)
    assert append(k=None) == append(v=None) == append(q=P) == append(qo=P) == append(heads=4) == append(h=12) == fb.FOCUS_EINVAL
    assert append(q=P, qo=P, heads=0) == append(q=P, qo=P, heads=4, qoh=128) == append(q=P, qo=P, heads=4, qoh=0) == fb.FOCUS_EINVAL


@pytest.mark.parametrize("cache", [
    dict(), dict(v=1 << 24, k_stride_h=0), dict(v=1 << 24, v_stride_h=0), dict(v=1 << 24, k_stride_p=0), dict(v=1 << 24, v_stride_p=0),
    dict(v=1 << 24, k_exp=1 << 25, v_exp=1 << 25, exp_stride_p=64, exp_stride_h=16, exp_stride_n=1), dict(v=1 << 24, k_exp=1 << 25, v_exp=1 << 26, exp_stride_p=64, exp_stride_n=1),
    dict(v=1 << 24, k_exp=1 << 25, v_exp=1 << 26, exp_stride_h=16, exp_stride_n=1)])
def test_shared_rows_are_not_written(cache):
    L, c, b = fb.lib(), _cache(**cache), _batch()
    assert L.focus_paged_append(C.byref(c), C.byref(b), P, P, 64, 256, None, None, 0, 0, None, 0, 0, 0, None) == fb.FOCUS_EINVAL
    assert "on one another" in fb.last_error()


@pytest.mark.parametrize("heads,rows,d,sh,sn,fine", [
    (4, 4, 64, 64, 256, True), (4, 4, 64, 256, 64, True), (4, 5, 64, 320, 64, True), (2, 4, 128, 136, 264, True), (2, 3, 128, 400, 128, True), (1, 4, 64, 0, 64, True),
    (4, 1, 64, 64, 0, True), (1, 1, 128, 0, 0, True), (4, 4, 64, 8, 256, False), (2, 4, 128, 8, 128, False), (4, 4, 64, 64, 248, False), (4, 4, 64, 64, 192, False),
    (4, 5, 64, 312, 64, False), (4, 4, 64, 256, 56, False), (1, 2, 128, 0, 120, False), (2, 1, 128, 120, 0, False), (3, 3, 64, 64, 64, False),
    (2, 1 << 25, 64, 1 << 31, 64, True), (2, 1 << 25, 64, (1 << 31) - 8, 64, False), (65535, 2, 64, 1 << 58, 64, True)])
def test_rows_that_are_written_are_clear_of_one_another(heads, rows, d, sh, sn, fine):
    """Strides less than what the rows along the smaller ones span are refused, others are not: by brute force where there are few rows.  The calls that go past this
    check end at a later one."""
    if heads * rows < 1000:
        at = sorted(h * sh + i * sn for h in range(heads) for i in range(rows))
        assert fine == all(b - a >= d for a, b in zip(at, at[1:]))
    L, at_8 = fb.lib(), C.c_void_p((1 << 20) + 8)  # (not aligned: the next check)
    b = _batch(n_rows=rows, n_req=1, row_start=1 << 20, max_rows=1)
    c = _cache(head_dim=d, n_heads=1, v=1 << 24, k_stride_n=d, v_stride_n=d, k_stride_p=16 * d, v_stride_p=16 * d)
    calls = [lambda: L.focus_rotary(P, 64, 256, at_8, sh, sn, rows, heads, d, None, 0, C.byref(_rot()), None),
             lambda: L.focus_paged_append(C.byref(c), C.byref(b), P, P, 64, 256, None, P, 64, 256, at_8, sh, sn, heads, None),
             lambda: L.focus_paged_attn(P, 64, 256, heads, C.byref(c), C.byref(b), 0, at_8, sh, sn, None, P, 1 << 40, None)]
    for call in calls:
        assert call() == fb.FOCUS_EINVAL and ("aligned" if fine else "on one another") in fb.last_error()


@pytest.mark.parametrize("kw,fine", [
    (dict(), True), (dict(k_stride_p=64, k_stride_h=8 * 64, k_stride_n=8 * 4 * 64), True), (dict(k_stride_h=64, k_stride_n=4 * 64), True), (dict(k_stride_p=8192, k_stride_n=72, k_stride_h=1152), True),
    (dict(k_stride_h=8), False), (dict(k_stride_h=960), False), (dict(v_stride_p=2048), False), (dict(k_stride_p=4088), False), (dict(v_stride_h=64), False), (dict(v_stride_n=72), False),
    (dict(n_heads=1, v_stride_h=8), True), (dict(n_pages=1, v_stride_p=0), True), (dict(page=1, k_stride_n=1 << 20), True)])
def test_caches_whose_rows_lie_on_one_another_are_not_written(kw, fine):
    c = _cache(**kw)  # k = v, which is refused last
    assert fb.lib().focus_paged_append(C.byref(c), C.byref(_batch()), P, P, 64, 256, None, None, 0, 0, None, 0, 0, 0, None) == fb.FOCUS_EINVAL
    assert ("k and v" if fine else "rows of " + next(iter(kw))[0]) + " lie on one another" in fb.last_error()


@pytest.mark.parametrize("strides,fine", [((64, 16, 1), True), ((64, 1, 4), True), ((1, 128, 8), True), ((64, 15, 1), False), ((63, 16, 1), False), ((64, 16, 4), False), ((64, 2, 1), False)])
def test_exponents_that_lie_on_one_another_are_not_written(strides, fine):
    c = _cache(k_exp=1 << 25, v_exp=1 << 26, exp_stride_p=strides[0], exp_stride_h=strides[1], exp_stride_n=strides[2])
    assert fb.lib().focus_paged_append(C.byref(c), C.byref(_batch()), P, P, 64, 256, None, None, 0, 0, None, 0, 0, 0, None) == fb.FOCUS_EINVAL
    assert ("k and v" if fine else "exponents") + " lie on one another" in fb.last_error()


def test_frequencies():
    f = fb.rotary_freqs(10000.0, 64)
    assert torch.allclose(f, 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64), rtol=1e-14)
    assert torch.allclose(fb.rotary_freqs(10000.0, 64, 4.0, 2048, math.inf, math.inf), f / 4, rtol=1e-14)  # all divided
    g = fb.rotary_freqs(10000.0, 128, 8.0, 8192, 1.0, 4.0)
    f = 10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)
    turns = 8192 * f / (2 * math.pi)
    assert torch.allclose(g[turns > 4], f[turns > 4], rtol=1e-14) and torch.allclose(g[turns < 1], f[turns < 1] / 8, rtol=1e-14)
    between = (turns >= 1) & (turns <= 4)
    share = (turns - 1) / 3
    assert bool(between.any()) and torch.allclose(g[between], (f * (share + (1 - share) / 8))[between], rtol=1e-13)
    for bad in ((0.0, 64), (10000.0, 63), (10000.0, 0), (10000.0, 64, 0.0), (10000.0, 64, 2.0, 0), (10000.0, 64, 2.0, 8, 4.0, 1.0), (math.nan, 64)):
        with pytest.raises(fb.FocusError):
            fb.rotary_freqs(*bad)


def test_frequencies_are_all_divided_where_no_turns_are_given():
    f = fb.rotary_freqs(10000.0, 64)
    assert torch.allclose(fb.rotary_freqs(10000.0, 64, 4.0), f / 4, rtol=1e-14) and torch.allclose(fb.rotary_freqs(10000.0, 64, 4.0, 8192), f / 4, rtol=1e-14)
    assert torch.allclose(fb.rotary_freqs(10000.0, 64, 4.0, 8192, 0.0, 0.0), f, rtol=1e-14)  # a step at no turn at all: none is
    with pytest.raises(fb.FocusError):
        fb.rotary_freqs(10000.0, 64, 4.0, 8192, turns_high=4.0)  # half of a range


@pytest.mark.parametrize("bad", [(10000.0, 16, 4.0, 8192, -math.inf, 4.0), (10000.0, 16, 4.0, 8192, -math.inf, math.inf), (10000.0, 16, 4.0, 8192, -math.inf, -1.0),
                                 (5e-324, 64), (10000.0, 64, 5e-324, 8192, 1.0, 4.0), (10000.0, 64, 4.0, 8192, math.nan, 4.0), (10000.0, 64, 4.0, 8192, 1.0, math.nan)])
def test_frequencies_are_finite_or_refused(bad):
    with pytest.raises(fb.FocusError):
        fb.rotary_freqs(*bad)


@pytest.mark.parametrize("low,high", [(-math.inf, -math.inf), (-1.0, 4.0), (1.0, math.inf), (0.0, 0.0), (math.inf, math.inf), (-1e300, 1e300)])
def test_frequencies_of_unusual_ranges(low, high):
    """Between what stays and what is divided, in order, for every range with two ends."""
    f, g = fb.rotary_freqs(10000.0, 64), fb.rotary_freqs(10000.0, 64, 4.0, 8192, low, high)
    assert bool(((g >= f / 4 * (1 - 1e-14)) & (g <= f * (1 + 1e-14))).all())
    share = (g / f - 0.25) / 0.75
    assert bool((share.diff() <= 1e-12).all())  # fewer turns, less of it stays
    if low == high:
        assert torch.allclose(g, f / 4 if low > 0 else f, rtol=1e-14)


# ---- rotation ---------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("n,heads,d,rot,interleaved,scale,first", [
    (1, 1, 64, 16, False, 1.0, 0), (1, 32, 128, 128, False, 1.25, 1_000_000), (5, 7, 128, 96, True, 1.0, 3), (9, 3, 64, 64, True, 0.5, 2_000_000_000),
    (33, 4, 64, 32, False, -1.0, 31), (130, 2, 128, 16, True, 1.0, 0), (1027, 9, 128, 128, False, 1.0, 5)])
def test_rotary(n, heads, d, rot, interleaved, scale, first):
    g = torch.Generator().manual_seed(n + heads)
    x = torch.randn((n, heads, d), generator=g).bfloat16().to(DEV)
    positions = torch.randperm(2 * n, generator=g)[:n].int()
    positions[n // 2] = -1 if n > 1 else 0
    out = torch.full_like(x, 7.0)
    fb.rotary(x, out, positions.to(DEV), first, rotation(rot, interleaved, scale))
    at = positions.numpy().astype(np.int64)
    x32 = x.float().cpu().numpy()
    want = bf16_bits(turned32(x32, at + first, freqs(rot), interleaved, scale))
    want[at < 0] = bf16_bits(np.float32(7.0))
    assert np.array_equal(bits(out), want)
    exact = turned64(x32, at + first, freqs(rot), interleaved, scale)
    a, b = pairs(d, rot, interleaved)
    both = np.zeros_like(exact)  # cos, sin, two products and the sum: 2^-24 of each
    both[..., a] = both[..., b] = abs(scale) * (np.abs(x32[..., a]) + np.abs(x32[..., b]))
    err = np.abs(out.float().cpu().numpy() - exact)
    assert (err <= 2.0 ** -8 * np.abs(exact) + 4 * 2.0 ** -24 * both)[at >= 0].all()


@pytest.mark.gpu
def test_rotary_strides_in_place_back_and_gradient():
    n, heads, d = 37, 6, 128
    g = torch.Generator().manual_seed(1)
    x = torch.randn((n, heads, d), generator=g).bfloat16().to(DEV)
    rot = rotation(d)
    want = torch.empty_like(x)
    fb.rotary(x, want, None, 11, rot)
    head_major = torch.empty((heads, n, d), dtype=torch.bfloat16, device=DEV)
    fb.rotary(x, head_major.transpose(0, 1), None, 11, rot)
    assert torch.equal(head_major.transpose(0, 1), want)
    wide = torch.zeros((n, heads + 2, d + 8), dtype=torch.bfloat16, device=DEV)
    part = wide[:, 1:-1, :d]
    part.copy_(x)
    fb.rotary(part, part, None, 11, rot)
    assert torch.equal(part, want) and not wide[:, 0].any() and not wide[:, -1].any() and not wide[..., d:].any()
    one = torch.empty_like(x[:1])
    fb.rotary(x[:1], one, torch.tensor([-1], dtype=torch.int32, device=DEV), 0, rot)  # left alone
    # frequencies the other way turn back: to the rounding of the two calls, each at most 2^-8 of a pair's length
    back = torch.empty_like(x)
    fb.rotary(want, back, None, 11, rotation(d, freq=-freqs(d)))
    length = (x.float()[..., :64].square() + x.float()[..., 64:].square()).sqrt().repeat(1, 1, 2)
    assert bool(((back.float() - x.float()).abs() <= 2.0 ** -8 * (2 * length + x.float().abs()) * 1.01).all())
    # and so the turn of a gradient: <turn(x), y> = <x, turn back(y)>
    y = torch.randn((n, heads, d), generator=g).bfloat16().to(DEV)
    grad = torch.empty_like(y)
    fb.rotary(y, grad, None, 11, rotation(d, freq=-freqs(d)))
    left, right = (want.double() * y.double()).sum(-1), (x.double() * grad.double()).sum(-1)
    size = (want.double() * y.double()).abs().sum(-1) + (x.double() * grad.double()).abs().sum(-1)
    assert bool(((left - right).abs() <= 2.0 ** -8 * size).all())


@pytest.mark.gpu
def test_rotary_special_values():
    x = torch.randn((2, 1, 64)).bfloat16()
    x[0, 0, 0], x[0, 0, 40], x[0, 0, 63] = math.inf, math.nan, -math.inf
    x = x.to(DEV)
    out = torch.empty_like(x)
    fb.rotary(x, out, None, 1, rotation(32))
    spoilt = torch.zeros(64, dtype=torch.bool)
    spoilt[[0, 16, 40, 63]] = True  # the pair of 0, and values that are not turned
    assert torch.equal(~torch.isfinite(out[0, 0]).cpu(), spoilt)
    assert torch.equal(out[:, :, 32:].view(torch.int16), x[:, :, 32:].view(torch.int16)) and bool(torch.isfinite(out[1]).all())


# ---- a cache and its requests -------------------------------------------------------------------------------------------------
class Pages:
    """A pool whose every byte is NaN, tables of pages in no order, and the plain form's view of both."""

    def __init__(self, lens, width, page, H, d, quant, rows_first, seed=0, spare=3):
        self.g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.H, self.d, self.quant = list(lens), page, H, d, quant
        n = len(lens) * width + spare
        sizes = (n, page, H) if rows_first else (n, H, page)
        order = (lambda t: t.transpose(1, 2)) if rows_first else (lambda t: t)
        kind = dict(dtype=torch.uint8) if quant else dict(dtype=torch.bfloat16)
        full = lambda: order(torch.full((*sizes, d), 0x7f if quant else math.nan, device=DEV, **kind))
        self.k, self.v = full(), full()
        self.k_exp, self.v_exp = (order(torch.full(sizes, 255, dtype=torch.uint8, device=DEV)) for _ in range(2)) if quant else (None, None)
        self.table = torch.randperm(n, generator=self.g)[:len(lens) * width].view(len(lens), width).int()
        self.cache = fb.make_paged_cache(self.k, self.v, self.k_exp, self.v_exp)

    def fill(self, loud=0.0):
        """Random rows where the requests have some."""
        for r, n in enumerate(self.lens):
            if n <= 0:
                continue
            j = torch.arange(n)
            page, at = self.table[r, j // self.page].long(), j % self.page
            there = (page >= 0) & (page < self.k.shape[0])
            page, at = page[there].to(DEV), at[there].to(DEV)
            for name in ("k", "v"):
                x = torch.randn((page.numel(), self.H, self.d), generator=self.g)
                if loud and name == "k":
                    x[:, :, 0] *= loud
                if self.quant:
                    codes, exps = e4m3_rows(x.numpy())
                    getattr(self, name)[page, :, at] = torch.from_numpy(codes).to(DEV)
                    getattr(self, name + "_exp")[page, :, at] = torch.from_numpy(exps).to(DEV)
                else:
                    getattr(self, name)[page, :, at] = x.bfloat16().to(DEV)
        return self

    def rows(self, r, n):
        """(positions, K, V) of request r in 64 bits, [keys, H, d]."""
        j = torch.arange(max(min(n, self.table.shape[1] * self.page), 0))
        page = self.table[r, j // self.page].long()
        j, page = j[(page >= 0) & (page < self.k.shape[0])], page[(page >= 0) & (page < self.k.shape[0])]
        get = lambda t: t[page.to(DEV), :, (j % self.page).to(DEV)].cpu()
        if self.quant:
            return j, values(get(self.k), get(self.k_exp)), values(get(self.v), get(self.v_exp))
        return j, get(self.k).double(), get(self.v).double()


def batch_of(lens, table, rows=None, positions=None, behind=0):
    start = None if rows is None else torch.tensor([0, *np.cumsum(rows)], dtype=torch.int32, device=DEV)
    total = (len(lens) if rows is None else sum(rows)) + behind
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    return fb.make_paged_batch(torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV), start, 1 if rows is None else max(max(rows), 1), total, pos)


def places(lens, rows, positions=None):
    """(row, request, position) of every row."""
    rows = [1] * len(lens) if rows is None else rows
    found, at = [], 0
    for r, n in enumerate(rows):
        for i in range(n):
            found.append((at, r, max(lens[r], 0) - n + i if positions is None else positions[at]))
            at += 1
    return found


def workspace(cache, batch, heads):
    return torch.full((fb.paged_attn_workspace(cache, batch, heads),), 0xff, dtype=torch.uint8, device=DEV)


# ---- new rows ---------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("lens,rows,H,group,d,page,rows_first,rot,interleaved,positions", [
    ([1], None, 1, 1, 64, 1, False, 16, False, None),
    ([5, 0, 17, 64], None, 8, 4, 128, 16, True, 128, False, None),
    ([100, 7, 33], [9, 0, 33], 3, 1, 64, 16, False, 64, True, None),
    ([300, 1, 555], [130, 1, 7], 2, 7, 128, 100, True, 96, False, None),
    ([40, 90], [6, 5], 4, 2, 128, 7, False, 32, True, [3, -1, 39, 0, 95, 3, 88, 88, 2, 200, -5]),  # gaps, past the table, the same twice
    ([70], [300], 2, 0, 64, 32, False, 64, False, [(i * 7) % 70 for i in range(300)]),  # every position more than once
    ([2], [5], 2, 1, 128, 16, False, None, False, None),  # more rows than positions: the first ones have none
])
def test_append(lens, rows, H, group, d, page, rows_first, rot, interleaved, positions, quant):
    width = -(-max(max(lens), 1) // page)
    pool = Pages(lens, width, page, H, d, quant, rows_first, seed=len(lens))
    pool.table[0, 0] = pool.k.shape[0] + 5 if len(lens) > 2 else pool.table[0, 0]  # a page that there is not
    batch = batch_of(lens, pool.table, rows, None if positions is None else positions + [0, 1], behind=2)
    total, g = batch.n_rows, torch.Generator().manual_seed(3)
    k, v = (torch.randn((total, H, d), generator=g).bfloat16() for _ in range(2))
    k[:, :, 1] *= 30
    q = torch.randn((total, H * group, d), generator=g).bfloat16() if group else None
    q_out = torch.full((total, H * group, d), 9.0, dtype=torch.bfloat16, device=DEV) if group else None
    spin = rotation(rot, interleaved) if rot else None
    before = [t.clone() for t in (pool.k, pool.v, pool.k_exp, pool.v_exp) if t is not None]
    fb.paged_append(pool.cache, batch, k.to(DEV), v.to(DEV), spin, None if q is None else q.to(DEV), q_out)
    turn = lambda x, p: turned32(x, p, freqs(rot), interleaved) if rot else x
    want = [t.cpu().clone() for t in before]
    q_want = torch.full((total, H * group, d), 9.0).bfloat16() if group else None
    for at, r, p in places(lens, rows, positions):
        if p < 0:
            continue
        one = np.array([p])
        if group:
            q_want[at] = torch.from_numpy(bf16_bits(turn(q[at:at + 1].float().numpy(), one)).view(np.int16)).view(torch.bfloat16)[0]
        if p // page >= width or not 0 <= int(pool.table[r, p // page]) < pool.k.shape[0]:
            continue
        pg, row = int(pool.table[r, p // page]), p % page
        new_k, new_v = turn(k[at:at + 1].float().numpy(), one)[0], v[at].float().numpy()
        if quant:
            for i, x in ((0, new_k), (1, new_v)):
                codes, exps = e4m3_rows(x)
                want[i][pg, :, row], want[2 + i][pg, :, row] = torch.from_numpy(codes), torch.from_numpy(exps)
        else:
            want[0][pg, :, row] = torch.from_numpy(bf16_bits(new_k).view(np.int16)).view(torch.bfloat16)
            want[1][pg, :, row] = v[at]
    for t, w in zip((pool.k, pool.v, pool.k_exp, pool.v_exp), want):
        raw = (lambda x: x.contiguous().view(torch.int16).cpu()) if t.dtype == torch.bfloat16 else (lambda x: x.contiguous().cpu())
        assert torch.equal(raw(t), raw(w))
    if group:
        assert torch.equal(q_out.cpu().view(torch.int16), q_want.view(torch.int16))


@pytest.mark.gpu
def test_append_quantised_special_rows():
    """Rows of zeros, of infinities and NaN, of the smallest and largest magnitudes: the codes of the definition."""
    d, rows = 128, 6
    x = torch.randn((rows, 1, d))
    x[1] = 0.0
    x[2, 0, 3], x[2, 0, 90], x[2, 0, 5] = math.inf, -math.inf, math.nan
    x[3] *= 1e-38
    x[4] *= 1e38
    x[5] *= 2.0 ** -120
    x = x.bfloat16()
    pool = Pages([rows], 1, 8, 1, d, True, False)
    fb.paged_append(pool.cache, batch_of([rows], pool.table, [rows]), x.to(DEV), x.to(DEV))
    codes, exps = e4m3_rows(x.float().numpy())
    pg = int(pool.table[0, 0])
    for t, e in ((pool.k, pool.k_exp), (pool.v, pool.v_exp)):
        assert np.array_equal(e[pg, 0, :rows].cpu().numpy(), exps[:, 0])
        got, nan = t[pg, 0, :rows].cpu().numpy(), np.isnan(x.float().numpy()[:, 0]) | np.isinf(x.float().numpy()[:, 0])
        assert np.array_equal(got[~nan], codes[:, 0][~nan]) and (got[nan] & 0x7f == 0x7f).all()


# ---- attention --------------------------------------------------------------------------------------------------------------
def run_attention(pool, lens, rows=None, group=1, causal=False, positions=None, behind=0, q=None, gain=1.0, strided=False):
    batch = batch_of(lens, pool.table, rows, None if positions is None else positions + [0] * behind, behind)
    n, heads, d = batch.n_rows, pool.H * group, pool.d
    if q is None:
        q = (gain * torch.randn((n, heads, d), generator=torch.Generator().manual_seed(5))).bfloat16()
    q = q.to(DEV)
    out = torch.full((heads, n, d) if strided else (n, heads, d), 5.0, dtype=torch.bfloat16, device=DEV)
    out = out.transpose(0, 1) if strided else out
    lse = torch.full((n, heads), 6.0, device=DEV)
    fb.paged_attn(q, pool.cache, batch, causal, out, lse, workspace(pool.cache, batch, heads))
    found = places(lens, rows, positions)
    out, lse, q = out.cpu(), lse.cpu(), q.cpu().double()
    for r in range(len(lens)):
        mine = [(at, p) for at, s, p in found if s == r]
        if not mine:
            continue
        j, k, v = pool.rows(r, lens[r])
        at = [x[0] for x in mine]
        seen = torch.ones((len(mine), j.numel()), dtype=torch.bool)
        if causal:
            seen = j[None] <= torch.tensor([x[1] for x in mine])[:, None]
        for h in range(heads):
            check_attention(out[at, h], lse[at, h], attend64(q[at, h], k[:, h // group], v[:, h // group], seen))
    untouched = out[len(found):]
    assert bool((untouched == 5.0).all()) and bool((lse[len(found):] == 6.0).all())
    return out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("lens,H,group,d,page,rows_first", [
    ([1], 1, 1, 64, 16, False), ([0], 2, 1, 128, 16, False), ([31], 1, 3, 128, 1, True), ([32], 4, 1, 64, 16, True), ([33], 2, 7, 128, 32, False),
    ([1000], 4, 1, 64, 16, False), ([5, 0, 129, 64, 1, 700], 3, 5, 128, 16, True), ([257, 3, 90], 1, 16, 64, 7, False),
    ([4099], 2, 4, 128, 100, True), ([8200, 31], 8, 1, 128, 64, False), ([300, 20], 2, 24, 64, 48, False), ([100, 2000], 1, 40, 128, 128, True)])
def test_attention(lens, H, group, d, page, rows_first, quant):
    pool = Pages(lens, -(-max(max(lens), 1) // page), page, H, d, quant, rows_first, seed=sum(lens)).fill(loud=3.0)
    run_attention(pool, lens, group=group, gain=1.5)


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,rows,H,group,d,page,positions", [
    ([40, 7, 500], [4, 1, 25], 2, 4, 128, 16, None),
    ([3, 0, 64], [5, 2, 3], 1, 1, 64, 32, None),  # more rows than positions
    ([600, 90], [17, 0], 3, 7, 64, 100, None),
    ([200, 33], [6, 3], 2, 1, 128, 16, [199, -1, 0, 50, 150, 1000, 5, 5, 32]),  # any positions, some of none
    ([70], [70], 1, 3, 128, 64, None),  # a prompt
])
def test_attention_of_several_rows(lens, rows, H, group, d, page, positions, causal, quant):
    pool = Pages(lens, -(-max(lens) // page), page, H, d, quant, False, seed=7).fill()
    run_attention(pool, lens, rows, group, causal, positions, behind=3, strided=True)


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("page", [16, 5, 64])
def test_pages_that_there_are_not(page, quant):
    """Entries outside the pool, past the table, everything left out: those rows do not exist."""
    lens = [200, 130, 90, 1 << 30]
    width = -(-200 // page)
    pool = Pages(lens[:3] + [width * page], width, page, 2, 128, quant, False)
    drop = torch.rand(pool.table.shape, generator=pool.g) < 0.5
    pool.table[drop] = torch.tensor([-1, pool.k.shape[0], -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)[torch.randint(0, 4, (int(drop.sum()),), generator=pool.g)]
    pool.table[1] = -1
    pool.fill()
    run_attention(pool, lens, group=3)
    run_attention(pool, lens, [2, 3, 1, 4], group=1, causal=True)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [64, 257, 700])
def test_many_requests(n):
    """More requests than a wavefront has lanes, and than it keeps in registers; some of no row, some of no key."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 90, n)]
    rows = [int(x) for x in rng.integers(0, 3, n)]
    lens[n // 2], rows[0], rows[-1] = 5000, 1, 1
    pool = Pages(lens, 5000 // 32 + 1, 32, 2, 64, False, True, spare=1).fill()
    run_attention(pool, lens, rows, group=2, causal=True, behind=1)


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("group", [4, 12])
def test_keys_that_a_row_does_not_see_do_not_reach_it(group, quant):
    """Infinities and NaN in V of positions that only the later rows see."""
    pool = Pages([100], 7, 16, 1, 128, quant, False).fill()
    page, at = int(pool.table[0, 6]), 3  # position 99, and 98 an infinity
    if quant:
        pool.v[page, 0, at, 5] = 0x7f
        pool.v[page, 0, at - 1, 9] = 0xff
    else:
        pool.v[page, 0, at, 5] = math.nan
        pool.v[page, 0, at - 1, 9], pool.v[page, 0, at - 1, 10] = math.inf, -math.inf
    batch = batch_of([100], pool.table, [4])
    q = torch.randn((4, group, 128), generator=torch.Generator().manual_seed(2)).bfloat16()
    out, lse = torch.empty((4, group, 128), dtype=torch.bfloat16, device=DEV), torch.empty((4, group), device=DEV)
    fb.paged_attn(q.to(DEV), pool.cache, batch, True, out, lse, workspace(pool.cache, batch, group))
    out, (j, k, v) = out.cpu(), pool.rows(0, 100)
    for i in range(4):
        n = 97 + i
        bad = ~torch.isfinite(v[:n, 0]).all(0)
        assert torch.equal(~torch.isfinite(out[i, 0].float()), bad) and int(bad.sum()) == (0, 0, 1 if quant else 2, 2 if quant else 3)[i]
        for h in range(group):
            ref = attend64(q[i:i + 1, h].double(), k[:n, 0], v[:n, 0].masked_fill(bad, 0.0), torch.ones((1, n), dtype=torch.bool))
            check_attention(out[i:i + 1, h].masked_fill(bad, 0.0), lse[i:i + 1, h].cpu(), ref)
    if not quant:
        assert out[2, 0, 9] == math.inf and out[2, 0, 10] == -math.inf and bool(out[3, 0, 5].isnan())


@pytest.mark.gpu
@pytest.mark.parametrize("d,group,page", [(128, 4, 16), (128, 12, 7), (64, 1, 32), (64, 24, 16)])
def test_memory_that_was_never_written_does_not_reach_earlier_rows(d, group, page):
    """Eight-bit pages whose later positions hold the NaN code and exponent bytes of 255 (infinity as a factor), which no row that is written has: rows
    before them get the attention over what is there."""
    lens, written = [100, 300], [61, 37]
    pool = Pages(lens, -(-300 // page), page, 2, d, True, False, seed=d + group)
    assert bool((pool.k_exp == 255).all()) and bool((pool.v_exp == 255).all())
    pool.lens = written
    pool.fill()
    positions = [60, 3, 0, 33, 36, 31, 20]
    rows = [4, 3]
    batch = batch_of(lens, pool.table, rows, positions)
    q = torch.randn((7, 2 * group, d), generator=torch.Generator().manual_seed(3)).bfloat16()
    out, lse = torch.empty((7, 2 * group, d), dtype=torch.bfloat16, device=DEV), torch.empty((7, 2 * group), device=DEV)
    fb.paged_attn(q.to(DEV), pool.cache, batch, True, out, lse, workspace(pool.cache, batch, 2 * group))
    for at, r, p in places(lens, rows, positions):
        j, k, v = pool.rows(r, p + 1)
        for h in range(2 * group):
            ref = attend64(q[at:at + 1, h].double(), k[:, h // group], v[:, h // group], torch.ones((1, p + 1), dtype=torch.bool))
            check_attention(out[at:at + 1, h].cpu(), lse[at:at + 1, h].cpu(), ref)


def spoil(pool, r, j, column, value):
    """Writes an infinity or a NaN into V of position j of request r (codes: the NaN code)."""
    page, at = int(pool.table[r, j // pool.page]), j % pool.page
    pool.v[page, :, at, column] = 0x7f if pool.quant else value


def check_not_finite(out, lse, q, k, v, seen):
    """One row and head against the definition: an infinity or a NaN of V comes out where a key that the row sees has it, infinities of both signs as NaN."""
    up, down = ((seen[:, None] & ((v == x) | v.isnan())).any(0) for x in (math.inf, -math.inf))
    assert torch.equal(out == math.inf, up & ~down) and torch.equal(out == -math.inf, down & ~up) and torch.equal(out.isnan(), up & down)
    finite = torch.where(v.isfinite(), v, 0.0)
    check_attention(out.masked_fill(up | down, 0.0)[None], lse[None], attend64(q[None].double(), k, finite.masked_fill((up | down)[None], 0.0), seen[None]))


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,rows,H,group,d,page,far", [
    ([100], None, 1, 1, 128, 16, False),
    ([64, 33], [3, 1], 2, 4, 64, 32, False),
    ([100, 7], [25, 2], 1, 7, 128, 5, False),  # 32 query rows at a time, pages that end within sixteen rows
    ([5000], None, 4, 2, 128, 100, False),  # pieces of many wavefronts
    ([3000, 40], [20, 1], 2, 2, 64, 16, True),  # keys of later tiles far above those with the infinities, whose weights are zero in 32 bits
    ([3000], None, 1, 1, 128, 16, True),
])
def test_values_that_are_not_finite(lens, rows, H, group, d, page, far, causal, quant):
    """Infinities and NaN in V, in whole tiles and in cut ones, at the first key, in the middle, at the last: the same result wherever the borders of tiles, pieces
    and limits lie."""
    pool = Pages(lens, -(-max(lens) // page), page, H, d, quant, False, seed=3).fill()
    if far and not quant:
        pool.k[:, :, :, 0] = torch.where(pool.k[:, :, :, 0].isnan(), math.nan, 0.0).bfloat16()
        for j in (2000, 2990):
            pool.k[int(pool.table[0, j // page]), :, j % page, 0] = 90.0 if j == 2000 else 120.0
    n = lens[0]
    for j, column, value in ((0, 1, math.inf), (n // 2, 2, -math.inf), (n // 2 + 1, 3, math.nan), (n - 1, 4, math.inf), (3, 5, math.inf), (n - 2, 5, -math.inf),
                             (2, d - 1, -math.inf), (n // 3, d // 2, math.inf), (n // 3 + 40 if n > 200 else n // 3, d // 2 + 1, math.inf)):
        spoil(pool, 0, j, column, value)
    batch = batch_of(lens, pool.table, rows)
    total, heads = batch.n_rows, H * group
    q = torch.randn((total, heads, d), generator=torch.Generator().manual_seed(2)).bfloat16()
    if far:
        q[:, :, 0] = 64.0
    out, lse = torch.empty((total, heads, d), dtype=torch.bfloat16, device=DEV), torch.empty((total, heads), device=DEV)
    fb.paged_attn(q.to(DEV), pool.cache, batch, causal, out, lse, workspace(pool.cache, batch, heads))
    out, lse = out.cpu(), lse.cpu()
    for r in range(len(lens)):
        j, k, v = pool.rows(r, lens[r])
        for at, _, p in [x for x in places(lens, rows) if x[1] == r]:
            for h in range(heads):
                check_not_finite(out[at, h], lse[at, h], q[at, h], k[:, h // group], v[:, h // group], j <= p if causal else j >= 0)


@pytest.mark.gpu
@pytest.mark.parametrize("group,rows", [(1, 1), (9, 3)])
def test_requests_beside_one_that_is_not_finite(group, rows):
    """600 requests, several to a wavefront: those with infinities and NaN get them, those before and behind are as without."""
    n, H, d, page = 600, 8, 64, 16
    lens = [70 + i % 50 for i in range(n)]
    pool = Pages(lens, 8, page, H, d, False, True, seed=1, spare=0).fill()
    batch = batch_of(lens, pool.table, [rows] * n if rows > 1 else None)
    q = torch.randn((n * rows, H * group, d), generator=torch.Generator().manual_seed(2)).bfloat16()
    results = []
    for spoilt in (False, True):
        if spoilt:
            for r, j, column, value in ((3, 0, 1, math.inf), (4, 69, 2, math.nan), (100, 40, 0, -math.inf), (101, 1, 63, math.inf), (350, 33, 7, math.inf), (599, 1, 9, -math.inf)):
                spoil(pool, r, j, column, value)
        out, lse = torch.empty((n * rows, H * group, d), dtype=torch.bfloat16, device=DEV), torch.empty((n * rows, H * group), device=DEV)
        fb.paged_attn(q.to(DEV), pool.cache, batch, True, out, lse, workspace(pool.cache, batch, H * group))
        results.append((out.cpu().view(n, rows, H * group, d), lse.cpu().view(n, rows, H * group)))
    there = torch.tensor([r in (3, 4, 100, 101, 350, 599) for r in range(n)])
    (clean, clean_lse), (out, lse) = results
    assert torch.equal(lse, clean_lse) and torch.equal(out[~there], clean[~there])
    for r in there.nonzero()[:, 0].tolist() + [0, 2, 5, 99, 349, 598]:
        j, k, v = pool.rows(r, lens[r])
        for i in range(rows):
            for h in range(0, H * group, 5):
                check_not_finite(out[r, i, h], lse[r, i, h], q[r * rows + i, h], k[:, h // group], v[:, h // group], j <= lens[r] - rows + i)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("max_rows", [1, 2])
def test_rows_past_the_most(max_rows, causal):
    """Requests that list more rows than max_rows: the first ones are worked on, at the positions that they have among all of them."""
    lens, rows = [40, 70, 5], [3, 4, 1]
    pool = Pages(lens, 3, 32, 2, 64, False, False, seed=3).fill()
    start = torch.tensor([0, 3, 7, 8], dtype=torch.int32, device=DEV)
    batch = fb.make_paged_batch(torch.tensor(lens, dtype=torch.int32, device=DEV), pool.table.to(DEV), start, max_rows, 9)
    q = torch.randn((9, 4, 64), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    out, lse = torch.full_like(q, 5.0), torch.full((9, 4), 6.0, device=DEV)
    fb.paged_attn(q, pool.cache, batch, causal, out, lse, workspace(pool.cache, batch, 4))
    out, lse, q, first, worked = out.cpu(), lse.cpu(), q.cpu().double(), [0, 3, 7], []
    for r in range(3):
        j, k, v = pool.rows(r, lens[r])
        for i in range(min(rows[r], max_rows)):
            at = first[r] + i
            worked.append(at)
            seen = j[None] <= lens[r] - rows[r] + i if causal else torch.ones((1, j.numel()), dtype=torch.bool)
            for h in range(4):
                check_attention(out[at:at + 1, h], lse[at:at + 1, h], attend64(q[at:at + 1, h], k[:, h // 2], v[:, h // 2], seen))
    rest = [i for i in range(9) if i not in worked]
    assert bool((out[rest] == 5.0).all()) and bool((lse[rest] == 6.0).all())


@pytest.mark.gpu
def test_attention_extreme_logits():
    """One key far above the others, all keys equal, logits that overflow an exponential."""
    pool = Pages([3000, 50], 94, 32, 1, 64, False, False).fill()
    pool.k[:, :, :, 0] = torch.where(pool.k[:, :, :, 0].isnan(), math.nan, 0.0).bfloat16()
    page = int(pool.table[0, 2999 // 32])
    pool.k[page, 0, 2999 % 32, 0] = 100.0
    q = torch.zeros((2, 1, 64)).bfloat16()
    q[0, 0, 0] = 200.0  # 2500 against 0
    out, _ = run_attention(pool, [3000, 50], q=q)
    assert torch.equal(out[0, 0], pool.v[page, 0, 2999 % 32].cpu())


@pytest.mark.gpu
def test_attention_of_far_pages():
    """Pages past 2^32 bytes, of which only a few hold rows."""
    n = (1 << 32) // (16 * 4 * 128 * 2) + 40
    k, v = (torch.empty((n, 4, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cache = fb.make_paged_cache(k, v)
    table = torch.tensor([[n - 1, 2, n - 7], [n - 30, n - 2, 0]], dtype=torch.int32, device=DEV)
    batch = fb.make_paged_batch(torch.tensor([41, 33], dtype=torch.int32, device=DEV), table, torch.tensor([0, 41, 74], dtype=torch.int32, device=DEV), 41, 74)
    g = torch.Generator().manual_seed(9)
    new_k, new_v, q = (torch.randn((74, h, 128), generator=g).bfloat16().to(DEV) for h in (4, 4, 8))
    fb.paged_append(cache, batch, new_k, new_v)
    out, lse = torch.empty_like(q), torch.empty((74, 8), device=DEV)
    fb.paged_attn(q, cache, batch, True, out, lse, workspace(cache, batch, 8))
    out, lse, q, new_k, new_v = out.cpu(), lse.cpu(), q.cpu().double(), new_k.cpu().double(), new_v.cpu().double()
    for rows in (slice(0, 41), slice(41, 74)):
        m = rows.stop - rows.start
        for h in range(8):
            check_attention(out[rows, h], lse[rows, h], attend64(q[rows, h], new_k[rows, h // 2], new_v[rows, h // 2], torch.ones((m, m)).tril().bool()))


@pytest.mark.gpu
def test_the_longest_table():
    """Two pages short of 2^31 - 1 rows, of which the first and the last exist: the last tile of 32 keys ends behind the last 32-bit number."""
    page, width = 42966, 49981
    assert page * width == 2 ** 31 - 2
    g = torch.Generator().manual_seed(11)
    k, v = (torch.randn((2, 1, page, 64), generator=g).bfloat16().to(DEV) for _ in range(2))
    q = torch.randn((1, 2, 64), generator=g).bfloat16().to(DEV)
    cache = fb.make_paged_cache(k, v)
    table = torch.full((1, width), -1, dtype=torch.int32, device=DEV)
    table[0, 0], table[0, -1] = 0, 1
    batch = fb.make_paged_batch(torch.tensor([2 ** 31 - 1], dtype=torch.int32, device=DEV), table)
    out, lse = torch.empty_like(q), torch.empty((1, 2), device=DEV)
    fb.paged_attn(q, cache, batch, False, out, lse, workspace(cache, batch, 2))
    keys, vals = (t.cpu().double().reshape(2 * page, 64) for t in (k, v))
    for h in range(2):
        check_attention(out.cpu()[:, h], lse.cpu()[:, h], attend64(q.cpu().double()[:, h], keys, vals, torch.ones((1, 2 * page), dtype=torch.bool)))


@pytest.mark.gpu
@pytest.mark.parametrize("page,d", [(16, 128), (24, 64)])
def test_pages_and_tables_within_larger_tensors(page, d):
    """K and V side by side in one pool with room between its rows, a table that is a part of a wider one, queries and results in wider rows."""
    H, group, n_pages, lens, rows = 3, 2, 40, [130, 5, 77], [3, 1, 2]
    pool = torch.full((n_pages, 2, page, H, d + 8), math.nan, dtype=torch.bfloat16, device=DEV)
    k, v = (pool[:, i, :, :, :d].transpose(1, 2) for i in range(2))
    cache = fb.make_paged_cache(k, v)
    width = -(-130 // page)
    g = torch.Generator().manual_seed(11)
    wide = torch.full((3, width + 5), -7, dtype=torch.int32)
    wide[:, 2:2 + width] = torch.randperm(n_pages, generator=g)[:3 * width].view(3, width).int()
    table = wide.to(DEV)[:, 2:2 + width]
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    history = [torch.randn((2, n, H, d), generator=g).bfloat16() for n in lens]
    start = torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device=DEV)
    fill = fb.make_paged_batch(seq, table, start, max(lens), sum(lens))
    new = torch.cat(history, 1).to(DEV)
    fb.paged_append(cache, fill, new[0], new[1])
    assert bool(pool[..., d:].isnan().all())
    n = sum(rows)
    batch = fb.make_paged_batch(seq, table, torch.tensor([0, *np.cumsum(rows)], dtype=torch.int32, device=DEV), max(rows), n)
    q = torch.randn((n, H * group + 1, 2 * d), generator=g).bfloat16().to(DEV)[:, 1:, d:]
    room = torch.full((n, 2 * H * group, d), 4.0, dtype=torch.bfloat16, device=DEV)
    out, lse = room[:, ::2], torch.zeros((n, H * group), device=DEV)
    fb.paged_attn(q, cache, batch, True, out, lse, workspace(cache, batch, H * group))
    assert bool((room[:, 1::2] == 4.0).all())
    for r, past in enumerate(history):
        at = [i for i, s, _ in places(lens, rows) if s == r]
        seen = torch.arange(lens[r])[None] <= torch.tensor([p for _, s, p in places(lens, rows) if s == r])[:, None]
        for h in range(H * group):
            ref = attend64(q[at, h].cpu().double(), past[0, :, h // group].double(), past[1, :, h // group].double(), seen)
            check_attention(out[at, h].cpu(), lse[at, h].cpu(), ref)


@pytest.mark.gpu
def test_same_bits_and_other_streams():
    pool = Pages([900, 33, 4000], 251, 16, 2, 128, False, True).fill()
    batch = batch_of([900, 33, 4000], pool.table)
    q = torch.randn((3, 8, 128), generator=torch.Generator().manual_seed(4)).bfloat16().to(DEV)
    results = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s in streams * 2:
        out, lse, ws = torch.empty_like(q), torch.empty((3, 8), device=DEV), workspace(pool.cache, batch, 8)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            fb.paged_attn(q, pool.cache, batch, False, out, lse, ws)
        results.append((out, lse, ws))
    torch.cuda.synchronize()
    for out, lse, _ in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])


@pytest.mark.gpu
def test_a_run_of_them_captured():
    """Append, turn and attend in one graph, replayed while the requests grow; a second graph shares the workspace."""
    H, group, d, page, width = 2, 4, 128, 16, 40
    lens = [1, 300, 64]
    pool = Pages([l - 1 for l in lens], width, page, H, d, False, False).fill()
    seq, table = torch.tensor(lens, dtype=torch.int32, device=DEV), pool.table.to(DEV)
    batch = fb.make_paged_batch(seq, table)
    g = torch.Generator().manual_seed(6)
    k, v, q, q_out, out = (torch.zeros((3, h, d), dtype=torch.bfloat16, device=DEV) for h in (H, H, H * group, H * group, H * group))
    lse, spin = torch.zeros((3, H * group), device=DEV), rotation(d)
    ws = workspace(pool.cache, batch, H * group)

    def step():
        fb.paged_append(pool.cache, batch, k, v, spin, q, q_out)
        fb.paged_attn(q_out, pool.cache, batch, False, out, lse, ws)
    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            step()
    now = list(lens)
    for turn in range(5):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g).bfloat16())
        out.fill_(3.0)
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        for r, n in enumerate(now):
            j, keys, vals = pool.rows(r, n)
            mine = torch.from_numpy(turned32(k[r:r + 1].float().cpu().numpy(), np.array([n - 1]), freqs(d), False)).bfloat16()
            assert torch.equal(keys[-1], mine[0].double()) and torch.equal(vals[-1], v[r].cpu().double())
            for h in range(H * group):
                check_attention(out[r:r + 1, h].cpu(), lse[r:r + 1, h].cpu(),
                                attend64(q_out[r:r + 1, h].cpu().double(), keys[:, h // group], vals[:, h // group], torch.ones((1, n), dtype=torch.bool)))
        seq.add_(1)
        now = [n + 1 for n in now]


@pytest.mark.gpu
def test_binding_refuses():
    pool = Pages([20], 2, 16, 2, 64, False, False)
    batch = batch_of([20], pool.table)
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        fb.rotary(x, x[:, :1], None, 0, rotation(64))
    with pytest.raises(TypeError):
        fb.rotary(x, x.float(), None, 0, rotation(64))
    with pytest.raises(TypeError):
        fb.rotary(x, x, torch.zeros(1, dtype=torch.int64, device=DEV), 0, rotation(64))
    with pytest.raises(TypeError):
        fb.make_rotation(torch.ones(32, device=DEV))
    with pytest.raises(ValueError):
        fb.make_paged_cache(pool.k, pool.v[:, :1])
    with pytest.raises(TypeError):
        fb.make_paged_cache(pool.k.float(), pool.v)
    with pytest.raises(ValueError):
        fb.make_paged_batch(torch.ones(2, dtype=torch.int32, device=DEV), pool.table.to(DEV))
    with pytest.raises(ValueError):
        fb.paged_append(pool.cache, batch, x[:, :1], x[:, :1])
    with pytest.raises(ValueError):
        fb.paged_append(pool.cache, batch, x, x, None, x)
    with pytest.raises(fb.FocusError):
        fb.paged_attn(torch.zeros((1, 3, 64), dtype=torch.bfloat16, device=DEV), pool.cache, batch, False, torch.zeros((1, 3, 64), dtype=torch.bfloat16, device=DEV), None,
                      torch.empty(1 << 20, dtype=torch.uint8, device=DEV))
    with pytest.raises(fb.FocusError):
        fb.paged_attn(x, pool.cache, batch, False, torch.empty_like(x), None, None)
    with pytest.raises(ValueError):
        fb.paged_attn(x, pool.cache, batch, False, torch.empty_like(x), torch.empty((1, 1), device=DEV), workspace(pool.cache, batch, 2))


@pytest.mark.gpu
def test_exponents_of_single_heads_and_rows():
    """Strides along an axis of one mean nothing: exponents that differ in those alone are common, and an expanded one is no stride of zero."""
    k, v = (torch.zeros((6, 1, 1, 64), dtype=torch.uint8, device=DEV) for _ in range(2))
    k_exp = torch.zeros((6, 5, 7), dtype=torch.uint8, device=DEV)[:, :1, :1]
    v_exp = torch.as_strided(torch.zeros(6 * 35, dtype=torch.uint8, device=DEV), (6, 1, 1), (35, 0, 0))
    assert k_exp.stride() != v_exp.stride() and v_exp.stride(2) == 0
    cache = fb.make_paged_cache(k, v, k_exp, v_exp)
    table = torch.tensor([[4, 2, 5]], dtype=torch.int32, device=DEV)
    batch = fb.make_paged_batch(torch.tensor([3], dtype=torch.int32, device=DEV), table, torch.tensor([0, 3], dtype=torch.int32, device=DEV), 3, 3)
    x = torch.randn((2, 3, 1, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
    fb.paged_append(cache, batch, x[0].to(DEV), x[1].to(DEV))
    for t, e, rows in ((k, k_exp, x[0]), (v, v_exp, x[1])):
        codes, exps = e4m3_rows(rows[:, 0].float().numpy())
        assert np.array_equal(t[[4, 2, 5], 0, 0].cpu().numpy(), codes) and np.array_equal(e[[4, 2, 5], 0, 0].cpu().numpy(), exps)
    with pytest.raises(ValueError, match="common strides"):
        fb.make_paged_cache(k, v, k_exp, torch.zeros((6, 1, 1), dtype=torch.uint8, device=DEV))


@pytest.mark.gpu
@pytest.mark.parametrize("first,fine", [(2 ** 31 - 1, True), (-2 ** 31, True), (2 ** 31, False), (2 ** 32, False), (-2 ** 31 - 1, False)])
def test_positions_past_32_bits(first, fine):
    x = torch.randn((2, 1, 64), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    out = torch.full_like(x, 3.0)
    if not fine:
        with pytest.raises(ValueError, match="pos_base"):
            fb.rotary(x, out, None, first, rotation(64))
        assert bool((out == 3.0).all())
        return
    fb.rotary(x, out, None, first, rotation(64))
    assert np.array_equal(bits(out), bf16_bits(turned32(x.float().cpu().numpy(), np.arange(2) + first, freqs(64), False)))


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("group,rows", [(2, 3), (12, 3)])
def test_rows_beside_a_query_that_is_not_finite(group, rows, quant):
    """A NaN or an infinity in one query row: that row is NaN, those of the same request and of the others are as without it."""
    lens = [100, 45]
    pool = Pages(lens, 7, 16, 2, 64, quant, False).fill()
    batch = batch_of(lens, pool.table, [rows] * 2)
    q = torch.randn((2 * rows, 2 * group, 64), generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    results = []
    for bad in (None, math.nan, math.inf):
        x = q.clone()
        if bad is not None:
            x[1, group - 1, 7] = bad
        out, lse = torch.empty_like(x), torch.empty((2 * rows, 2 * group), device=DEV)
        fb.paged_attn(x, pool.cache, batch, True, out, lse, workspace(pool.cache, batch, 2 * group))
        results.append((out, lse))
    there = torch.zeros((2 * rows, 2 * group), dtype=torch.bool, device=DEV)
    there[1, group - 1] = True
    for out, lse in results[1:]:
        assert bool(out[there].isnan().all()) and torch.equal(out[~there], results[0][0][~there]) and torch.equal(lse[~there], results[0][1][~there])


@pytest.mark.gpu
@pytest.mark.parametrize("group", [4, 12])
def test_bf16_memory_that_was_never_written_does_not_reach_earlier_rows(group):
    """NaN in K and V of all positions behind the rows, in their own tiles and in whole ones."""
    lens, positions, rows = [100, 300], [60, 3, 0, 33, 36, 31, 20], [4, 3]
    pool = Pages(lens, 19, 16, 2, 128, False, True, seed=group)
    pool.lens = [61, 37]
    pool.fill()
    batch = batch_of(lens, pool.table, rows, positions)
    q = torch.randn((7, 2 * group, 128), generator=torch.Generator().manual_seed(3)).bfloat16()
    out, lse = torch.empty((7, 2 * group, 128), dtype=torch.bfloat16, device=DEV), torch.empty((7, 2 * group), device=DEV)
    fb.paged_attn(q.to(DEV), pool.cache, batch, True, out, lse, workspace(pool.cache, batch, 2 * group))
    for at, r, p in places(lens, rows, positions):
        j, k, v = pool.rows(r, p + 1)
        for h in range(2 * group):
            check_attention(out[at:at + 1, h].cpu(), lse[at:at + 1, h].cpu(),
                            attend64(q[at:at + 1, h].double(), k[:, h // group], v[:, h // group], torch.ones((1, p + 1), dtype=torch.bool)))
