"""The quantised KV cache: writing, reading, attention and sparse layers over it, against the fp64 reference and against the bf16 entry
points over what the cache reads back as."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

from oracle import focus_oracle as fo
from oracle import step_oracle as so
from paper_2602_02159_amd import binding as fb

DEV = "cuda:0"


# ---- refusals (no GPU): validation fails before any pointer is followed
@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2602_02159_amd import build
        build.build(verbose=False)
    return fb.lib()


def _shape(**kw):
    s = fb.Shape()
    s.n_heads, s.head_dim, s.n_ctx, s.n_resp, s.block, s.n_gen = 4, 64, 1024, 32, 64, 32
    for n, rows in (("q", 32), ("k", 1056), ("v", 1056), ("o", 8)):
        setattr(s, n + "_stride_n", 64)
        setattr(s, n + "_stride_h", 64 * rows)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_refusals(L):
    fake, big = C.c_void_p(4096), 1 << 40

    def cache(**kw):
        c = fb.QuantCache(4096, 4096, 4097, 4099, 1056, 1)
        for k, v in kw.items():
            setattr(c, k, v)
        return C.byref(c)

    def update(c=cache(), s=_shape(), kn=fake, sh=512, sn=64, idx=fake, n=8):
        return L.focus_quant_update(c, C.byref(s), kn, fake, sh, sn, idx, None, n, 1024, None)

    def refresh(c=cache(), s=_shape(), kn=C.c_void_p(8192), kbar=fake, sn=64):
        return L.focus_quant_refresh(c, C.byref(s), kn, C.c_void_p(8192), 64 * 1056, sn, kbar, None)

    def read(c=cache(), s=_shape(), first=0, n=10, out=fake, sn=64):
        return L.focus_quant_read(c, C.byref(s), first, n, out, fake, 640, sn, None)

    def attn(c=cache(), s=_shape(), q=fake, n=8, kept=fake, keep=4, sinks=fake, sink=2, out=fake, ws=fake, nbytes=big):
        return L.focus_quant_attn(q, fake, None, n, c, C.byref(s), kept, keep, sinks, sink, out, None, ws, nbytes, None)

    def layer(c=cache(), s=_shape(), focus=fake, nf=8, kbar=fake, keep=4, ws=fake, nbytes=big):
        return L.focus_quant_layer(fake, focus, fake, None, nf, 8, c, kbar, C.byref(s), keep, fake, 2, None, fake, fake, None, ws, nbytes, None)

    for call in (update, refresh, read, attn, layer):
        for bad in (dict(k=None), dict(v_exp=None), dict(k=4104), dict(exp_stride_n=0), dict(exp_stride_h=-1)):
            assert call(c=cache(**bad)) == fb.FOCUS_EINVAL, (call, bad)
        assert call(c=None) == fb.FOCUS_EINVAL
        assert call(s=_shape(k_stride_n=72)) == fb.FOCUS_EINVAL and "16" in fb.last_error()
        assert call(s=_shape(v_stride_h=64 * 1056 + 8)) == fb.FOCUS_EINVAL
        assert call(s=_shape(head_dim=96)) == fb.FOCUS_EUNSUPPORTED
        assert call(s=_shape(n_ctx=0)) == fb.FOCUS_EINVAL
        assert call(s=_shape(n_heads=70000)) == fb.FOCUS_EUNSUPPORTED
    assert update(kn=None) == update(sn=60) == update(idx=None) == update(n=0) == update(n=70000) == fb.FOCUS_EINVAL
    assert refresh(kn=None) == refresh(sn=32) == refresh(kbar=C.c_void_p(4100)) == refresh(kn=fake) == fb.FOCUS_EINVAL
    assert read(first=-1) == read(first=1050) == read(n=-1) == read(out=None) == read(sn=62) == read(out=C.c_void_p(4104)) == fb.FOCUS_EINVAL
    assert attn(q=None) == attn(n=0) == attn(n=33) == attn(keep=17) == attn(sink=1025) == attn(kept=None) == attn(sinks=None) == fb.FOCUS_EINVAL
    assert attn(out=C.c_void_p(4100)) == attn(s=_shape(o_stride_n=60)) == fb.FOCUS_EINVAL
    assert layer(focus=None) == layer(nf=0) == layer(nf=33) == layer(kbar=None) == layer(keep=17) == layer(kbar=C.c_void_p(4100)) == fb.FOCUS_EINVAL
    need = fb.workspace_bytes(fb.FN_QUANT_ATTN, _shape(), 8, 16, 2)
    assert attn(keep=16, nbytes=need - 1) == attn(keep=16, ws=None) == attn(keep=16, ws=C.c_void_p(4100)) == fb.FOCUS_EWORKSPACE
    assert layer(nbytes=fb.workspace_bytes(fb.FN_QUANT_LAYER, _shape(), 8, 4, 2) - 1) == layer(ws=None) == fb.FOCUS_EWORKSPACE
    for fn in (fb.FN_QUANT_ATTN, fb.FN_QUANT_LAYER):
        assert fb.workspace_bytes(fn, _shape(), 33) == fb.workspace_bytes(fn, _shape(), 8, 17) == fb.workspace_bytes(fn, _shape(), 8, 4, 1025) == 0


# ---- on the GPU
def _rows(H, n, d, seed, spread=3.0):
    """bf16 rows whose sizes differ by orders of magnitude from row to row and, less, within a row."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((H, n, d), generator=g) * torch.exp(spread * torch.randn((H, n, 1), generator=g))
    x[..., :3] *= 8.0
    return x.to(torch.bfloat16)


class Cache:
    """A cache of H x L rows with rows, heads and exponents further apart than they need to be, filled with `fill` bytes."""

    def __init__(self, H, L, d, block, n_ctx, layout="heads", fill=0):
        u8 = lambda *s: torch.full(s, fill, dtype=torch.uint8, device=DEV)
        if layout == "heads":
            k, v, e = u8(H, L, d), u8(H, L, d), u8(2, H, L)
            self.k, self.v, self.k_exp, self.v_exp = k, v, e[0], e[1]
        elif layout == "rows":  # [L, H, d] storage
            self.k, self.v = u8(L, H, d).transpose(0, 1), u8(L, H, d).transpose(0, 1)
            self.k_exp, self.v_exp = u8(L, H).T, u8(L, H).T
        else:  # padded rows and heads
            self.k, self.v = u8(H, L + 3, d + 16)[:, :L, :d], u8(H, L + 1, d + 48)[:, 1:, 16:16 + d]
            self.k_exp, self.v_exp = u8(H, L + 5, 3)[:, :L, 1], u8(H, L + 5, 3)[:, 2:L + 2, 2]
        self.struct = fb.make_quant_cache(self.k, self.v, self.k_exp, self.v_exp)
        self.block, self.n_ctx = block, n_ctx

    def shape(self, q=None, out=None):
        return fb.make_shape(self.k if q is None else q, self.k, self.v, self.n_ctx, self.block, out)

    def put(self, k, v):
        """What the reference writes."""
        for x, codes, exps in ((k, self.k, self.k_exp), (v, self.v, self.v_exp)):
            c, e = so.quantise_rows(x.double().numpy())
            codes.copy_(torch.from_numpy(c))
            exps.copy_(torch.from_numpy(e))
        return self

    def read(self):
        out = torch.empty((2, *self.k.shape), dtype=torch.bfloat16, device=DEV)
        fb.quant_read(self.struct, self.shape(), 0, out[0], out[1])
        return out[0], out[1]

    def bytes(self):
        return [t.cpu().numpy() for t in (self.k, self.v, self.k_exp, self.v_exp)]


def _same_codes(a, b):
    v = so.e4m3_values()
    return np.array_equal(v[a], v[b], equal_nan=True) and np.array_equal(a[~np.isnan(v[a])], b[~np.isnan(v[b])])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["heads", "rows", "padded"])
def test_update_writes_the_listed_rows_and_no_other(d, layout):
    H, M, N, n = 3, 70, 21, 37
    k, v = _rows(H, n, d, 1), _rows(H, n, d, 2, 20.0)
    idx = np.array([5, -1, 20, 0, 7, 400, 3, 5, 9, 11, 7, 12, 13, 14, 15, 16, 17, 18, 19, -90, 5, 1, 2] + list(range(21, 35)))  # 5 and 7 repeat
    assert idx.size == n
    for n_act, base in ((n, M - 14), (9, 0), (0, 3), (1, -4)):
        c = Cache(H, M + N, d, 16, M, layout, fill=0x5a)
        want = [t.copy() for t in c.bytes()]
        ck, ek = so.quantise_rows(k.double().numpy())
        cv, ev = so.quantise_rows(v.double().numpy())
        for a in range(n_act):
            row = base + idx[a]
            if idx[a] >= 0 and 0 <= row < M + N:
                want[0][:, row], want[1][:, row], want[2][:, row], want[3][:, row] = ck[:, a], cv[:, a], ek[:, a], ev[:, a]
        kn, vn = torch.zeros((2, H, n, d + 8), dtype=torch.bfloat16, device=DEV)[..., :d].unbind(0)
        kn.copy_(k)
        vn.copy_(v)
        counts = torch.tensor([0, n_act], dtype=torch.int32, device=DEV)
        fb.quant_update(c.struct, c.shape(), kn, vn, torch.tensor(idx, dtype=torch.int32, device=DEV), counts, base)
        for got, ref in zip(c.bytes(), want):
            assert _same_codes(got, ref) if got.ndim == 3 else np.array_equal(got, ref), (n_act, base)


@pytest.mark.gpu
def test_update_of_a_long_list_that_repeats_itself():
    H, M, n, d = 1, 300, 1000, 64
    k, v = _rows(H, n, d, 3), _rows(H, n, d, 4)
    idx = np.random.default_rng(5).integers(0, M, n)
    c = Cache(H, M, d, 32, M)
    fb.quant_update(c.struct, c.shape(), k.to(DEV), v.to(DEV), torch.tensor(idx, dtype=torch.int32, device=DEV), None, 0)
    last = {int(i): a for a, i in enumerate(idx)}
    rows, slots = np.array(list(last)), np.array(list(last.values()))
    ck, ek = so.quantise_rows(k.double().numpy()[:, slots])
    got = c.bytes()
    assert np.array_equal(got[0][:, rows], ck) and np.array_equal(got[2][:, rows], ek)


@pytest.mark.gpu
@pytest.mark.parametrize("H,n,n_act,d", [(7, 9001, 8999, 128), (33, 3000, 3000, 64), (2, 513, 500, 64), (3, 700, 0, 128), (1, 600, 1, 128), (70, 1500, 777, 128)])
def test_update_of_long_lists_of_many_heads(H, n, n_act, d):
    M = 9000
    rng = np.random.default_rng(n)
    idx = rng.permutation(np.concatenate([rng.permutation(M)[:n - 200], rng.integers(-3, M + 3, 200 + max(0, n - 200 - M))])[:n])
    c = Cache(H, M, d, 50, M, "padded", fill=0x5a)
    g = torch.Generator(device=DEV).manual_seed(n)
    kn, vn = (torch.randn((H, n, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    whole = Cache(H, n, d, 50, n)  # every slot's row
    fb.quant_refresh(whole.struct, whole.shape(), kn, vn, None)
    want = [t.copy() for t in c.bytes()]
    last = {int(i): a for a, i in enumerate(idx[:n_act]) if 0 <= i < M}
    rows, slots = np.array(list(last), dtype=int), np.array(list(last.values()), dtype=int)
    for w, x in zip(want, whole.bytes()):
        w[:, rows] = x[:, slots]
    fb.quant_update(c.struct, c.shape(), kn, vn, i32(idx), i32([0, n_act]), 0)
    for got, ref in zip(c.bytes(), want):
        assert np.array_equal(got, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_values_at_the_ends_of_the_formats(d):
    big = torch.finfo(torch.bfloat16).max
    special = [big, -big, 448 * 2.0 ** 119, 449 * 2.0 ** 118, 448 * 2.0 ** -110, 2.0 ** -112, 2.0 ** -120, 2.0 ** -126, 2.0 ** -133, 0.0, -0.0, 1.0, 448.0, 450.0,
               456.0, 464.0, -17.0, math.inf, -math.inf, math.nan, 1.75, 1.7578125, 15.5, 0.0175]
    rows = torch.zeros((1, len(special) + 2, d), dtype=torch.bfloat16)
    for i, s in enumerate(special):
        rows[0, i] = torch.linspace(-1, 1, d) * (s if math.isfinite(s) else 1.0)
        rows[0, i, 3] = s
        rows[0, i, 5] = s / 16 if math.isfinite(s) else s
    rows[0, -2] = torch.tensor(special * 6)[:d]
    rows[0, -1] = math.nan
    n = rows.shape[1]
    c = Cache(1, n, d, 8, n)
    fb.quant_refresh(c.struct, c.shape(), rows.to(DEV), rows.flip(1).contiguous().to(DEV), None)
    want_k, want_e = so.quantise_rows(rows.double().numpy())
    got = c.bytes()
    assert np.array_equal(got[2], want_e) and _same_codes(got[0], want_k)
    assert np.array_equal(got[3], want_e[:, ::-1]) and _same_codes(got[1], want_k[:, ::-1])
    k, v = c.read()
    assert np.array_equal(k.double().cpu().numpy(), so.read_rows(want_k, want_e), equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("H,M,N,d,B,layout", [(3, 1000, 17, 128, 128, "heads"), (2, 1000, 0, 64, 100, "rows"), (5, 257, 300, 128, 64, "padded"),
                                              (1, 1, 0, 64, 1, "heads"), (2, 33, 1, 128, 7, "padded"), (1, 513, 3, 64, 512, "heads"), (2, 50, 1, 64, 64, "rows")])
def test_refresh_writes_every_row_and_the_means_of_what_it_wrote(H, M, N, d, B, layout):
    k, v = _rows(H, M + N, d, 6), _rows(H, M + N, d, 7)
    c = Cache(H, M + N, d, B, M, layout)
    kbar = torch.full((H, -(-M // B), d), math.nan, device=DEV)
    fb.quant_refresh(c.struct, c.shape(), k.to(DEV), v.to(DEV), kbar)
    got = c.bytes()
    for x, codes, exps in ((k, got[0], got[2]), (v, got[1], got[3])):
        wc, we = so.quantise_rows(x.double().numpy())
        assert np.array_equal(codes, wc) and np.array_equal(exps, we)
    kr, _ = c.read()
    means = torch.full_like(kbar, math.nan)
    fb.block_means(kr, fb.make_shape(kr, kr, None, M, B), means)
    assert torch.equal(kbar, means)


@pytest.mark.gpu
@pytest.mark.parametrize("first,n", [(0, 300), (299, 1), (7, 130), (150, 150), (0, 1), (31, 0)])
@pytest.mark.parametrize("d,layout", [(64, "padded"), (128, "rows")])
def test_read_of_a_range(first, n, d, layout):
    H, M, N = 2, 280, 20
    c = Cache(H, M + N, d, 64, M, layout).put(_rows(H, 300, d, 8), _rows(H, 300, d, 9))
    got = c.bytes()
    out = torch.full((2, H, n + 2, d + 8), -7.0, dtype=torch.bfloat16, device=DEV)
    fb.quant_read(c.struct, c.shape(), first, out[0, :, 1:n + 1, :d], out[1, :, 1:n + 1, :d])
    for i in range(2):
        want = torch.full((H, n + 2, d + 8), -7.0, dtype=torch.float64)
        want[:, 1:n + 1, :d] = torch.from_numpy(so.read_rows(got[i][:, first:first + n], got[2 + i][:, first:first + n]))
        assert torch.equal(out[i].double().cpu(), want)


def _reference(q, k, v, active, keys):
    """fp64 attention, its log-sum-exps, the same with |v|, and how far a logit may be off by fp32 products and sums."""
    Q, K, V = (t.double().cpu().numpy() for t in (q, k, v))
    d = Q.shape[2]
    x = np.einsum("had,hjd->haj", Q[:, active], K[:, keys]) / math.sqrt(d)
    size = np.einsum("had,hjd->haj", np.abs(Q[:, active]), np.abs(K[:, keys])) / math.sqrt(d)
    top = x.max(-1, keepdims=True)
    p = np.exp(x - top)
    total = p.sum(-1, keepdims=True)
    off = size.max(-1) * (d + 4) * 2.0 ** -24
    return (p / total) @ V[:, keys], (top + np.log(total))[..., 0], (p / total) @ np.abs(V[:, keys]), off


def check_attention(out, lse, q, k, v, active, keys):
    """Output: the probabilities are rounded to bf16 as an operand (2^-8 of each), so is the output, the probabilities carry twice
    the error of a logit, and the fp32 sums and exponentials 2^-24 a key and 2^-20.  Log-sum-exp: a logit's error, the sum's, and its own
    rounding with that of the base-2 scaling."""
    ref, ref_lse, size, off = _reference(q, k, v, active, keys)
    got = out.double().cpu().numpy()[:, :len(active)]
    sums = len(keys) * 2.0 ** -24 + 2.0 ** -20
    assert np.isfinite(got).all()
    worst = np.abs(got - ref) - size * (2 * 2.0 ** -8 + 2 * off[..., None] + sums)
    assert (worst <= 2.0 ** -120).all(), worst.max()
    assert (np.abs(lse.double().cpu().numpy()[:, :len(active)] - ref_lse) <= off + sums + 2.0 ** -22 * (np.abs(ref_lse) + 1)).all()


def attn(c, q, active, counts, kept, sinks, slots=None, fill=math.nan):
    H, _, d = q.shape
    n = active.numel()
    out = torch.full((H, n, d + 8), fill, dtype=torch.bfloat16, device=DEV)[..., :d]
    lse = torch.full((H, n), fill, device=DEV)
    s = c.shape(q, out)
    ws = torch.full((max(fb.workspace_bytes(fb.FN_QUANT_ATTN, s, n, kept.numel(), sinks.numel()), 256),), 0xab, dtype=torch.uint8, device=DEV)
    fb.quant_attn(q, active, counts, c.struct, s, kept, kept.numel(), sinks, sinks.numel(), out, lse, ws)
    return out, lse


i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def key_set(M, N, B, kept, sinks):
    n_b = -(-M // B)
    rows = {r for b in kept if 0 <= b < n_b for r in range(b * B, min((b + 1) * B, M))}
    return np.array(sorted(rows | {s for s in sinks if 0 <= s < M} | set(range(M, M + N))), dtype=int)


CASES = [  # H, d, M, N, B, gen, active, slots, kept, sinks, layout
    (4, 64, 1024, 32, 64, 32, 8, 8, (1, 4, 15), (3, 70, 700), "heads"),
    (4, 128, 1024, 32, 64, 32, 16, 16, (0, 15), (), "rows"),
    (1, 128, 1, 0, 1, 1, 1, 1, (0,), (), "heads"),               # one key, one query
    (2, 64, 50, 1, 64, 3, 2, 3, (0,), (0, 49), "padded"),          # a block that is not full
    (2, 128, 999, 0, 100, 20, 17, 20, (9, 2, 5), (998, 1, 1, 250, -4, 2000, 555), "heads"),  # odd blocks, a sink list out of order, repeated, out of range
    (3, 64, 999, 257, 33, 70, 33, 40, tuple(range(0, 30, 2)), tuple(range(0, 999, 7)), "padded"),  # many sinks, three query tiles
    (2, 128, 513, 5, 1, 64, 64, 64, tuple(range(0, 513, 5)), (7,), "rows"),  # blocks of one row
    (32, 128, 2050, 64, 128, 40, 25, 40, tuple(range(17)), (), "heads"),  # a key loop, 2 tiles
    (32, 128, 2050, 64, 128, 40, 5, 5, tuple(range(17)), tuple(range(0, 2050, 41)), "heads"),
    (8, 64, 6000, 99, 128, 130, 129, 130, tuple(range(47)), (0, 5999), "rows"),  # a key loop, three query groups
    (8, 128, 6000, 99, 128, 180, 175, 180, tuple(range(3, 47)), tuple(range(0, 6000, 60)), "heads"),
    (2, 128, 40, 64, 64, 20, 20, 20, (), (), "heads"),            # response rows only
    (2, 64, 40, 0, 64, 20, 20, 20, (), (39,), "heads"),           # one sink only
    (2, 64, 400, 3, 64, 20, 20, 20, (7, -1, 3, 900), (10,), "heads"),  # block ids that do not exist
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:8])) + "-" + c[10])
def test_attention_over_the_quantised_cache(case):
    H, d, M, N, B, gen, n_act, slots, kept, sinks, layout = case
    rng = np.random.default_rng(M + d)
    c = Cache(H, M + N, d, B, M, layout).put(_rows(H, M + N, d, 10, 0.5), _rows(H, M + N, d, 11, 2.0))
    q = torch.randn((H, gen, d), generator=torch.Generator().manual_seed(12)).to(torch.bfloat16).to(DEV)
    active = np.sort(rng.permutation(gen)[:n_act])
    padded = i32(list(active) + [-1] * (slots - n_act))
    out, lse = attn(c, q, padded, i32([0, n_act]), i32(kept), i32(sinks))
    k, v = c.read()
    check_attention(out, lse, q, k, v, active, key_set(M, N, B, kept, sinks))
    assert torch.isnan(out[:, n_act:].float()).all() and torch.isnan(lse[:, n_act:]).all()  # slots past the count keep what they held
    again = attn(c, q, padded, i32([0, n_act]), i32(kept), i32(sinks))
    assert torch.equal(again[0][:, :n_act], out[:, :n_act]) and torch.equal(again[1][:, :n_act], lse[:, :n_act])


@pytest.mark.gpu
def test_attention_of_an_empty_key_set_and_of_no_query():
    c = Cache(2, 40, 64, 64, 40).put(_rows(2, 40, 64, 1), _rows(2, 40, 64, 2))
    q = torch.randn((2, 5, 64), device=DEV).to(torch.bfloat16)
    out, lse = attn(c, q, i32(range(5)), None, i32([]), i32([]))
    assert (out == 0).all() and (lse == -math.inf).all()
    out, lse = attn(c, q, i32(range(5)), i32([0, 0]), i32([0]), i32([]))
    assert torch.isnan(out.float()).all() and torch.isnan(lse).all()
    out, lse = attn(c, q, i32([0, 77, -1, 3, 4]), None, i32([0]), i32([]))  # rows that Q does not have count as zero queries
    k, v = c.read()
    want = v.double().mean(1)
    assert (out[:, 1:3].double() - want[:, None]).abs().max() <= 2.0 ** -7 * v.double().abs().mean(1).max()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_attended_may_hold_anything(d):
    H, M, N, B = 2, 300, 10, 70
    c = Cache(H, M + N, d, B, M).put(_rows(H, M + N, d, 3, 0.5), _rows(H, M + N, d, 4, 0.5))
    q = torch.randn((H, 20, d), device=DEV).to(torch.bfloat16)
    kept, sinks = (1, 4), (5, 290)
    args = (i32(range(20)), None, i32(kept), i32(sinks))
    want = attn(c, q, *args)
    keys = key_set(M, N, B, kept, sinks)
    others = np.setdiff1d(np.arange(M + N), keys)
    for t, b in ((c.k, 0x7f), (c.v, 0xff), (c.k_exp, 246), (c.v_exp, 246)):
        t[:, others] = b
    got = attn(c, q, *args)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_values_far_apart():
    """Rows of V that differ by 2^60, logits of some thousands: the exponents reach the sums without loss."""
    H, M, d = 2, 500, 128
    k, v = _rows(H, M, d, 5, 0.5), _rows(H, M, d, 6, 14.0)
    k[:, 77] *= 64.0
    c = Cache(H, M, d, 50, M).put(k, v)
    q = (4 * torch.randn((H, 9, d), generator=torch.Generator().manual_seed(1))).to(torch.bfloat16).to(DEV)
    out, lse = attn(c, q, i32(range(9)), None, i32(range(10)), i32([]))
    kr, vr = c.read()
    check_attention(out, lse, q, kr, vr, np.arange(9), np.arange(M))


@pytest.mark.gpu
@pytest.mark.parametrize("H,d,M,N,B,gen,n_act,keep,n_sink", [
    (4, 64, 1024, 32, 64, 32, 8, 4, 2), (32, 128, 4096, 64, 128, 64, 16, 6, 4), (5, 128, 3000, 49, 100, 49, 20, 7, 100),
    (2, 64, 20000, 30, 64, 80, 70, 60, 40), (3, 128, 20000, 30, 16, 40, 9, 100, 4), (2, 64, 20000, 10, 8, 40, 9, 30, 4), (2, 64, 300, 10, 64, 40, 9, 0, 4)])
def test_layer_is_scores_then_attention_bit_for_bit(H, d, M, N, B, gen, n_act, keep, n_sink):
    """The number of blocks passes 256, 1024 and 2048."""
    n_b = -(-M // B)
    c = Cache(H, M + N, d, B, M)
    kbar = torch.empty((H, n_b, d), device=DEV)
    fb.quant_refresh(c.struct, c.shape(), _rows(H, M + N, d, 1, 0.3).to(DEV), _rows(H, M + N, d, 2, 0.3).to(DEV), kbar)
    q = torch.randn((H, gen, d), device=DEV).to(torch.bfloat16)
    n_focus = min(gen, 6)
    focus, active, counts = i32(range(n_focus)), i32(list(range(n_act)) + [-1] * 3), i32([n_focus - 1, n_act])
    sinks = i32(np.linspace(0, M - 1, n_sink).astype(int))
    out = torch.full((H, n_act + 3, d), math.nan, dtype=torch.bfloat16, device=DEV)
    lse, scores, kept = torch.full((H, n_act + 3), math.nan, device=DEV), torch.empty(n_b, device=DEV), i32([-7] * max(keep, 1))
    s = c.shape(q, out)
    ws = torch.full((fb.workspace_bytes(fb.FN_QUANT_LAYER, s, n_act + 3, keep, n_sink),), 0xcd, dtype=torch.uint8, device=DEV)
    fb.quant_layer(q, focus, active, counts, c.struct, kbar, s, keep, sinks, n_sink, scores, kept, out, lse, ws)
    ref_scores, ref_kept = torch.empty(n_b, device=DEV), i32([-7] * max(keep, 1))
    ws2 = torch.empty(fb.workspace_bytes(fb.FN_BLOCK_SCORES, s), dtype=torch.uint8, device=DEV)
    fb.block_scores(q, focus, counts, None, kbar, s, keep, ref_scores, ref_kept, ws2)
    assert torch.equal(kept, ref_kept) and torch.equal(scores, ref_scores)
    ref = attn(c, q, active, counts, ref_kept[:keep], sinks)
    assert torch.equal(out[:, :n_act], ref[0][:, :n_act]) and torch.equal(lse[:, :n_act], ref[1][:, :n_act])
    assert torch.isnan(out[:, n_act:].float()).all()
    k, v = c.read()
    lay = fo.focus_layer(*(t.float().cpu().numpy() for t in (q, k, v)), np.arange(n_focus - 1), np.arange(n_act), sinks.cpu().numpy(), M, B, keep)
    assert sorted(kept[:keep].tolist()) == sorted(lay["blocks"].tolist())
    check_attention(out, lse, q, k, v, np.arange(n_act), key_set(M, N, B, kept[:keep].tolist(), sinks.tolist()))


@pytest.mark.gpu
@pytest.mark.parametrize("d,M,N,B,n_act,keep,n_sink", [
    (128, 26000, 77, 128, 16, 204, 0), (128, 26000, 0, 64, 28, 400, 3), (128, 27000, 9, 16, 3, 1640, 2), (64, 53000, 40, 256, 32, 200, 50),
    (64, 52000, 40, 64, 7, 812, 0)])
def test_caches_of_more_than_two_hundred_megabytes(d, M, N, B, n_act, keep, n_sink):
    """Such rows pass the caches by.  The number of blocks passes 256 and 1024."""
    H, n_b, some = 32, -(-M // B), [0, 17, 31]
    c = Cache(H, M + N, d, B, M)
    g = torch.Generator(device=DEV).manual_seed(d + B)
    kbar = torch.empty((H, n_b, d), device=DEV)
    k, v = (torch.randn((H, M + N, d), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    fb.quant_refresh(c.struct, c.shape(), k, v, kbar)
    q = torch.randn((H, 40, d), generator=g, device=DEV).to(torch.bfloat16)
    focus, active, counts, sinks = i32(range(6)), i32(range(n_act)), i32([6, n_act]), i32(np.linspace(0, M - 1, n_sink).astype(int))
    out, lse = torch.full((H, n_act, d), math.nan, dtype=torch.bfloat16, device=DEV), torch.full((H, n_act), math.nan, device=DEV)
    scores, kept = torch.empty(n_b, device=DEV), i32([-7] * keep)
    s = c.shape(q, out)
    ws = torch.full((fb.workspace_bytes(fb.FN_QUANT_LAYER, s, n_act, keep, n_sink),), 0xcd, dtype=torch.uint8, device=DEV)
    fb.quant_layer(q, focus, active, counts, c.struct, kbar, s, keep, sinks, n_sink, scores, kept, out, lse, ws)
    ref = attn(c, q, active, counts, kept, sinks)
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
    k, v = c.read()
    check_attention(out[some], lse[some], q[some], k[some], v[some], np.arange(n_act), key_set(M, N, B, kept.tolist(), sinks.tolist()))


@pytest.mark.gpu
def test_rows_past_four_gigabytes():
    """One head's codes are 4.6 GB: row offsets pass 32 bits, and so do those of a row stride that is as large."""
    d, B, M = 128, 128, 36_000_000
    k, v = (torch.zeros((1, M, d), dtype=torch.uint8, device=DEV) for _ in range(2))
    e = torch.zeros((2, 1, M), dtype=torch.uint8, device=DEV)
    cache = fb.make_quant_cache(k, v, e[0], e[1])
    n = 300
    rows = np.sort(np.concatenate([np.arange(M - 200, M), np.arange(100)]))
    kn, vn = _rows(1, n, d, 1, 0.5).to(DEV), _rows(1, n, d, 2, 0.5).to(DEV)
    s = fb.make_shape(kn, k, v, M, B)
    fb.quant_update(cache, s, kn, vn, i32(rows), None, 0)
    back = torch.empty((2, 1, 200, d), dtype=torch.bfloat16, device=DEV)
    fb.quant_read(cache, s, M - 200, back[0], back[1])
    wc, we = so.quantise_rows(kn.double().cpu().numpy())
    assert np.array_equal(back[0].double().cpu().numpy(), so.read_rows(wc, we)[:, 100:])
    q = torch.randn((1, 20, d), device=DEV).to(torch.bfloat16)
    kept, sinks = [M // B - 1], [0, 5, M - 190, M - 1]
    out, lse = torch.empty((1, 20, d), dtype=torch.bfloat16, device=DEV), torch.empty((1, 20), device=DEV)
    s = fb.make_shape(q, k, v, M, B, out)
    ws = torch.empty(max(256, fb.workspace_bytes(fb.FN_QUANT_ATTN, s, 20, 1, 4)), dtype=torch.uint8, device=DEV)
    fb.quant_attn(q, i32(range(20)), None, cache, s, i32(kept), 1, i32(sinks), 4, out, lse, ws)
    keys = key_set(M, 0, B, kept, sinks)
    at = torch.from_numpy(keys).to(DEV)
    read = lambda codes, exps: torch.from_numpy(so.read_rows(codes[:, at].cpu().numpy(), exps[:, at].cpu().numpy()))
    check_attention(out, lse, q, read(k, e[0]), read(v, e[1]), np.arange(20), np.arange(len(keys)))


@pytest.mark.gpu
def test_another_stream_and_a_captured_call():
    """An update, a layer and a read captured together and replayed on new inputs, with eager work in between."""
    H, d, M, N, B, gen, n = 4, 128, 2000, 40, 64, 40, 12
    n_b = -(-M // B)
    c = Cache(H, M + N, d, B, M).put(_rows(H, M + N, d, 1, 0.3), _rows(H, M + N, d, 2, 0.3))
    kbar = torch.randn((H, n_b, d), device=DEV)
    kn, vn = _rows(H, n, d, 3, 0.3).to(DEV), _rows(H, n, d, 4, 0.3).to(DEV)
    q = torch.randn((H, gen, d), device=DEV).to(torch.bfloat16)
    active, focus, sinks = i32(range(5, 5 + n)), i32([1, 2]), i32([0, 9])
    out, lse = torch.zeros((H, n, d), dtype=torch.bfloat16, device=DEV), torch.zeros((H, n), device=DEV)
    scores, kept, back = torch.zeros(n_b, device=DEV), i32([-1] * 6), torch.zeros((2, H, M + N, d), dtype=torch.bfloat16, device=DEV)
    s = c.shape(q, out)
    ws = torch.empty(fb.workspace_bytes(fb.FN_QUANT_LAYER, s, n, 6, 2), dtype=torch.uint8, device=DEV)

    def calls():
        fb.quant_update(c.struct, s, kn, vn, active, None, M)
        fb.quant_layer(q, focus, active, None, c.struct, kbar, s, 6, sinks, 2, scores, kept, out, lse, ws)
        fb.quant_read(c.struct, s, 0, back[0], back[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        kn.copy_(_rows(H, n, d, 30 + i, 0.3))
        q.copy_(torch.randn((H, gen, d), device=DEV))
        out.zero_()
        back.zero_()
        graph.replay()
        got = [t.clone() for t in (out, lse, scores, kept, back)]
        torch.cuda.synchronize()
        calls()
        for a, b in zip(got, (out, lse, scores, kept, back)):
            assert torch.equal(a, b)
        check_attention(out, lse, q, back[0], back[1], np.arange(5, 5 + n), key_set(M, N, B, kept.tolist(), [0, 9]))


@pytest.mark.gpu
def test_another_device_than_the_current_one_is_refused(monkeypatch):
    c = Cache(1, 40, 64, 8, 40)
    s, rows = c.shape(), torch.zeros((1, 4, 64), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    s = c.shape(rows, rows)
    for call in (lambda: fb.quant_update(c.struct, s, rows, rows, i32(range(4)), None, 0), lambda: fb.quant_refresh(c.struct, s, rows, rows, None),
                 lambda: fb.quant_read(c.struct, s, 0, rows, rows), lambda: fb.quant_attn(rows, i32([0]), None, c.struct, s, i32([0]), 1, None, 0, rows, None, ws),
                 lambda: fb.quant_layer(rows, i32([0]), i32([0]), None, c.struct, rows.float(), s, 1, None, 0, None, i32([0]), rows, None, ws)):
        with pytest.raises(ValueError, match="current device"):
            call()


# ---- what the wrappers refuse, without a GPU: tensors that say that they are on one, and a library that notes its calls
class _Claims(torch.Tensor):
    is_cuda = True
    where = 0

    def get_device(self):
        return self.where


class _Noted:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append(name) or fb.FOCUS_OK


def _on(t, where=0):
    t = t.as_subclass(_Claims)
    t.where = where
    return t


@pytest.fixture
def noted(monkeypatch):
    library = _Noted()
    monkeypatch.setattr(fb, "lib", lambda: library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    return library.calls


H_, M_, N_, D_, B_, GEN_, SLOTS_ = 3, 70, 10, 64, 16, 12, 5


def _calls():
    """Arguments that fit, by name, of every wrapper over one cache."""
    u8, bf = lambda *s: _on(torch.zeros(s, dtype=torch.uint8)), lambda *s: _on(torch.zeros(s, dtype=torch.bfloat16))
    i32_, f32 = lambda n: _on(torch.zeros(n, dtype=torch.int32)), lambda *s: _on(torch.zeros(s))
    k, v, n_b = u8(H_, M_ + N_, D_), u8(H_, M_ + N_, D_), -(-M_ // B_)
    cache = fb.make_quant_cache(k, v, u8(H_, M_ + N_), u8(H_, M_ + N_))
    q, out = bf(H_, GEN_, D_), bf(H_, SLOTS_, D_)
    both = dict(cache=cache, shape=fb.make_shape(q, k, v, M_, B_, out))
    update = dict(both, k_new=bf(H_, SLOTS_, D_), v_new=bf(H_, SLOTS_, D_), active_idx=i32_(SLOTS_), counts=i32_(2), row_base=M_)
    refresh = dict(both, k_new=bf(H_, M_ + N_, D_), v_new=bf(H_, M_ + N_, D_), kbar=f32(H_, n_b, D_))
    read = dict(both, first_row=3, k_out=bf(H_, 9, D_), v_out=bf(H_, 9, D_))
    attn_ = dict(both, q=q, active_idx=i32_(SLOTS_), counts=i32_(2), kept_blocks=i32_(2), n_keep=2, sink_idx=i32_(3), n_sink=3, out=out, lse=f32(H_, SLOTS_),
                 workspace=u8(4096))
    layer = dict(attn_, focus_idx=i32_(4), kbar=f32(H_, n_b, D_), scores=f32(n_b))
    return k, v, {fb.quant_update: update, fb.quant_refresh: refresh, fb.quant_read: read, fb.quant_attn: attn_, fb.quant_layer: layer}


def test_wrappers_take_what_fits(noted):
    _, _, calls = _calls()
    for n, (call, args) in enumerate(calls.items()):
        call(**args)
        for name, t in args.items():  # more rows than a call needs, and what it does not need
            if isinstance(t, torch.Tensor) and name in ("k_new", "v_new", "out", "lse", "kept_blocks", "sink_idx", "counts", "kbar", "scores", "workspace"):
                if name not in ("k_new", "v_new", "out"):
                    call(**{**args, name: _on(torch.zeros((t.numel() + 8,), dtype=t.dtype))})
        for name in ("counts", "lse", "scores", "workspace") + (("kbar",) if call is fb.quant_refresh else ()):
            if name in args:
                call(**{**args, name: None})
        if "sink_idx" in args:
            call(**{**args, "sink_idx": None, "n_sink": 0})
    rows = _on(torch.zeros((2, H_ + 1, SLOTS_ + 4, D_ + 8), dtype=torch.bfloat16))
    fb.quant_update(**{**calls[fb.quant_update], "k_new": rows[0], "v_new": rows[1]})
    assert set(noted) == {c.__name__.replace("quant", "focus_quant") for c in calls}


def test_wrappers_refuse_tensors_that_the_kernels_would_leave(noted):
    """Fewer heads, rows, columns or values than the shape and the lists say, other types, other strides, other devices: nothing is called."""
    k, v, calls = _calls()
    bad_calls = []
    for call, args in calls.items():
        for name, t in args.items():
            if not isinstance(t, torch.Tensor):
                continue
            bad = [_on(t, 1)]  # another device
            if t.dtype != torch.uint8:  # (a workspace's type means nothing, its size is the library's to judge)
                bad.append(_on(torch.zeros(t.shape, dtype=torch.int64)))
            if t.dim() == 3 and t.dtype == torch.bfloat16:
                pair = {"k_new": "v_new", "v_new": "k_new", "k_out": "v_out", "v_out": "k_out"}.get(name)
                for axis in range(3):
                    if (call is fb.quant_read or name == "q") and axis == 1:
                        continue  # (its rows are the call's)
                    less = list(t.shape)
                    less[axis] -= 1
                    small = _on(torch.zeros(t.shape, dtype=t.dtype)[:less[0], :less[1], :less[2]])
                    bad_calls.append((call, {**args, name: small}))
                    if pair:
                        bad_calls.append((call, {**args, name: small, pair: small}))
                bad.append(_on(torch.zeros((*t.shape[:2], 2 * t.shape[2]), dtype=t.dtype)[..., ::2]))
                bad.append(_on(torch.zeros((t.shape[0], t.shape[1], t.shape[2] + 8), dtype=t.dtype)[..., :-8]))  # not those of the other or of the shape
                bad.append(t[0])
            elif name != "workspace" and name not in ("active_idx", "focus_idx"):
                bad.append(_on(torch.zeros(t.numel() - 1, dtype=t.dtype)))
                bad.append(_on(torch.zeros(2 * t.numel(), dtype=t.dtype)[::2]))
            else:
                bad.append(_on(torch.zeros(2 * t.numel(), dtype=t.dtype)[::2]))
            bad_calls += [(call, {**args, name: b}) for b in bad]
        s = args["shape"]
        for field, value in (("n_heads", H_ + 1), ("n_heads", H_ - 1), ("n_ctx", M_ + 1), ("n_resp", N_ + 7), ("head_dim", 128), ("k_stride_h", 1 << 20),
                             ("k_stride_n", 128), ("v_stride_h", 16), ("v_stride_n", 192)):
            other = fb.Shape.from_buffer_copy(s)
            setattr(other, field, value)
            bad_calls.append((call, {**args, "shape": other}))
        if call in (fb.quant_attn, fb.quant_layer):
            for field, value in (("n_gen", GEN_ + 1), ("q_stride_h", 1 << 20), ("q_stride_n", 128), ("o_stride_h", 1 << 20), ("o_stride_n", 128)):
                other = fb.Shape.from_buffer_copy(s)
                setattr(other, field, value)
                bad_calls.append((call, {**args, "shape": other}))
            bad_calls += [(call, {**args, "kept_blocks": None}), (call, {**args, "n_keep": 3}), (call, {**args, "sink_idx": None}), (call, {**args, "n_sink": 4}),
                          (call, {**args, "active_idx": _on(torch.zeros(SLOTS_ + 1, dtype=torch.int32))})]
        if call is fb.quant_update:
            bad_calls.append((call, {**args, "active_idx": _on(torch.zeros(SLOTS_ + 1, dtype=torch.int32))}))
    for call, args in bad_calls:
        with pytest.raises((TypeError, ValueError)):
            call(**args)
    assert noted == [] and len(bad_calls) > 150
    exps = _on(torch.zeros((H_, M_ + N_), dtype=torch.uint8))
    for bad in ((k[..., ::2], v[..., ::2], exps, exps), (k, v, exps, _on(exps, 1)), (k, _on(v.clone(), 1), exps, exps), (k, v, exps[:, 1:], exps), (k[0], v[0], exps, exps)):
        with pytest.raises(ValueError):
            fb.make_quant_cache(*bad)


def test_strides_of_one_head_or_one_row_mean_nothing(noted):
    u8 = lambda *s: _on(torch.zeros(s, dtype=torch.uint8))
    k, v, e = u8(1, 40, 64), u8(1, 40, 64), u8(1, 40)
    cache = fb.make_quant_cache(k, v, e, e)
    q = _on(torch.zeros((1, 9, 64), dtype=torch.bfloat16))
    out = _on(torch.zeros((1, 1, 64), dtype=torch.bfloat16))
    shape = fb.make_shape(q, k, v, 40, 8, out)
    shape.k_stride_h = shape.q_stride_h = shape.o_stride_h = shape.o_stride_n = 1 << 20
    one = _on(torch.zeros(1, dtype=torch.int32))
    fb.quant_attn(q, one, None, cache, shape, one, 1, None, 0, out, None, None)
    assert noted == ["focus_quant_attn"]
