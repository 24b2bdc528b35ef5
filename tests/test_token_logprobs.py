"""Log probabilities of given tokens, entropies and likeliest tokens: against the definitions in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2602_02159_amd import binding as fb

DEV = "cuda:0"
BIGGEST = 3.4028234663852886e38


def exact(z, targets, masked, top):
    """numpy float64 rows, as the header says."""
    z = np.where(np.isnan(z), -np.inf, np.minimum(z, BIGGEST))
    n, V = z.shape
    logprob, entropy = np.zeros(n), np.zeros(n)
    ids, best = np.full((n, top), -1), np.full((n, top), -np.inf)
    for i in range(n):
        if masked is not None and not masked[i]:
            continue
        m = z[i].max()
        there = targets is not None and 0 <= targets[i] < V
        if m == -np.inf:
            logprob[i] = -np.inf if there else 0.0
            continue
        y = z[i] - m
        w = np.exp(y)
        rest = np.sort(w)[:-1].sum()
        total = math.log1p(rest)
        lp = y - total
        if there:
            logprob[i] = lp[targets[i]]
        entropy[i] = total - (w[w > 0] * y[w > 0]).sum() / (1 + rest)
        order = np.lexsort((np.arange(V), -z[i]))[:top]
        order = order[z[i][order] > -np.inf]
        ids[i, :order.size], best[i, :order.size] = order, lp[order]
    return logprob, entropy, ids, best


def close(got, want, V, scale=None):
    """Weights are good to 2^-20 of themselves (the exponent is a product rounded to 32 bits, at most 2^-24 of 30 where a weight counts, and exp2's
    own 2^-22), their sum of V terms in a tree of 32 and log2 V levels to 2^-18, and so is log1p of it; then one subtraction: 2^-23 of both sides.
    A weight below 2^-126, the least normal number of 32 bits, may be zero: V of them are V 2^-126 (times y, at most 2^8 where a weight is 2^-149 or more)."""
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want)
    sure = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), sure) and np.array_equal(got[~sure], want[~sure])
    tol = 2.0 ** -18 * np.minimum(np.abs(want), 1.0) + 2.0 ** -22 * np.abs(want) + V * 2.0 ** -118
    if scale is not None:
        tol = tol + scale
    assert (np.abs(got - want)[sure] <= (tol * np.ones_like(want))[sure]).all(), np.max(np.abs(got - want)[sure] / (tol * np.ones_like(want))[sure])


def run(logits, targets, masked, top):
    n, V = logits.shape
    out = [torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV), torch.full((n, top), 77, dtype=torch.int32, device=DEV), torch.full((n, top), 7.0, device=DEV)]
    t = None if targets is None else torch.tensor(targets, dtype=torch.int32, device=DEV)
    m = None if masked is None else torch.tensor(masked, dtype=torch.uint8, device=DEV)
    ws = torch.full((fb.token_logprobs_workspace(n, V, top),), 0xff, dtype=torch.uint8, device=DEV)
    fb.token_logprobs(logits, t, m, None if t is None else out[0], out[1], out[2] if top else None, out[3] if top else None, ws)
    return [x.cpu().numpy() for x in out]


def check(z, targets, masked, top):
    V = z.shape[1]
    got = run(z, targets, masked, top)
    want = exact(z.double().cpu().numpy(), targets, masked, top)
    if targets is not None:
        close(got[0], want[0], V)
    close(got[1], want[1], V, scale=2.0 ** -22 * np.log(V))
    if top:
        assert np.array_equal(got[2], want[2])
        close(got[3], want[3], V)


def rows_of(n, V, dtype, seed=0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((n, V), generator=g) * spread
    stride = -(-V // 8) * 8 + 8
    buffer = torch.full((n, stride), math.nan, dtype=dtype, device=DEV)
    buffer[:, :V] = z.to(dtype)
    return buffer[:, :V]


# ---- arguments, on the host ---------------------------------------------------------------------------------------------------
def test_refused():
    L, P = fb.lib(), C.c_void_p(1 << 20)
    call = lambda z=P, dtype=0, stride=104, t=P, n=4, V=100, top=5, lp=P, ids=P, best=P, ws=P, size=1 << 30: L.focus_token_logprobs(
        z, dtype, stride, t, None, n, V, top, lp, P, ids, best, ws, size, None)
    assert call(z=None) == call(t=None) == call(lp=None) == call(ids=None) == call(best=None) == call(z=C.c_void_p(8)) == fb.FOCUS_EINVAL
    assert call(stride=96) == call(stride=108) == call(n=0) == call(n=65536) == call(V=0) == call(V=(1 << 21) + 1, stride=1 << 22) == call(top=33) == call(top=-1) == fb.FOCUS_EINVAL
    assert call(dtype=2) == call(dtype=-1) == fb.FOCUS_EUNSUPPORTED
    need = fb.token_logprobs_workspace(4, 100, 5)
    assert need > 0 and call(size=need - 1) == call(ws=None) == call(ws=C.c_void_p((1 << 20) + 4)) == fb.FOCUS_EWORKSPACE
    for bad in ((0, 100, 5), (65536, 100, 5), (4, 0, 5), (4, (1 << 21) + 1, 5), (4, 100, 33), (4, 100, -1)):
        assert fb.token_logprobs_workspace(*bad) == 0
    for V in (1, 8192, 8193, 1 << 21):
        assert all(fb.token_logprobs_workspace(n, V, 7) <= fb.token_logprobs_workspace(n + 1, V, 7) for n in (1, 2, 63, 500))


# ---- on the GPU ---------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,top", [(1, 1, 1), (3, 2, 5), (2, 7, 32), (5, 100, 20), (1, 8191, 3), (4, 8192, 20), (3, 8193, 20), (7, 32003, 5), (2, 126464, 20), (65, 1000, 0),
                                     (1, 1 << 21, 32), (300, 17, 1)])
def test_rows(n, V, top, dtype):
    rng = np.random.default_rng(V)
    check(rows_of(n, V, dtype, seed=V), [int(x) for x in rng.integers(0, V, n)], None, top)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_rows_targets_outside_and_empty_rows(dtype):
    z = rows_of(9, 9000, dtype)
    z[3] = -math.inf
    z[4, :8999] = -math.inf
    z[5] = math.nan
    z[6, 10:] = -math.inf
    check(z, [5, -1, 9000, 7, 8999, 0, 10, 3, 2 ** 31 - 1], [1, 1, 1, 1, 1, 1, 1, 0, 1], 20)
    check(z, None, [0, 2, 255, 0, 1, 0, 0, 0, 1], 3)
    check(z, [1] * 9, [0] * 9, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_special_logits(dtype):
    z = rows_of(6, 20000, dtype)
    z[0, 17000] = math.inf
    z[1, 5], z[1, 6], z[1, 19999] = math.inf, math.inf, math.nan
    z[2, ::3] = math.nan
    z[3] *= 1e30
    z[4, 8191] = 300.0  # certain: what the others have left is below 2^-149
    z[5] = 0.0
    z[5, 1::2] = -0.0
    check(z, [17000, 5, 1, 77, 8191, 19999], None, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [600, 8192, 40000])
def test_ties(dtype, V):
    """Equal logits: all of them, more than a list holds, across parts; the lower id first."""
    z = rows_of(5, V, dtype, seed=1)
    z[0] = 1.5
    z[1] = (z[1] * 0.5).round()
    z[2, :] = -2.0
    z[2, V // 2:V // 2 + 10] = 4.0
    z[3, 3::7] = 30.0
    z[4] = z[4].clamp(max=2.0)
    check(z, [0, 1, V - 1, 3, V // 2], None, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,top", [(1000, 32), (2040, 20), (40000, 32), (131071, 3)])
def test_ordered_rows(dtype, V, top):
    """Close logits in ascending order, each of them better than all before, and in descending; runs of neighbours that alone are above -inf."""
    rows = torch.full((6, (V + 7) // 8 * 8), -math.inf)  # of which the kernels see V
    z = rows[:, :V]
    z[0] = 3.0 + torch.arange(V) * 1e-5
    z[1] = z[0].flip(0)
    z[2, 600:640] = torch.arange(40) * 0.25
    z[3, V // 8:V // 2] = 1.0
    z[4] = -1.0
    z[4, -50:] = torch.arange(50) * 0.5
    z[5] = (torch.arange(V) % 1500) * 1e-4
    check(rows.to(dtype).to(DEV)[:, :V], [0, V - 1, 620, V // 4, V - 1, 7], None, top)


@pytest.mark.gpu
def test_rows_that_are_all_but_certain():
    """1 - p down to 2^-60: log1p keeps its digits."""
    z = torch.full((40, 5000), -math.inf)
    z[:, 123] = 0.0
    z[:, 4000] = -torch.arange(1, 41).float()
    check(z.to(DEV), [123 if i % 2 else 4000 for i in range(40)], None, 3)


@pytest.mark.gpu
def test_differences_and_the_same_bits():
    """d logprob_t / d z_t = 1 - p_t and d entropy / d z_j = -p_j (log p_j + entropy), by differences of the kernel's own results; calls repeat
    themselves; a row does not depend on those beside it."""
    z = rows_of(3, 500, torch.float32, seed=3, spread=1.0)
    t = [7, 100, 499]
    base = run(z, t, None, 20)
    again = run(z, t, None, 20)
    assert all(np.array_equal(a, b) for a, b in zip(base, again))
    alone = run(z[1:2], t[1:2], None, 20)
    assert all(np.array_equal(a[1:2], b) for a, b in zip(base, alone))
    p = torch.softmax(z.double(), 1).cpu().numpy()
    h = 2.0 ** -4
    for i, j in enumerate(t):
        up, down = z.clone(), z.clone()
        up[i, j] += h
        down[i, j] -= h
        a, b = run(up, t, None, 0), run(down, t, None, 0)
        want = [1 - p[i, j], -p[i, j] * (math.log(p[i, j]) + base[1][i])]
        for k in range(2):  # differences of two values good to 2^-21 of up to 8, and h^2 / 6 of third derivatives, at most 1 and log V
            assert abs((float(a[k][i]) - float(b[k][i])) / (2 * h) - want[k]) <= 2.0 ** -18 / h + h * h


@pytest.mark.gpu
def test_captured():
    z = rows_of(4, 33000, torch.bfloat16)
    t = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device=DEV)
    lp, ent, ids, best = torch.zeros(4, device=DEV), torch.zeros(4, device=DEV), torch.zeros((4, 8), dtype=torch.int32, device=DEV), torch.zeros((4, 8), device=DEV)
    ws = torch.empty(fb.token_logprobs_workspace(4, 33000, 8), dtype=torch.uint8, device=DEV)
    fb.token_logprobs(z, t, None, lp, ent, ids, best, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fb.token_logprobs(z, t, None, lp, ent, ids, best, ws)
    for turn in range(4):
        z.copy_(torch.randn((4, 33000), generator=torch.Generator().manual_seed(turn)).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        want = run(z, [1, 2, 3, 4], None, 8)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip((lp, ent, ids, best), want))


@pytest.mark.gpu
def test_binding_refuses():
    z = rows_of(2, 100, torch.bfloat16)
    t, f = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    ids, best = torch.zeros((2, 4), dtype=torch.int32, device=DEV), torch.zeros((2, 4), device=DEV)
    for bad in ((z.half(), t, None, f, f, None, None), (z, t.long(), None, f, f, None, None), (z, t, None, None, f, None, None), (z, t, None, f, f[:1], None, None),
                (z, t, None, f, f, ids, None), (z, t, None, f, f, ids, best[:, :2]), (z.T, t, None, f, f, None, None), (z, t, f[:1], f, f, None, None)):
        with pytest.raises((TypeError, ValueError)):
            fb.token_logprobs(*bad, ws)
    with pytest.raises(fb.FocusError):
        fb.token_logprobs(z, t, None, f, f, ids, best, None)
