"""focus_sample_tokens against the fp64 reference."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2602_02159_amd import binding as fb

DEV = "cuda:0"


def test_refusals():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2602_02159_amd import build
        build.build(verbose=False)
    L, fake = fb.lib(), C.c_void_p(4096)

    def call(logits=fake, dtype=0, stride=1000, uniform=fake, rows=4, vocab=1000, tokens=fake, ws=fake, nbytes=1 << 40):
        return L.focus_sample_tokens(logits, dtype, stride, None, uniform, None, None, None, None, rows, vocab, tokens, None, None, ws, nbytes, None)

    assert call(logits=None) == call(uniform=None) == call(tokens=None) == call(rows=0) == call(rows=70000) == call(vocab=0) == fb.FOCUS_EINVAL
    assert call(stride=1001) == call(stride=992) == call(logits=C.c_void_p(4104)) == call(dtype=1, stride=1002) == fb.FOCUS_EINVAL
    assert call(vocab=(1 << 21) + 1, stride=1 << 22) == fb.FOCUS_EINVAL and "vocab" in fb.last_error()
    assert call(dtype=2) == call(dtype=-1) == fb.FOCUS_EUNSUPPORTED
    need = fb.sample_tokens_workspace(4, 1000)
    assert need > 0 and call(nbytes=need - 1) == call(ws=None) == call(ws=C.c_void_p(4104)) == fb.FOCUS_EWORKSPACE
    assert fb.sample_tokens_workspace(0, 10) == fb.sample_tokens_workspace(1, 0) == fb.sample_tokens_workspace(1, (1 << 21) + 1) == 0


def run(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, masked=None, want=("conf", "prob")):
    """On [n, vocab] logits in rows further apart than they need to be; per-row values may be numbers."""
    n, V = logits.shape
    wide = logits.dtype == torch.float32
    step = 4 if wide else 8
    t = torch.full((n, (V + step - 1) // step * step + step), 50.0, dtype=logits.dtype, device=DEV)[:, :V]
    t.copy_(logits)
    row = lambda x, dtype: None if x is None else torch.tensor(np.broadcast_to(np.asarray(x), (n,)).copy(), dtype=dtype, device=DEV)
    tokens = torch.full((n,), -7, dtype=torch.int32, device=DEV)
    conf, prob = (torch.full((n,), math.nan, device=DEV) if name in want else None for name in ("conf", "prob"))
    ws = torch.full((fb.sample_tokens_workspace(n, V),), 0xab, dtype=torch.uint8, device=DEV)
    args = (t, row(masked, torch.uint8), row(u, torch.float32), row(temperature, torch.float32), row(top_k, torch.int32), row(top_p, torch.float32),
            row(min_p, torch.float32), tokens, conf, prob, ws)
    fb.sample_tokens(*args)
    back = lambda x: None if x is None else x.cpu().numpy()
    return back(tokens), back(conf), back(prob)


def check(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, got=None):
    """Tokens exactly, but where a border between two tokens lies within 2^-30 of the random number's share (the weights are good to
    about 2^-23 each, some of thousands of them err in each direction).  conf and prob: 2^-20, the weight of a token and a sum."""
    n = logits.shape[0]
    z = logits.double().cpu().numpy()
    per_row = [np.broadcast_to(np.asarray(x), (n,)) for x in (u, temperature, top_k, top_p, min_p)]
    tokens, conf, prob = got or run(logits, u, temperature, top_k, top_p, min_p)
    for i in range(n):
        ui, ti, ki, pi, mi = (float(np.float32(x[i])) if j != 2 else int(x[i]) for j, x in enumerate(per_row))
        t, c, p = so.sample_token(z[i], ui, ti, ki, pi, mi)
        if tokens[i] != t:
            near = {so.sample_token(z[i], min(max(ui + s * 2.0 ** -30, 0.0), 1.0 - 2.0 ** -40), ti, ki, pi, mi)[0] for s in (-1, 1)}
            assert int(tokens[i]) in near, (i, tokens[i], t, ui, ti, ki, pi, mi)
            continue
        assert abs(conf[i] - c) <= 2.0 ** -20 * c and abs(prob[i] - p) <= 2.0 ** -20 * p, (i, conf[i], c, prob[i], p)
    return tokens


def _logits(n, V, dtype, seed, sigma=3.0, peak=True):
    g = torch.Generator().manual_seed(seed)
    z = sigma * torch.randn((n, V), generator=g)
    if peak:
        z[torch.arange(n), torch.randint(0, V, (n,), generator=g)] += 14 * torch.rand(n, generator=g)
    return z.to(dtype)


PARAMS = [  # temperature, top_k, top_p, min_p
    (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (1.3, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (0.8, 40, 0.95, 0.02), (2.5, 1000, 0.5, 1e-4),
    (1.0, 1, 1.0, 0.0), (1.0, 3, 0.2, 0.9), (1.0, 0, 1e-6, 0.0), (1.0, 0, 0.999999, 0.0), (1.0, 0, 0.3, 1.0), (1.0, 10 ** 9, 1.0, 2.0), (30.0, 0, 0.97, 0.0)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n,V", [(5, 1), (4, 2), (7, 7), (3, 8), (9, 1000), (6, 4097), (3, 32003), (2, 126464)])
def test_every_filter(n, V, dtype):
    for i, (T, k, p, m) in enumerate(PARAMS):
        u = np.random.default_rng(V + i).random(n).astype(np.float32)
        check(_logits(n, V, dtype, 100 * i + V), u, T, k, p, m)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_values_per_row(dtype):
    n, V = 200, 3001
    rng = np.random.default_rng(1)
    T = np.where(rng.random(n) < 0.1, 0.0, rng.uniform(0.2, 2, n))
    k = np.where(rng.random(n) < 0.3, 0, np.exp(rng.uniform(0, 8, n)).astype(int))
    p = np.where(rng.random(n) < 0.3, 1.0, rng.uniform(0.01, 1, n))
    m = np.where(rng.random(n) < 0.3, 0.0, rng.uniform(0, 0.5, n) ** 3)
    check(_logits(n, V, dtype, 3), rng.random(n).astype(np.float32), T, k, p, m)


@pytest.mark.gpu
def test_ties_go_to_the_lower_id():
    V = 700
    z = torch.zeros((1, V), dtype=torch.bfloat16)
    z[0, 300:500] = 2.0  # two hundred at the top
    rows = z.repeat(9, 1)
    u = np.array([0.0, 0.1, 0.5, 0.999, 0.5, 0.5, 0.5, 0.5, 0.0], dtype=np.float32)
    k = np.array([10, 10, 10, 10, 200, 201, 1, 0, 0])
    t = check(rows, u, 1.0, k)
    assert list(t[:4]) == [300, 301, 305, 309] and t[6] == 300
    assert list(check(rows, u, 0.0, 0)) == [300] * 9
    p = np.array([0.25, 0.5, 0.01, 1e-9, 0.8, 0.9999, 0.3, 0.77, 0.6], dtype=np.float32)
    check(rows, u, 1.0, 0, p)
    check(rows, u, 1.0, 250, p, 0.1)
    check(torch.full((9, 5000), -3.0), u, 1.0, k, p)  # every logit the same
    signs = torch.tensor([[-0.0, 0.0, -0.0, 0.0]])
    assert check(signs, np.float32(0.0), 0.0)[0] == 0 and check(signs, np.float32(0.9), 1.0, 2)[0] == 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_rows_with_infinities_and_nan(dtype):
    V = 1003
    z = _logits(8, V, dtype, 4)
    z[0] = -math.inf
    z[1] = math.nan
    z[2, ::2] = -math.inf
    z[3, 1::2] = math.nan
    z[4, 7] = z[4, 900] = math.inf
    z[5] = -math.inf
    z[5, 1002] = -50.0  # one number
    z[6] = torch.finfo(dtype).min
    z[7, 5] = torch.finfo(dtype).max
    u = np.full(8, 0.6, dtype=np.float32)
    for T, k, p, m in PARAMS[:9]:
        got = run(z, u, T, k, p, m)
        assert list(got[0][:2]) == [-1, -1] and (got[1][:2] == 0).all() and (got[2][:2] == 0).all()
        assert got[0][5] == 1002 and got[2][5] == 1
        zd = z.double().numpy()
        for i in range(2, 8):
            t, c, q = so.sample_token(zd[i], float(np.float32(0.6)), T, k, float(np.float32(p)), float(np.float32(m)))
            assert got[0][i] == t and abs(got[1][i] - c) <= 2.0 ** -20 * c and abs(got[2][i] - q) <= 2.0 ** -20 * q, (i, T, k, p, m)


@pytest.mark.gpu
def test_values_that_switch_a_filter_off_and_the_ends_of_the_others():
    n, V = 6, 900
    z = _logits(n, V, torch.float32, 5)
    u = np.linspace(0, 0.9999, n).astype(np.float32)
    plain = check(z, u)
    assert list(run(z, u)[0]) == list(plain)
    for other in (dict(top_k=-5), dict(top_k=0), dict(top_k=V), dict(top_p=1.5), dict(top_p=math.nan), dict(min_p=-1.0), dict(min_p=math.nan), dict(min_p=0.0)):
        assert list(run(z, u, **other)[0]) == list(plain), other
    first = z.argmax(1).numpy()
    for other in (dict(temperature=-1.0), dict(temperature=math.nan), dict(top_k=1), dict(top_p=0.0), dict(top_p=-3.0), dict(min_p=1.0), dict(min_p=5.0),
                  dict(temperature=1e-30), dict(temperature=1e-42)):
        tokens, conf, prob = run(z, u, **other)
        assert list(tokens) == list(first) and (prob == 1).all(), other
        assert np.allclose(conf, torch.softmax(z.double(), 1).max(1).values.numpy(), rtol=2.0 ** -20, atol=0)
    flat = run(z, np.float32(0.5) + 0 * u, temperature=math.inf)[0]
    assert (np.abs(flat - V // 2) <= 1).all()
    ends = run(z, np.array([math.nan, -1.0, 1.0, 2.0, 0.0, 0.0], dtype=np.float32), top_k=3)
    kept = [so.kept_tokens(z[i].double().numpy(), 1.0, 3, 1.0, 0.0) for i in range(n)]
    assert [ends[0][i] for i in range(4)] == [kept[0][0], kept[1][0], kept[2][-1], kept[3][-1]]


@pytest.mark.gpu
def test_masked_rows_and_outputs_that_are_not_asked_for():
    n, V = 5, 500
    z, u = _logits(n, V, torch.bfloat16, 6), np.full(n, 0.4, dtype=np.float32)
    full = run(z, u, 0.9, 30)
    masked = np.array([1, 0, 255, 0, 1])
    some = run(z, u, 0.9, 30, masked=masked)
    for a, b, off in zip(full, some, (-1, 0, 0)):
        assert (b == np.where(masked > 0, a, off)).all()
    alone = run(z, u, 0.9, 30, want=())
    assert (alone[0] == full[0]).all() and alone[1] is None


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,sigma", [(1, 200000, 3.0), (300, 1000, 1.0), (2, 1 << 21, 2.0), (64, 20000, 0.0)])
def test_large_calls(n, V, sigma):
    z = _logits(n, V, torch.bfloat16, 7, sigma)
    u = np.random.default_rng(8).random(n).astype(np.float32)
    rows = np.arange(n) if n * V < 3e6 else np.arange(min(n, 2))
    got = run(z, u, 1.1, 0, 0.98, 0.0)
    check(z[rows], u[rows], 1.1, 0, 0.98, 0.0, got=[g[rows] for g in got])
    again = run(z, u, 1.1, 0, 0.98, 0.0)
    assert all((a == b).all() for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V,sigma,top_k,top_p", [(32003, 1.0, 12000, 0.5), (32003, 1.0, 12000, 0.999), (32003, 1.0, 0, 0.6), (20000, 0.6, 9000, 0.4),
                                                 (126464, 1.5, 30000, 0.8), (32003, 0.02, 9000, 0.9), (126464, 0.02, 0, 0.7)])
def test_ends_among_many_tokens_of_like_weight(V, sigma, top_k, top_p, dtype):
    """Some hundred to some thousand tokens lie within a sixteenth of a nat of where top_k and top_p end, and those places apart or not;
    at last all tokens of the row."""
    z = _logits(4, V, dtype, V + top_k, sigma, peak=False)
    check(z, np.array([0.001, 0.3, 0.7, 0.9999], dtype=np.float32), 1.0, top_k, top_p, 0.0)
    check(z, np.array([0.2, 0.4, 0.6, 0.8], dtype=np.float32), np.array([0.5, 0.9, 1.5, 4.0], dtype=np.float32), top_k, top_p, 1e-3)


@pytest.mark.gpu
def test_the_greedy_token_and_confidence_are_those_of_token_confidence():
    n, V = 40, 30000
    z = _logits(n, V, torch.bfloat16, 9)
    tokens, conf, _ = run(z, np.zeros(n, dtype=np.float32), 0.0)
    t = z.to(DEV)
    tok, cf = torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)
    fb.token_confidence(t, None, tok, cf, torch.empty(max(fb.token_confidence_workspace(n, V), 256), dtype=torch.uint8, device=DEV))
    assert (tok.cpu().numpy() == tokens).all() and np.allclose(cf.cpu().numpy(), conf, rtol=2.0 ** -18, atol=0)


@pytest.mark.gpu
def test_shares_of_many_draws():
    """Even random numbers give every token its share of them, to one draw."""
    z = torch.tensor([[0.0, 2.0, -1.0, 1.0, 0.5, -math.inf, 2.0]])
    n = 4096
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tokens = run(z.repeat(n, 1), u, 0.8, 5, 0.99, 0.01)[0]
    kept = so.kept_tokens(z[0].double().numpy(), float(np.float32(0.8)), 5, float(np.float32(0.99)), float(np.float32(0.01)))
    w = np.exp(z[0].double().numpy()[kept] / float(np.float32(0.8)))
    for t, share in zip(kept, w / w.sum()):
        assert abs((tokens == t).sum() - n * share) <= 1
    assert set(tokens) == set(kept)


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    n, V = 20, 5000
    t = _logits(n, V, torch.bfloat16, 10).to(DEV)
    u, T, k, p = torch.rand(n, device=DEV), torch.full((n,), 0.9, device=DEV), torch.full((n,), 60, dtype=torch.int32, device=DEV), torch.full((n,), 0.95, device=DEV)
    out = (torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV))
    ws = torch.empty(fb.sample_tokens_workspace(n, V), dtype=torch.uint8, device=DEV)
    call = lambda: fb.sample_tokens(t, None, u, T, k, p, None, *out, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(5):
        t.copy_(_logits(n, V, torch.bfloat16, 20 + i, peak=i % 2 == 0))
        u.copy_(torch.rand(n))
        T.fill_(0.5 + 0.3 * i)
        k.fill_(0 if i == 3 else 60)
        ws.fill_(0xee)
        graph.replay()
        got = [x.clone() for x in out]
        torch.cuda.synchronize()
        call()
        assert all(torch.equal(a, b) for a, b in zip(got, out))
        check(t.cpu(), u.cpu().numpy(), T.cpu().numpy(), k.cpu().numpy(), p.cpu().numpy(), got=[x.cpu().numpy() for x in got])


@pytest.mark.gpu
def test_tensors_that_do_not_fit_the_call_are_refused(monkeypatch):
    n, V = 4, 64
    f32 = lambda *s: torch.zeros(s, device=DEV)
    ok = dict(logits=torch.zeros((n, V), dtype=torch.bfloat16, device=DEV), masked=None, uniform=f32(n), temperature=None, top_k=None, top_p=None, min_p=None,
              tokens=torch.full((n,), -7, dtype=torch.int32, device=DEV), conf=None, prob=None,
              workspace=torch.empty(fb.sample_tokens_workspace(n, V), dtype=torch.uint8, device=DEV))
    bad = [dict(uniform=f32(n - 1)), dict(uniform=f32(2 * n)[::2]), dict(temperature=f32(n, 1)), dict(conf=f32(n - 1)), dict(prob=f32()), dict(logits=f32(n, V, 1)),
           dict(logits=f32(V, n).T), dict(masked=torch.ones(n, dtype=torch.int32, device=DEV)), dict(masked=torch.ones(n + 1, dtype=torch.uint8, device=DEV))]
    for b in bad:
        with pytest.raises(ValueError):
            fb.sample_tokens(**{**ok, **b})
    for b in (dict(top_k=f32(n)), dict(uniform=f32(n).double()), dict(uniform=torch.zeros(n)), dict(logits=torch.zeros((n, V), dtype=torch.float16, device=DEV))):
        with pytest.raises(TypeError):
            fb.sample_tokens(**{**ok, **b})
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="current device"):
            fb.sample_tokens(**ok)
    assert (ok["tokens"] == -7).all()
    fb.sample_tokens(**ok)
    assert (ok["tokens"] == 0).all()
    one = {**ok, "logits": f32(n, 63)[2:3].clone(), "uniform": f32(n, 3)[:1, 0], "tokens": ok["tokens"][:1].fill_(-7)}  # one row: its stride means nothing
    fb.sample_tokens(**one)
    assert one["tokens"].item() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("between", [1, 2, 11])
def test_weights_far_below_the_largest_keep_their_share(between, dtype):
    """Two tokens of weight 1 and, between them, some of w = exp(-17) = 0.69 * 2^-24 down to exp(-29) = 1.1 * 2^-42: whole numbers of 2^-42, all alike,
    so half of the mass ends in their middle, however small they are.  exp(-30) is 0.4 of a unit: nothing.  prob: a weight is good
    to 2^-22 of itself, and rounded."""
    V = between + 2
    for T in (1.0, 0.5, 4.0):
        down = 17.0 + np.arange(14)
        z = torch.zeros((14, V), dtype=dtype)
        z[:, 1:-1] = torch.tensor(-down[:, None] * T).to(dtype)
        tokens, _, prob = run(z, np.float32(0.5), T)
        assert list(tokens) == [1 + between // 2] * 13 + [V - 1], T
        w = np.exp(-down[:13])
        assert (np.abs(prob[:13] - w / (2 + between * w)) <= 2.0 ** -21 * w).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("n", [3, 7, 30, 200])
def test_top_p_counts_weights_far_below_the_largest(n, dtype):
    """One token of weight 1 and n of w = exp(-17) = 0.69 * 2^-24: top_p = 1 - 2^-24 leaves one of the n out, by a margin of 0.44 w (their errors
    are 200 * 2^-23 w and 100 units of 2^-42, of which w has 181 000)."""
    w, p = math.exp(-17.0), 1.0 - 2.0 ** -24
    kept = math.ceil((p * (1 + n * w) - 1) / w)
    assert kept == n - 1
    for first in (0, n):  # the largest in front, and behind
        z = torch.full((1, n + 1), -17.0, dtype=dtype)
        z[0, first] = 0.0
        cum = np.cumsum([1.0] + [w] * kept if first == 0 else [w] * kept + [1.0])
        at = int((cum <= p * cum[-1]).sum())
        want = n if first == n and at == kept else at
        tokens, _, prob = run(z, np.float32(p), 1.0, 0, np.float32(p))
        assert tokens[0] == want, first
        share = (1.0 if want == first else w) / cum[-1]
        assert abs(prob[0] - share) <= 2.0 ** -21 * share


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [9000, 126464])
def test_a_row_gives_the_same_token_alone_and_among_others(V, dtype):
    """The ends and borders do not hang on how a row is cut into slices, which follows from the number of rows."""
    n = 130 if V == 9000 else 40
    z = _logits(n, V, dtype, 77, 2.0)
    rng = np.random.default_rng(6)
    u, T, k, p = rng.random(n).astype(np.float32), rng.uniform(0.3, 1.5, n), rng.choice([0, 0, 1000], n), rng.choice([0.5, 0.9, 0.99, 1.0], n)
    tokens, _, prob = run(z, u, T, k, p, 1e-6)
    for i0 in range(0, n, 5):
        at = slice(i0, i0 + 5)
        some = run(z[at], u[at], T[at], k[at], p[at], 1e-6)
        assert (some[0] == tokens[at]).all() and (some[2] == prob[at]).all()


def test_a_workspace_holds_fewer_rows_and_smaller_vocabularies_too():
    size = fb.sample_tokens_workspace
    for V in (1, 1000, 4096, 4097, 16384, 16385, 32003, 126464, 200000, 1 << 20, (1 << 20) + 1, 1 << 21):
        sizes = [size(n, V) for n in range(1, 140)] + [size(n, V) for n in (1000, 1024, 1025, 4096, 65535)]
        assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:])), V
    rng = np.random.default_rng(2)
    for n in (1, 2, 3, 7, 8, 9, 16, 31, 64, 65, 1000):
        vocabs = sorted({int(x) for x in np.exp(rng.uniform(0, math.log(1 << 21), 400))} | {16384 * i + j for i in range(1, 128) for j in (0, 1)})
        sizes = [size(n, V) for V in vocabs]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), n


@pytest.mark.gpu
def test_one_workspace_for_every_batch_up_to_the_largest():
    n, V = 24, 126464
    z = _logits(n, V, torch.bfloat16, 3).to(DEV)
    u = torch.rand(n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4))
    k = torch.full((n,), 40, dtype=torch.int32, device=DEV)
    guard = 4096
    size = fb.sample_tokens_workspace(n, V)
    ws = torch.full((size + guard,), 0xab, dtype=torch.uint8, device=DEV)
    want = None
    for m in (24, 16, 9, 8, 4, 1):
        out = (torch.full((m,), -7, dtype=torch.int32, device=DEV), torch.zeros(m, device=DEV), torch.zeros(m, device=DEV))
        fb.sample_tokens(z[:m], None, u[:m], None, k[:m], None, None, *out, ws[:size])
        want = out if want is None else want
        assert torch.equal(out[0], want[0][:m]) and torch.equal(out[2], want[2][:m])
        assert torch.allclose(out[1], want[1][:m], rtol=2.0 ** -19, atol=0)
    assert (ws[size:] == 0xab).all()


def test_tensors_of_more_than_one_device_are_refused(monkeypatch):
    """Without a GPU: tensors that say that they are on one, and a library that notes its calls."""
    class Claims(torch.Tensor):
        is_cuda = True
        where = 0

        def get_device(self):
            return self.where

    def on(t, where=0):
        t = t.as_subclass(Claims)
        t.where = where
        return t

    calls = []

    class Noted:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or fb.FOCUS_OK

    monkeypatch.setattr(fb, "lib", Noted)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    n, V = 3, 16
    f32, i32 = lambda: on(torch.zeros(n)), lambda: on(torch.zeros(n, dtype=torch.int32))
    args = dict(logits=on(torch.zeros((n, V), dtype=torch.bfloat16)), masked=on(torch.ones(n, dtype=torch.uint8)), uniform=f32(), temperature=f32(), top_k=i32(),
                top_p=f32(), min_p=f32(), tokens=i32(), conf=f32(), prob=f32(), workspace=on(torch.zeros(1 << 16, dtype=torch.uint8)))
    for name, t in args.items():
        with pytest.raises(ValueError):
            fb.sample_tokens(**{**args, name: on(t.clone(), 1)})
    with pytest.raises(ValueError):
        fb.sample_tokens(**{**args, "workspace": on(torch.zeros(1 << 16, dtype=torch.uint8)[::2])})
    assert calls == []
    fb.sample_tokens(**args)
    fb.sample_tokens(**{**args, "masked": None, "conf": None, "top_k": None})
    assert calls == ["focus_sample_tokens"] * 2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [3, 20000])  # (20000 logits of nearly the same share: ends that are searched for in the whole row)
def test_the_confidence_of_a_token_far_below_the_largest(V, dtype):
    """At a temperature of 100 a token 85 below the largest is drawn nearly as often: its confidence, at temperature 1, is exp(-85) of the sum, 2^-122.6."""
    for down in (40.0, 42.0, 60.0, 85.0):
        z = torch.full((2, V), -down, dtype=dtype)
        z[:, 0] = 0.0
        tokens, conf, prob = run(z, np.float32(0.75), 100.0, 0, np.array([1.0, 0.97], dtype=np.float32))
        for i, p in enumerate((1.0, float(np.float32(0.97)))):
            t, c, q = so.sample_token(z[i].double().numpy(), 0.75, 100.0, 0, p, 0.0)
            assert t > 0 and tokens[i] == t
            assert abs(conf[i] - c) <= 2.0 ** -20 * c and abs(prob[i] - q) <= 2.0 ** -20 * q
