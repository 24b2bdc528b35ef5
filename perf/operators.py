"""Operators of a decoding step on a quantised cache, for timing them through the public entry points and for comparing them.

  write   new K / V states into a cache of eight-bit values: the rows of a step's active positions, or all rows with the block means
  read    a range of rows of that cache back as bfloat16
  attn    attention of the active queries over kept blocks, sinks and response rows of that cache
  layer   a sparse layer over that cache: relevance of the blocks, their choice, attention
  sample  tokens and confidences from vocabulary logits: temperature, top-k, top-p, min-p, given random numbers

A cache row of one head is d e4m3 codes and one power of two: the smallest 2^E, -110 <= E <= 119, with which the largest finite
absolute value is at most 448.  A code c stands for c * 2^E; the byte that is stored is E + 127.

`own` False: elementary torch operations; True: the framework's entry points.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E_MIN, E_MAX, CODE_MAX = -110, 119, 448.0
VOCAB = 126464


def _case(path, **more):
    return dict(path=path, **more)


def _attn(path, heads, head_dim, ctx, resp, block, gen, active, slots, keep, sinks, focus=0):
    return _case(path, heads=heads, head_dim=head_dim, ctx=ctx, resp=resp, block=block, gen=gen, active=active, slots=slots,
                 keep=keep, sinks=sinks, focus=focus)


def listed():
    named = lambda name, case: dict(case, name=name)
    return [
        # a step's eight active rows into the smallest cache: the launch is all there is
        named("write-rows-4x64", _case("write", heads=4, head_dim=64, ctx=1024, resp=32, block=64, rows=8)),
        # a block entry: every row of the longest ordinary prompt, with the block means of the same pass
        named("write-all-32k", _case("write", heads=32, head_dim=128, ctx=32768, resp=64, block=128, rows=0)),
        # a few rows of a small cache back, from a row and in a number that divide nothing
        named("read-999-d64", _case("read", heads=4, head_dim=64, ctx=1024, resp=32, block=64, first=33, rows=999)),
        # the whole cache of a 32K layer back, as a layer that needs bfloat16 rows takes it
        named("read-all-32k", _case("read", heads=32, head_dim=128, ctx=32768, resp=64, block=128, first=0, rows=32832)),
        # one query over every row of a short prompt
        named("attn-1k-one-query", _attn("attn", 4, 64, 1024, 32, 64, 32, 1, 1, 16, 0)),
        # a dense layer of the 32K stack: sixteen queries over every row
        named("attn-32k-dense", _attn("attn", 32, 128, 32768, 64, 128, 64, 16, 16, 256, 0)),
        # half of the 64-row blocks, one sink per hundred positions, window-expanded queries, a padded list
        named("attn-32k-half", _attn("attn", 32, 128, 32768, 256, 64, 32, 25, 32, 256, 327)),
        # the headline sparse layer: seven of 256 blocks, four sinks
        named("layer-32k", _attn("layer", 32, 128, 32768, 64, 128, 64, 16, 16, 7, 4, 16)),
        # grouped-query attention in the row view: seven query heads on each of four K/V heads, a ragged prompt
        named("layer-16k-grouped", _attn("layer", 4, 128, 15937, 255, 64, 224, 175, 224, 125, 159, 28)),
        # one position of one sequence, everything filtered
        named("sample-one", _case("sample", rows=1, vocab=VOCAB, wide=False, filters="all", masked=False)),
        # the positions of a generation block, a quarter of them decided already
        named("sample-64", _case("sample", rows=64, vocab=VOCAB, wide=False, filters="all", masked=True)),
        # a batch of sequences with float32 logits of a vocabulary that divides nothing, nucleus only
        named("sample-511-wide", _case("sample", rows=511, vocab=32003, wide=True, filters="nucleus", masked=False)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Prompts of 100 to 32768 rows, one query to 256, vocabularies of 1000 to 200000 and one row to 512."""
    path = rng.choice(("write", "read", "attn", "attn", "layer", "layer", "sample", "sample"))
    if path == "sample":
        vocab = _log_int(rng, 1000, 200000)
        rows = min(_log_int(rng, 1, 512), max(1, 16_000_000 // vocab))
        return _case("sample", rows=rows, vocab=vocab, wide=rng.random() < 0.4, filters=rng.choice(("all", "nucleus", "none")),
                     masked=rng.random() < 0.3)
    heads, head_dim = rng.choice((1, 4, 8, 28, 32)), rng.choice((64, 128, 128))
    ctx, resp, block = _log_int(rng, 100, 32768), rng.randint(0, 256), rng.choice((32, 64, 100, 128))
    if path == "write":
        rows = 0 if rng.random() < 0.4 else min(ctx, rng.randint(1, 64))
        return _case("write", heads=heads, head_dim=head_dim, ctx=ctx, resp=resp, block=block, rows=rows)
    if path == "read":
        first = rng.randint(0, ctx - 1)
        return _case("read", heads=heads, head_dim=head_dim, ctx=ctx, resp=resp, block=block, first=first,
                     rows=rng.randint(1, ctx + resp - first))
    n_b = -(-ctx // block)
    slots = _log_int(rng, 1, 256)
    keep = max(1, min(n_b, int(n_b * math.exp(rng.uniform(math.log(0.03), 0.0)))))
    sinks = min(ctx, rng.choice((0, 2, 4, 16, max(2, ctx // 100))))
    gen = slots + rng.randint(0, 40)
    return _attn(path, heads, head_dim, ctx, resp, block, gen, rng.randint(max(1, slots - 8), slots), slots, keep, sinks,
                 rng.randint(1, min(gen, 28)) if path == "layer" else 0)


# ---- inputs ------------------------------------------------------------------------------------------------------------
def quantised(x):
    """bfloat16 rows [..., d] -> (codes as float8, exponent bytes)."""
    magnitude = x.view(torch.int16).to(torch.int32) & 0x7fff
    finite = magnitude < 0x7f80
    largest = torch.where(finite, magnitude, 0).amax(-1)
    e = (((largest + 0x1f) >> 7) - 127 - 8).clamp(E_MIN, E_MAX)  # 1.75 * 2^8 = 448
    y = torch.ldexp(x.float(), -e[..., None]).clamp(-CODE_MAX, CODE_MAX)
    y = torch.where(finite, y, math.nan)
    return y.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    pick = lambda n, of: torch.randperm(of, generator=g, device="cuda")[:n].sort().values.int()
    if case["path"] == "sample":
        return _prepare_sample(case, g, uniform)
    H, d, M, N = case["heads"], case["head_dim"], case["ctx"], case["resp"]
    L = M + N
    n_b = -(-M // case["block"])
    s = {"case": case}
    k, v = normal(H, L, d), normal(H, L, d)
    k[:, :, :2] *= 6.0  # two channels of larger values, as keys have them
    u = torch.randn(d, generator=g, device="cuda")
    u /= torch.linalg.vector_norm(u)
    pull = math.sqrt(3.0 * math.sqrt(d))
    k[:, torch.randint(0, M, (4,), generator=g, device="cuda")] += (4.0 * pull * u).to(k.dtype)  # a few keys that every query attends to
    if case["path"] == "write":
        rows = case["rows"] or L
        s["k_new"], s["v_new"] = k[:, :rows].contiguous(), v[:, :rows].contiguous()
        s["k"], s["v"] = (torch.zeros((H, L, d), dtype=torch.uint8, device="cuda") for _ in range(2))
        s["k_exp"], s["v_exp"] = (torch.zeros((H, L), dtype=torch.uint8, device="cuda") for _ in range(2))
        if case["rows"]:
            s["active"] = pick(rows, min(L, 2 * rows))
        else:
            s["kbar"] = torch.zeros((H, n_b, d), device="cuda")
        return s
    (kq, s["k_exp"]), (vq, s["v_exp"]) = quantised(k), quantised(v)
    s["k"], s["v"] = kq.view(torch.uint8), vq.view(torch.uint8)
    del k, v
    if case["path"] == "read":
        s["k_out"], s["v_out"] = (torch.zeros((H, case["rows"], d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return s
    s["q"] = normal(H, case["gen"], d) + (0.5 * pull * u).to(torch.bfloat16)
    s["active"] = torch.full((case["slots"],), -1, dtype=torch.int32, device="cuda")
    s["active"][:case["active"]] = pick(case["active"], case["gen"])
    s["counts"] = torch.tensor([case["focus"], case["active"]], dtype=torch.int32, device="cuda")
    s["sinks"] = pick(case["sinks"], M)
    s["out"] = torch.zeros((H, case["slots"], d), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((H, case["slots"]), device="cuda")
    if case["path"] == "attn":
        s["kept"] = pick(case["keep"], n_b)
        return s
    s["kept"] = torch.full((case["keep"],), -1, dtype=torch.int32, device="cuda")
    s["focus"] = pick(case["focus"], case["gen"])
    s["scores"] = torch.zeros(n_b, device="cuda")
    s["kbar"] = torch.stack([_means(_values(s["k"][h, :M], s["k_exp"][h, :M]), case["block"]) for h in range(H)])
    return s


def _prepare_sample(case, g, uniform):
    n, V = case["rows"], case["vocab"]
    t = torch.randn((n, V), generator=g, device="cuda").mul_(3.0)
    peaks = torch.randint(0, V, (n, 6), generator=g, device="cuda")  # a handful of likely tokens, sharper in some rows than in others
    t.scatter_add_(1, peaks, 6.0 + 12.0 * uniform(n, 1) + 2.0 * uniform(n, 6))
    t[:, V - V // 100:] = -math.inf  # ids that the vocabulary does not use
    stride = V if case["wide"] else -(-V // 8) * 8
    stride = -(-stride // 4) * 4
    logits = torch.zeros((n, stride), dtype=torch.float32 if case["wide"] else torch.bfloat16, device="cuda")[:, :V]
    logits.copy_(t)
    s = {"case": case, "logits": logits, "uniform": uniform(n), "masked": None}
    if case["masked"]:
        s["masked"] = torch.ones(n, dtype=torch.uint8, device="cuda")
        s["masked"][torch.randperm(n, generator=g, device="cuda")[:n // 4]] = 0
    some = lambda share: uniform(n) < share
    s["temperature"] = torch.where(some(0.1), 0.0, 0.3 + 1.2 * uniform(n))
    s["top_p"] = None if case["filters"] == "none" else torch.where(some(0.1), 1.0, 0.3 + 0.69 * uniform(n))
    s["top_k"] = s["min_p"] = None
    if case["filters"] == "all":
        s["top_k"] = torch.where(some(0.2), 0, torch.exp(uniform(n) * math.log(min(V, 2000))).int()).int()
        s["min_p"] = torch.where(some(0.3), 0.0, 0.2 * uniform(n))
    for name, dtype in (("tokens", torch.int32), ("conf", torch.float32), ("prob", torch.float32)):
        s[name] = torch.zeros(n, dtype=dtype, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(s):
    path = s["case"]["path"]
    if own:
        _call(s)
    elif path == "write":
        _write(s)
    elif path == "read":
        _read(s)
    elif path == "sample":
        _sample(s)
    else:
        if path == "layer":
            _choose(s)
        _attend(s)
    if path == "write":  # the codes as the values that they are; the cache is the state's own
        r = {"k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn), "k_exp": s["k_exp"], "v_exp": s["v_exp"]}
        return dict(r, kbar=s["kbar"]) if "kbar" in s else r
    names = {"read": ("k_out", "v_out"), "attn": ("out", "lse"), "layer": ("kept", "scores", "out", "lse"),
             "sample": ("tokens", "conf", "prob")}[path]
    return {name: s[name] for name in names}


def _call(s):
    from paper_2602_02159_amd import binding as fb
    c = s["case"]
    if "plan" not in s:
        s["plan"] = _plan(s, c, fb)
    cache, shape, ws = s["plan"]
    if c["path"] == "write" and c["rows"]:
        fb.quant_update(cache, shape, s["k_new"], s["v_new"], s["active"], None, 0)
    elif c["path"] == "write":
        fb.quant_refresh(cache, shape, s["k_new"], s["v_new"], s["kbar"])
    elif c["path"] == "read":
        fb.quant_read(cache, shape, c["first"], s["k_out"], s["v_out"])
    elif c["path"] == "attn":
        fb.quant_attn(s["q"], s["active"], s["counts"], cache, shape, s["kept"], c["keep"], s["sinks"], c["sinks"], s["out"], s["lse"], ws)
    elif c["path"] == "layer":
        fb.quant_layer(s["q"], s["focus"], s["active"], s["counts"], cache, s["kbar"], shape, c["keep"], s["sinks"], c["sinks"],
                       s["scores"], s["kept"], s["out"], s["lse"], ws)
    else:
        fb.sample_tokens(s["logits"], s["masked"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["tokens"],
                         s["conf"], s["prob"], ws)


def _plan(s, c, fb):
    """What a program makes once for its buffers: the descriptions of cache and shape, the workspace."""
    space = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    if c["path"] == "sample":
        return None, None, space(fb.sample_tokens_workspace(c["rows"], c["vocab"]))
    cache = fb.make_quant_cache(s["k"], s["v"], s["k_exp"], s["v_exp"])
    rows = s["q"] if "q" in s else s["k_new"] if "k_new" in s else s["k_out"]
    shape = fb.make_shape(rows, s["k"], s["v"], c["ctx"], c["block"], s.get("out"))
    if "q" not in s:
        return cache, shape, None
    fn = fb.FN_QUANT_ATTN if c["path"] == "attn" else fb.FN_QUANT_LAYER
    return cache, shape, space(fb.workspace_bytes(fn, shape, c["slots"], c["keep"], c["sinks"]))


# ---- the plain forms: 32 bits, one rounding at the end ----------------------------------------------------------------------
def _values(codes, exps):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), exps[..., None].int() - 127)


def _means(k, block):
    """Means over blocks of rows [..., M, d], the last one over what it has."""
    M = k.shape[-2]
    whole = M // block * block
    parts = [k[..., :whole, :].unflatten(-2, (M // block, block)).mean(-2)] if whole else []
    return torch.cat(parts + ([k[..., whole:, :].mean(-2, keepdim=True)] if whole < M else []), -2)


def _write(s):
    c = s["case"]
    (kq, ke), (vq, ve) = quantised(s["k_new"]), quantised(s["v_new"])
    if c["rows"]:
        at = s["active"].long()
        s["k"][:, at], s["v"][:, at] = kq.view(torch.uint8), vq.view(torch.uint8)
        s["k_exp"][:, at], s["v_exp"][:, at] = ke, ve
        return
    for name, t in (("k", kq.view(torch.uint8)), ("v", vq.view(torch.uint8)), ("k_exp", ke), ("v_exp", ve)):
        s[name].copy_(t)
    s["kbar"].copy_(_means(_values(s["k"][:, :c["ctx"]], s["k_exp"][:, :c["ctx"]]), c["block"]))


def _read(s):
    c = s["case"]
    rows = slice(c["first"], c["first"] + c["rows"])
    s["k_out"].copy_(_values(s["k"][:, rows], s["k_exp"][:, rows]))
    s["v_out"].copy_(_values(s["v"][:, rows], s["v_exp"][:, rows]))


def _choose(s):
    q = s["q"][:, s["focus"].long()].float().mean(1)
    s["scores"].copy_((q[:, None] * s["kbar"]).sum(-1).mean(0))
    s["kept"].copy_(torch.sort(s["scores"], descending=True, stable=True).indices[:s["case"]["keep"]].sort().values)


def _attend(s):
    c = s["case"]
    M, B, n_act = c["ctx"], c["block"], c["active"]
    kept, sinks = s["kept"].long(), s["sinks"].long()
    at = (kept[:, None] * B + torch.arange(B, device="cuda")).flatten()
    alone = ~(sinks[:, None] // B == kept).any(1)
    at = torch.cat((at, sinks, M + torch.arange(c["resp"], device="cuda")))
    valid = torch.ones_like(at, dtype=torch.bool)
    valid[:kept.numel() * B] = at[:kept.numel() * B] < M
    valid[kept.numel() * B:kept.numel() * B + sinks.numel()] = alone
    at = torch.where(valid, at, kept[0] * B)
    q = s["q"][:, s["active"][:n_act].long()].float()
    logits = torch.matmul(q, _values(s["k"][:, at], s["k_exp"][:, at]).transpose(1, 2).contiguous()) / math.sqrt(c["head_dim"])
    logits = torch.where(valid, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    s["out"][:, :n_act] = (torch.matmul(p, _values(s["v"][:, at], s["v_exp"][:, at])) / total).to(torch.bfloat16)
    s["lse"][:, :n_act] = (top + torch.log(total)).squeeze(-1)


def _sample(s):
    z = s["logits"].double()  # the token is the one whose share of the mass a random number falls into: borders
    V = z.shape[1]
    temperature = s["temperature"].double()[:, None]
    greedy = temperature <= 0
    top = z.amax(1, keepdim=True)
    w = torch.exp((z - top) / torch.where(greedy, 1.0, temperature))
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    rank = torch.arange(V, device="cuda")
    ws = w.gather(1, order)
    keep = torch.where(greedy, rank < 1, rank < V)
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep &= (k <= 0) | (rank < k)
    ws = torch.where(keep, ws, 0.0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        before = ws.cumsum(1) - ws
        keep &= (p >= 1) | (before < p * ws.sum(1, keepdim=True)) | (rank < 1)
    if s["min_p"] is not None:
        keep &= (ws >= s["min_p"].double()[:, None]) | (rank < 1)
    w = torch.zeros_like(z).scatter_(1, order, torch.where(keep, ws, 0.0))
    cum = w.cumsum(1)
    last = torch.where(w > 0, rank, 0).amax(1)
    token = torch.minimum((cum <= s["uniform"].double()[:, None] * cum[:, -1:]).sum(1), last)[:, None]
    prob = w.gather(1, token) / cum[:, -1:]
    conf = torch.exp(z.gather(1, token) - top) / torch.exp(z - top).sum(1, keepdim=True)
    here = torch.ones_like(token, dtype=torch.bool) if s["masked"] is None else s["masked"][:, None] != 0
    s["tokens"].copy_(torch.where(here, token, -1)[:, 0])
    s["conf"].copy_(torch.where(here, conf, 0.0)[:, 0])
    s["prob"].copy_(torch.where(here, prob, 0.0)[:, 0])


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------------
def _to_grid(x, e):
    """x / 2^e on the e4m3 grid: steps of 2^-3 of the binade, binades from 2^-6 on, half a step to the even one."""
    y = np.clip(np.ldexp(x, -e), -CODE_MAX, CODE_MAX)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -20))), -6.0) - 3.0)
    return np.rint(y / step) * step


def _exact_rows(x):
    a = np.abs(x).max(-1, keepdims=True)
    e = np.full(a.shape, E_MIN)
    m, b = np.frexp(a)  # a = m * 2^b, 0.5 <= m < 1
    e = np.where(a > 0, np.clip(np.where(m <= 0.875, b - 9, b - 8), E_MIN, E_MAX), e)
    return _to_grid(x, e), e


def exact(case, seed):
    s = prepare(case, seed)
    host = lambda t: t.double().cpu().numpy()
    code = lambda t: host(t.view(torch.float8_e4m3fn).float())
    if case["path"] == "sample":
        return _exact_sample(s)
    if case["path"] == "write":
        if s["k_new"].numel() > 20_000_000:
            return None
        kq, ke = _exact_rows(host(s["k_new"]))
        vq, _ = _exact_rows(host(s["v_new"]))
        if case["rows"]:
            k, v = np.zeros(s["k"].shape), np.zeros(s["v"].shape)
            at = s["active"].cpu().numpy()
            k[:, at], v[:, at] = kq, vq
            return {"k": k, "v": v, "k_exp": None, "v_exp": None}
        k = np.ldexp(kq, ke)
        means = [k[:, b:min(b + case["block"], case["ctx"])].mean(1) for b in range(0, case["ctx"], case["block"])]
        return {"k": kq, "v": vq, "k_exp": None, "v_exp": None, "kbar": np.stack(means, 1)}
    if case["path"] == "read":
        if s["k_out"].numel() > 20_000_000:
            return None
        rows = slice(case["first"], case["first"] + case["rows"])
        full = lambda t, e: np.ldexp(code(t[:, rows].contiguous()), e[:, rows].cpu().numpy().astype(np.int64)[..., None] - 127)
        return {"k_out": full(s["k"], s["k_exp"]), "v_out": full(s["v"], s["v_exp"])}
    M, n_act, H = case["ctx"], case["active"], case["heads"]
    scores, kept = None, s["kept"].cpu().numpy()
    if case["path"] == "layer":
        q = host(s["q"][:, s["focus"].long()]).mean(1)
        scores = np.einsum("hd,hbd->b", q, host(s["kbar"])) / H
        kept = np.sort(np.argsort(-scores, kind="stable")[:case["keep"]])
    attended = np.zeros(M + case["resp"], dtype=bool)
    for b in kept:
        attended[b * case["block"]:min((b + 1) * case["block"], M)] = True
    attended[s["sinks"].cpu().numpy()] = True
    attended[M:] = True
    at = torch.from_numpy(np.flatnonzero(attended)).cuda()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for h in range(H):
        value = lambda t, e: t[h, at].contiguous().view(torch.float8_e4m3fn).double() * torch.exp2(e[h, at].double() - 127)[:, None]
        x = s["q"][h, s["active"][:n_act].long()].double() @ value(s["k"], s["k_exp"]).T.contiguous() / math.sqrt(case["head_dim"])
        lse[h, :n_act] = torch.logsumexp(x, 1)
        out[h, :n_act] = torch.exp(x - lse[h, :n_act, None]) @ value(s["v"], s["v_exp"])
    r = {"out": out, "lse": lse}
    return r if scores is None else dict(r, kept=None, scores=scores)


def _exact_sample(s):
    n, V = s["logits"].shape
    conf, prob = np.zeros(n), np.zeros(n)
    number = lambda name, i, off: off if s[name] is None else float(s[name][i])
    z_all = s["logits"].double().cpu().numpy()
    for i in range(n):
        if s["masked"] is not None and not int(s["masked"][i]):
            continue
        z = z_all[i] - z_all[i].max()
        T = number("temperature", i, 1.0)
        order = np.lexsort((np.arange(V), -z))
        if T <= 0:
            token, kept, share = order[0], order[:1], np.ones(1)
        else:
            k = int(number("top_k", i, 0))
            kept = order[:k] if k > 0 else order
            share = np.exp(z[kept] / T)
            p = number("top_p", i, 1.0)
            if p < 1:
                m = max(1, int(np.searchsorted(np.cumsum(share), p * share.sum())) + 1)
                kept, share = kept[:m], share[:m]
            m = max(1, int((share >= number("min_p", i, 0.0)).sum()))
            kept = np.sort(kept[:m])
            share = np.exp(z[kept] / T)
            cum = np.cumsum(share)
            token = kept[min(int(np.searchsorted(cum, number("uniform", i, 0.0) * cum[-1], side="right")), len(kept) - 1)]
        prob[i] = 1.0 if T <= 0 else math.exp(z[token] / T) / share.sum()
        conf[i] = math.exp(z[token]) / np.exp(z).sum()
    return {"tokens": None, "conf": conf, "prob": prob}


# ---- bytes and operations that a pass cannot do without --------------------------------------------------------------------
def work(case):
    if case["path"] == "sample":
        rows = case["rows"] - (case["rows"] // 4 if case["masked"] else 0)
        return {"bytes": rows * case["vocab"] * (4 if case["wide"] else 2) + rows * 32, "flops": 2.0 * rows * case["vocab"]}
    H, d, M, N = case["heads"], case["head_dim"], case["ctx"], case["resp"]
    n_b = -(-M // case["block"])
    if case["path"] in ("write", "read"):
        rows = case["rows"] or M + N
        means = 4 * H * n_b * d if case["path"] == "write" and not case["rows"] else 0
        return {"bytes": 2 * H * rows * (2 * d + d + 1) + means, "flops": 4.0 * H * rows * d}
    inside = min(M, case["keep"] * case["block"])
    keys = inside + N + case["sinks"] * (1.0 - inside / M)
    bytes_ = 2 * keys * H * (d + 1) + case["active"] * H * (4 * d + 4)
    flops = 4.0 * case["active"] * keys * H * d
    if case["path"] == "layer":
        bytes_ += 4 * H * n_b * d + 2 * case["focus"] * H * d + 4 * n_b
        flops += 2.0 * H * n_b * d
    return {"bytes": bytes_, "flops": flops}
