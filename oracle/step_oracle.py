"""fp64 reference of the quantised KV cache and of the token sampling, from their definitions: numpy, no blocking, no fusion.
Test infrastructure only."""
from __future__ import annotations

import numpy as np

CODE_MAX = 448.0
E_MIN, E_MAX = -110, 119


def e4m3_values() -> np.ndarray:
    """What the 256 codes stand for: sign, four bits of exponent (bias 7, 0 = subnormal), three of mantissa; 0x7f and 0xff are NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7), m / 8.0 * 2.0 ** -6)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def nearest_code(y: np.ndarray) -> np.ndarray:
    """Code of the e4m3 number nearest to y, the one with the even mantissa on a tie; past the largest the largest; NaN: 0x7f."""
    positive = e4m3_values()[:127]
    a = np.minimum(np.abs(y), CODE_MAX)
    a = np.where(np.isnan(a), 0.0, a)
    up = np.searchsorted(positive, a)  # positive[up - 1] < a <= positive[up]
    down = np.maximum(up - 1, 0)
    to_up, to_down = positive[up] - a, a - positive[down]
    code = np.where((to_up < to_down) | ((to_up == to_down) & (up % 2 == 0)), up, down)
    code = code | np.where(np.signbit(y), 128, 0)
    return np.where(np.isnan(y), 0x7f, code).astype(np.uint8)


def row_exponents(x: np.ndarray) -> np.ndarray:
    """Smallest E in [E_MIN, E_MAX] with max of the finite |x| <= 448 * 2^E; rows along the last axis."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(a.shape, E_MIN)
    for cand in range(E_MIN, E_MAX):
        e = np.where(a > CODE_MAX * 2.0 ** cand, cand + 1, e)
    return e


def quantise_rows(x: np.ndarray):
    """x [..., d] -> (codes uint8 [..., d], exponent bytes uint8 [...])."""
    x = np.asarray(x, dtype=np.float64)
    e = row_exponents(x)
    y = np.where(np.isfinite(x), x, np.nan) * 2.0 ** -e[..., None].astype(np.float64)
    return nearest_code(y), (e + 127).astype(np.uint8)


def read_rows(codes: np.ndarray, exps: np.ndarray) -> np.ndarray:
    return e4m3_values()[codes] * np.where(exps > 0, 2.0 ** (exps.astype(np.float64) - 127), 0.0)[..., None]


def kept_tokens(z: np.ndarray, temperature: float, top_k: int, top_p: float, min_p: float) -> np.ndarray:
    """Ids (ascending) that a token may be drawn from, one row of logits.

    Order: larger logit first, then the lower id; -inf and NaN have no probability, +inf counts as the largest finite float32.
    top_k: the first top_k of the order (<= 0: all).  top_p: of those the shortest prefix whose mass is at least top_p of theirs (>= 1:
    all).  min_p: of those the ones with at least min_p times the largest probability.  The first of the order always stays.
    temperature <= 0 or NaN: only the first.  A NaN among the others switches that one off."""
    z = clean_logits(z)
    order = np.lexsort((np.arange(z.size), -z))
    order = order[z[order] > -np.inf]
    if order.size == 0:
        return order
    if not temperature > 0:
        return order[:1]
    w = np.exp((z[order] - z[order[0]]) / temperature)
    n = order.size
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        before = np.cumsum(w[:n]) - w[:n]
        n = max(1, int((before < top_p * w[:n].sum()).sum()))
    if min_p > 0:
        n = max(1, int((w[:n] >= min_p).sum()))
    return np.sort(order[:n])


def clean_logits(z: np.ndarray) -> np.ndarray:
    z = np.asarray(z, dtype=np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    return np.minimum(z, float(np.finfo(np.float32).max))


def sample_token(z, u: float, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
    """(token, conf, prob): the first kept id whose cumulative mass (ids ascending) exceeds u times the kept mass; conf is its softmax
    probability over the whole row at temperature 1, prob that among the kept ones at the given temperature.  No finite logit: (-1, 0, 0)."""
    z = clean_logits(z)
    kept = kept_tokens(z, temperature, top_k, top_p, min_p)
    if kept.size == 0:
        return -1, 0.0, 0.0
    top = z.max()
    w = np.exp((z[kept] - top) / temperature) if temperature > 0 else np.ones(1)
    cum = np.cumsum(w)
    i = min(int((cum <= u * cum[-1]).sum()), int(np.flatnonzero(w > 0)[-1]))
    e = np.exp(z - top)
    return int(kept[i]), float(e[kept[i]] / e.sum()), float(w[i] / cum[-1])
