"""FocusDecoder with quantised caches and drawn tokens: a block entry and steps, eagerly and replayed, against the single entry points."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2602_02159_amd import binding as fb
from paper_2602_02159_amd.step import FocusDecoder
from tests.test_quant_cache import check_attention, key_set

DEV = "cuda:0"
LAYERS, L_DENSE, TAIL, H, D, M, N, GEN, BLOCK, K, WINDOW, KEEP, SINKS, VOCAB = 5, 1, 1, 4, 128, 900, 64, 32, 64, 4, 2, 5, 6, 5003


def _fill(dec, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda t, scale=1.0: t.copy_(torch.randn(t.shape, generator=g, device=DEV) * scale)
    for l in range(LAYERS):
        for t in (dec.q_all[l], dec.k_all[l], dec.v_all[l], dec.q[l], dec.k_new[l], dec.v_new[l]):
            normal(t)
    normal(dec.logits, 3.0)
    dec.uniform.copy_(torch.rand(GEN, generator=g, device=DEV))
    dec.temperature.copy_(0.4 + torch.rand(GEN, generator=g, device=DEV))
    dec.temperature[3] = 0.0
    dec.top_k.fill_(50)
    dec.top_p.fill_(0.95)
    dec.min_p.fill_(0.01)
    dec.masked.fill_(1)
    dec.masked[5:9] = 0


def _make():
    return FocusDecoder(LAYERS, L_DENSE, TAIL, H, D, M, N, GEN, M, BLOCK, K, WINDOW, KEEP, SINKS, torch.device(DEV), VOCAB, quantised=True, sample=True)


def _buffers(dec):
    sparse = [l for l in range(LAYERS) if dec.is_sparse(l)]
    caches = [t for l in range(LAYERS) for t in (dec.k_cache[l], dec.v_cache[l], dec.k_exp[l], dec.v_exp[l]) if t is not None]
    return ([dec.tokens, dec.conf, dec.prob, dec.focus_idx, dec.active_idx, dec.counts, dec.sink_idx, dec.col_mass] + dec.out_all + dec.out + caches +
            [dec.kept[l] for l in sparse] + [dec.scores[l] for l in sparse] + [dec.kbar[l] for l in sparse])


@pytest.mark.gpu
def test_entry_and_step_are_the_single_calls():
    dec = _make()
    assert dec.quantised == [True, False, True, True, True]
    _fill(dec, 1)
    dec.run_entry()
    for l in range(LAYERS):
        k, v = dec.read_cache(l)
        assert k.dtype == torch.bfloat16
        if dec.quantised[l]:
            assert np.array_equal(k.double().cpu().numpy(), so.read_rows(*so.quantise_rows(dec.k_all[l].double().cpu().numpy())))
        else:
            assert torch.equal(k, dec.k_all[l]) and torch.equal(v, dec.v_all[l])
        want = torch.empty_like(dec.out_all[l])
        fb.refresh_attn(dec.q_all[l], dec.k_all[l], dec.v_all[l], fb.make_shape(dec.q_all[l], dec.k_all[l], dec.v_all[l], M, BLOCK, want), want, None)
        assert torch.equal(want, dec.out_all[l])
    dec.run_step()
    z, row = dec.logits.double().cpu().numpy(), lambda t, i: float(t[i])
    for i in range(GEN):
        t, c, p = (-1, 0.0, 0.0) if 5 <= i < 9 else so.sample_token(z[i], row(dec.uniform, i), row(dec.temperature, i), 50, row(dec.top_p, i), row(dec.min_p, i))
        assert int(dec.tokens[i]) == t and abs(row(dec.conf, i) - c) <= 2.0 ** -20 * c and abs(row(dec.prob, i) - p) <= 2.0 ** -20 * p
    n = int(dec.counts[1])
    active = dec.active_idx[:n].long()
    for l in range(LAYERS):
        k, v = dec.read_cache(l)
        new = dec.k_new[l][:, :n]
        if dec.quantised[l]:
            new = torch.from_numpy(so.read_rows(*so.quantise_rows(new.double().cpu().numpy()))).to(DEV).to(torch.bfloat16)
        assert torch.equal(k[:, M + active], new)
        # the bf16 attention over the same keys: each rounds its probabilities and outputs to 2^-8 of at most the largest value
        blocks, n_keep, sinks, n_sink = (dec.kept[l], KEEP, dec.sink_idx, SINKS) if dec.is_sparse(l) else (dec.all_blocks, dec.n_b, None, 0)
        want = torch.zeros_like(dec.out[l])
        s = fb.make_shape(dec.q[l], k, v, M, BLOCK, want)
        ws = torch.empty(fb.workspace_bytes(fb.FN_SPARSE_ATTN, s, dec.max_active, n_keep, n_sink), dtype=torch.uint8, device=DEV)
        fb.sparse_attn(dec.q[l], dec.active_idx, dec.counts, k, v, s, blocks, n_keep, sinks, n_sink, want, None, ws)
        assert (dec.out[l][:, :n].double() - want[:, :n].double()).abs().max() <= 4 * 2.0 ** -8 * float(v.abs().max())


@pytest.mark.gpu
def test_replayed_graphs_give_what_eager_calls_give():
    eager, graph = _make(), _make()
    _fill(eager, 2)
    _fill(graph, 2)
    graph.capture()
    for i in range(4):
        _fill(eager, 10 + i)
        _fill(graph, 10 + i)
        for dec in (eager, graph):
            if i % 2 == 0:
                dec.run_entry()
            dec.run_step()
        torch.cuda.synchronize()
        if i == 0:  # (the capture's warm run has been through both calls once)
            for dec in (eager, graph):
                dec.run_entry()
                dec.run_step()
        for a, b in zip(_buffers(eager), _buffers(graph)):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_a_steps_layers_are_the_single_calls_bit_for_bit():
    """Over the caches that the step leaves behind, with its lists: no sink, block, query or row of them may be missing.  And against the fp64
    attention over exactly those keys, whose bounds scale with what is attended."""
    dec = _make()
    _fill(dec, 5)
    dec.run_entry()
    dec.run_step()
    n, focus = int(dec.counts[1]), int(dec.counts[0])
    active, sinks = dec.active_idx[:n].cpu().numpy(), dec.sink_idx.tolist()
    assert len(set(sinks)) == SINKS and n > 1 and focus > 0
    for l in range(LAYERS):
        out, lse = torch.full_like(dec.out[l], 7.0), torch.zeros((H, dec.max_active), device=DEV)
        s = fb.make_shape(dec.q[l], dec.k_cache[l], dec.v_cache[l], M, BLOCK, out)
        if dec.is_sparse(l):
            scores, kept = torch.zeros_like(dec.scores[l]), torch.zeros_like(dec.kept[l])
            ws = torch.empty(fb.workspace_bytes(fb.FN_QUANT_LAYER, s, dec.max_active, KEEP, SINKS), dtype=torch.uint8, device=DEV)
            fb.quant_layer(dec.q[l], dec.focus_idx, dec.active_idx, dec.counts, dec.caches[l], dec.kbar[l], s, KEEP, dec.sink_idx, SINKS, scores, kept, out,
                           lse, ws)
            assert torch.equal(kept, dec.kept[l]) and torch.equal(scores, dec.scores[l])
            keys = key_set(M, N, BLOCK, kept.tolist(), sinks)
        elif dec.quantised[l]:
            ws = torch.empty(fb.workspace_bytes(fb.FN_QUANT_ATTN, s, dec.max_active, dec.n_b, 0), dtype=torch.uint8, device=DEV)
            fb.quant_attn(dec.q[l], dec.active_idx, dec.counts, dec.caches[l], s, dec.all_blocks, dec.n_b, None, 0, out, lse, ws)
            keys = np.arange(M + N)
        else:
            mass, found = torch.zeros_like(dec.col_mass), torch.zeros_like(dec.sink_idx)
            ws = torch.empty(fb.workspace_bytes(fb.FN_PROBE_LAYER, s, dec.max_active, 0, SINKS), dtype=torch.uint8, device=DEV)
            fb.probe_layer(dec.q[l], dec.active_idx, dec.counts, dec.k_cache[l], dec.v_cache[l], s, SINKS, out, lse, mass, found, ws)
            assert torch.equal(mass, dec.col_mass) and torch.equal(found, dec.sink_idx)
            keys = np.arange(M + N)
        assert torch.equal(out[:, :n], dec.out[l][:, :n]), l
        k, v = dec.read_cache(l)
        check_attention(dec.out[l], lse, dec.q[l], k, v, active, keys)


def test_options_that_do_not_go_together():
    with pytest.raises(AssertionError):
        FocusDecoder(2, 0, 0, 1, 64, 64, 8, 8, 64, 64, 2, 0, 1, 1, torch.device("cpu"), None, sample=True)
