"""A step of many requests over pages: against the single calls bit for bit, and a request's rows against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_02159_amd import binding as fb
from paper_2602_02159_amd.step import FocusPagedStep

from test_paged import attend64, bf16_bits, check_attention, e4m3_rows, freqs, rotation, turned32, values

DEV = "cuda:0"


def fill(step, g, lens, rows=None, positions=None):
    step.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
    if rows is not None:
        step.row_start.copy_(torch.tensor([0, *np.cumsum(rows)], dtype=torch.int32))
    if positions is not None:
        step.positions.copy_(torch.tensor(positions + [-1] * (step.n_rows - len(positions)), dtype=torch.int32))
    for tensors in (step.q, step.k_new, step.v_new):
        for t in tensors:
            t.copy_(torch.randn(t.shape, generator=g).bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("quantised", [False, True])
def test_requests_come_grow_and_go(quantised):
    """Captured once, replayed while a request joins, one leaves and the lengths grow over page borders; every layer's rows against 64 bits."""
    layers, page, H, Hq, d, n_req, width = 2, 16, 2, 6, 64, 3, 5
    step = FocusPagedStep(layers, n_req * width, page, H, Hq, d, n_req, width, DEV, rotation=rotation(d), quantised=quantised, vocab=1000, top_n=4)
    step.capture()
    table = torch.randperm(n_req * width, generator=torch.Generator().manual_seed(0)).view(n_req, width).int()
    step.page_table.copy_(table)
    g = torch.Generator().manual_seed(1)
    history = [[[] for _ in range(n_req)] for _ in range(layers)]  # (k, v) rows as the pages hold them
    lens = [0, 0, 0]

    def held(x):
        if not quantised:
            return torch.from_numpy(bf16_bits(x).view(np.int16)).view(torch.bfloat16).double()
        codes, exps = e4m3_rows(x)
        return values(torch.from_numpy(codes), torch.from_numpy(exps))
    for turn in range(40):
        there = [turn < 33, turn >= 5, 10 <= turn < 20 or turn >= 30]
        for r in range(n_req):
            if not there[r] or (r == 2 and turn == 30):
                lens[r] = 0
                for l in range(layers):
                    history[l][r] = []
            lens[r] += there[r]
        fill(step, g, lens)
        step.logits.copy_(torch.randn(step.logits.shape, generator=g).bfloat16())
        step.run()
        step.score()
        torch.cuda.synchronize()
        for l in range(layers):
            for r in range(n_req):
                if lens[r] == 0:
                    assert not step.out[l][r].any() and bool((step.lse[l][r] == -np.inf).all())
                    continue
                at = np.array([lens[r] - 1])
                history[l][r].append((held(turned32(step.k_new[l][r:r + 1].float().cpu().numpy(), at, freqs(d), False))[0],
                                      held(step.v_new[l][r:r + 1].float().cpu().numpy())[0]))
                q = turned32(step.q[l][r:r + 1].float().cpu().numpy(), at, freqs(d), False)[0]
                q = torch.from_numpy(bf16_bits(q).view(np.int16)).view(torch.bfloat16).double()
                k, v = (torch.stack([x[i] for x in history[l][r]]) for i in range(2))
                for h in range(Hq):
                    ref = attend64(q[h:h + 1], k[:, h // 3], v[:, h // 3], torch.ones((1, lens[r]), dtype=torch.bool))
                    check_attention(step.out[l][r:r + 1, h].cpu(), step.lse[l][r:r + 1, h].cpu(), ref)
        z = step.logits.double().cpu()
        lp = torch.log_softmax(z, 1)
        assert torch.allclose(step.top_logprobs.double().cpu(), lp.gather(1, step.top_ids.long().cpu()), rtol=2.0 ** -18, atol=0)
        assert torch.equal(step.top_ids.long().cpu(), torch.sort(z, dim=1, descending=True, stable=True).indices[:, :4])


@pytest.mark.gpu
@pytest.mark.parametrize("quantised", [False, True])
def test_active_positions_of_a_block(quantised):
    """Scattered rows of a generation block, attention over all of it: the captured step, the eager one and the single calls agree bit for bit."""
    layers, page, H, Hq, d, n_req, width, most = 2, 32, 4, 8, 128, 4, 6, 9
    make = lambda: FocusPagedStep(layers, n_req * width, page, H, Hq, d, n_req, width, DEV, max_rows=most, n_rows=30, rotation=rotation(64), quantised=quantised,
                                  scattered=True)
    steps = [make(), make()]
    table = torch.randperm(n_req * width, generator=torch.Generator().manual_seed(2)).view(n_req, width).int()
    steps[0].capture()
    for s in steps:
        s.page_table.copy_(table)
    lens, rows = [150, 33, 192, 64], [9, 3, 0, 8]
    g = torch.Generator().manual_seed(3)
    for turn in range(3):
        picks = [torch.randperm(lens[r], generator=g)[:rows[r]].sort().values.tolist() for r in range(n_req)]
        positions = sum(picks, [])
        positions[4] = -1
        fill(steps[0], g, lens, rows, positions)
        for a, b in zip((steps[0].seq_len, steps[0].row_start, steps[0].positions, *steps[0].q, *steps[0].k_new, *steps[0].v_new),
                        (steps[1].seq_len, steps[1].row_start, steps[1].positions, *steps[1].q, *steps[1].k_new, *steps[1].v_new)):
            b.copy_(a)
        steps[0].run()
        steps[1].run()
        s = steps[1]
        for l in range(layers):
            assert torch.equal(steps[0].out[l], s.out[l]) and torch.equal(steps[0].lse[l], s.lse[l])
            assert torch.equal(steps[0].k_pages[l], s.k_pages[l]) and torch.equal(steps[0].v_pages[l], s.v_pages[l])
            turned, out, lse = torch.zeros_like(s.q[l]), torch.zeros_like(s.out[l]), torch.zeros_like(s.lse[l])
            fb.paged_append(s.caches[l], s.batch, s.k_new[l], s.v_new[l], s.rotation, s.q[l], turned)
            turned[4] = s.q_turned[4]  # (a row without a position: what the buffer held)
            fb.paged_attn(turned, s.caches[l], s.batch, False, out, lse, s.workspace)
            n, rest = sum(rows), [i for i in range(sum(rows)) if i != 4]
            assert torch.equal(out[rest], s.out[l][rest]) and torch.equal(lse[rest], s.lse[l][rest])
            assert not s.out[l][n:].any() and not s.lse[l][n:].any()


def test_sizes_are_refused():
    with pytest.raises((fb.FocusError, ValueError, RuntimeError, AssertionError, TypeError)):
        FocusPagedStep(1, 4, 16, 2, 4, 80, 2, 2, "cpu")


def test_a_rotation_of_another_device_is_refused():
    rotation = fb.Rotation(1 << 20, 64, 0, 1.0)
    rotation.device = 1
    with pytest.raises(ValueError, match="rotation on device 1"):
        FocusPagedStep(1, 4, 16, 2, 4, 64, 2, 2, "cpu", rotation=rotation)


@pytest.mark.parametrize("vocab,top_n", [(1000, 33), (1000, -1), (0, 0), ((1 << 21) + 1, 5)])
def test_scores_of_unsupported_sizes_are_refused_at_once(vocab, top_n):
    with pytest.raises(fb.FocusError, match=f"vocab={vocab}, top_n={top_n}"):
        FocusPagedStep(1, 4, 16, 2, 4, 64, 2, 2, "cpu", vocab=vocab, top_n=top_n)


@pytest.mark.gpu
@pytest.mark.parametrize("head_dim,n_q_heads,page", [(80, 4, 16), (64, 5, 16), (64, 4, 65537)])
def test_unsupported_sizes_are_refused_at_once(head_dim, n_q_heads, page):
    FocusPagedStep(1, 4, 16, 2, 4, 64, 2, 2, DEV)  # this one is not
    with pytest.raises(fb.FocusError):
        FocusPagedStep(1, 4, page, 2, n_q_heads, head_dim, 2, 2, DEV)
