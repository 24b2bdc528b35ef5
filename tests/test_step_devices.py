"""The objects that sequence calls refuse to enqueue them where their buffers are not."""
import pytest
import torch

from paper_2602_02159_amd.step import FocusDecoder, FocusPagedStep, FocusStep


def call_that_must_not_be_made(*args):
    raise AssertionError("called")


class Graph:
    replayed = 0

    def replay(self):
        self.replayed += 1


class Buffers:
    """What an object looks at: buffers on cuda:1."""
    device = "cuda:1"

    def get_device(self):
        return 1


def made(kind, **attributes):
    step = kind.__new__(kind)
    step.__dict__.update(attributes)
    return step


def with_calls(kind, graph):
    calls = [(call_that_must_not_be_made, ())]
    return made(kind, focus_idx=Buffers(), seq_len=Buffers(), calls={"select": calls}, entry_calls=calls, step_calls=calls, layer_calls=[calls], score_calls=calls, n_layers=1,
                _graph=graph, _g_entry=graph, _g_step=graph, _g_run=graph, _g_score=graph, sequence=lambda: calls)


KINDS = [(FocusStep, ("run",), ("select",)), (FocusDecoder, ("run_entry", "run_step"), None), (FocusPagedStep, ("run", "score"), (0,))]


@pytest.mark.parametrize("kind,runs,issued", KINDS)
def test_buffers_of_another_device_are_refused(kind, runs, issued, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for name in runs + ("capture",) + (("issue",) if issued else ()):
        with pytest.raises(ValueError, match="cuda:1, but the current device is cuda:0"):
            getattr(with_calls(kind, None), name)(*(issued if name == "issue" else ()))


@pytest.mark.parametrize("kind,runs,issued", KINDS)
def test_a_captured_graph_runs_where_it_was_captured(kind, runs, issued, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    graph = Graph()
    for name in runs:
        getattr(with_calls(kind, graph), name)()
    assert graph.replayed == len(runs)
