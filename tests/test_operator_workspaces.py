"""The scratch memory of the calls in perf/operators.py: one for each stream."""
import pytest
import torch

import perf.operators as operators
from paper_2409_11600_amd import binding as B


def test_each_stream_has_its_own(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(operators, "_WORKSPACES", {})
    made = {}
    for stream in (0, 71, 0, 72, 71):
        monkeypatch.setattr(B, "_stream", lambda: stream)
        assert made.setdefault(stream, operators._workspace()) is operators._workspace()
    assert len({id(ws) for ws in made.values()}) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("case", [{"call": "glr_fwd", "dtype": "bf16", "T": 4000, "N": 20, "H": 40, "ragged": True}, {"call": "glr_bwd", "dtype": "f32", "T": 2100, "N": 3, "H": 24, "ragged": True},
                                  {"call": "ln_bwd", "dtype": "bf16", "rows": 4000, "C": 768, "residual": True}])
def test_calls_beside_each_other(monkeypatch, case):
    """Two streams at once, each with inputs of its own, against the same calls one after the other, bit by bit."""
    monkeypatch.setattr(operators, "own", True)
    states = [operators.prepare(case, seed) for seed in (1, 2)]
    want = [operators.run(s) for s in states]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in states], []
    for _ in range(8):
        for stream, state in zip(streams, states):
            with torch.cuda.stream(stream):
                got.append(operators.run(state))
    torch.cuda.synchronize()
    for k, g in enumerate(got):
        assert all(torch.equal(g[name], want[k % 2][name]) for name in g), k
