"""The handles of perf/operators.py: one for every device and stream that inputs are prepared on (no GPU: handles and streams are stand-ins)."""
import importlib.util
import os
import types

import pytest
import torch

from paper_2112_09335_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def cases(monkeypatch):
    spec = importlib.util.spec_from_file_location("operator_cases", os.path.join(ROOT, "perf", "operators.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    made = []

    class Handle:
        def __init__(self, *args, stream=0, device=0, **kw):
            self.place, self.calls = (device, stream), 0
            made.append(self)

        def grouped_product(self, *args, **kw):
            self.calls += 1
    now = types.SimpleNamespace(device=0, stream=0)
    monkeypatch.setattr(binding, "GcnAdmm", Handle)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now.device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=now.stream))
    module.own = True
    t = torch.zeros(4, 4)
    case = dict(path="product", type="f32", out="f32", groups=1, rows=4, k=4, n=4)
    monkeypatch.setattr(module, "_inputs", lambda case, seed: dict(case=case, held=4, offsets=t, x=t, w=t, out=t), raising=False)
    return types.SimpleNamespace(prepare=lambda: module.prepare(case, 0), run=module.run, made=made, now=now)


def test_a_state_keeps_the_handle_of_the_stream_it_was_prepared_on(cases):
    states = []
    for device, stream in ((0, 0), (0, 0), (0, 7), (1, 7)):
        cases.now.device, cases.now.stream = device, stream
        states.append(cases.prepare())
    for i, place in ((1, (0, 0)), (3, (1, 7)), (2, (0, 7)), (0, (0, 0))):
        before = {h.place: h.calls for h in cases.made}
        cases.run(states[i])
        assert {h.place: h.calls - before[h.place] for h in cases.made} == {**dict.fromkeys(before, 0), place: 1}
    assert [h.place for h in cases.made] == [(0, 0), (0, 7), (1, 7)]      # one each
