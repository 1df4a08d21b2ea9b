"""What the example of cached feed-forward sub-blocks times: a computed step with its cache steps."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.mark.gpu
def test_a_computed_step_is_timed_with_its_cache_steps(monkeypatch):
    import cached_feed_forward as example
    log = []

    class Event(torch.cuda.Event):
        def record(self, *a):
            log.append("mark")
            return super().record(*a)

    def counted(name):
        call = getattr(example.svdc, name)

        def wrapper(*a, **kw):
            log.append(name)
            return call(*a, **kw)
        monkeypatch.setattr(example.svdc, name, wrapper)

    monkeypatch.setattr(torch.cuda, "Event", Event)
    for name in ("svdcache_full_step", "svdcache_forecast_combine", "svdcache_matmul8"):
        counted(name)
    example.run(tokens=256, hidden=256, blocks=2, rank=16, steps=5, interval=4, say=lambda s: None)
    timed, marks = [], [i for i, name in enumerate(log) if name == "mark"]
    for begin, end in zip(marks[::2], marks[1::2]):
        timed.append(log[begin + 1:end])
    assert [step.count("svdcache_full_step") for step in timed] == [2, 0, 0, 0, 2]
    assert [step.count("svdcache_matmul8") for step in timed] == [4, 0, 0, 0, 4]
    assert [step.count("svdcache_forecast_combine") for step in timed] == [0, 2, 2, 2, 0]
    assert log.count("svdcache_full_step") == 4          # each computed output enters its state once
