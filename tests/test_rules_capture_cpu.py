"""Recording a step with marks: whose weights the run ahead of the recording adds to (no GPU needed: the recording is left out)."""
import pytest
import torch

from paper_2510_21270_amd import binding as b
from test_serving_capture_cpu import recording             # noqa: F401 (the fixture)


def _step(monkeypatch, weights=True):
    monkeypatch.setattr(b, "_same_device", lambda *a: None)
    s = b.DecodeStep.__new__(b.DecodeStep)
    s.cache = b.Cache.__new__(b.Cache)
    s.cache.K, s.cache.dev, s.O = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), 0, torch.zeros(1)
    position = torch.zeros(3, 2, 16, dtype=torch.int32)
    s.marks = b.CacheMarks(s.cache, torch.ones(3, 2, 16) if weights else None, position)
    return s


def test_the_run_ahead_of_a_recording_weighs_for_nobody(recording, monkeypatch):     # noqa: F811
    s, seen = _step(monkeypatch), []
    marks = s.marks

    def run(*a):
        seen.append(s.marks)
        s.marks.weight.add_(5.0)

    monkeypatch.setattr(s, "run", run)
    s.capture()
    first, recorded = seen
    assert recorded is marks and s.marks is marks and bool((marks.weight == 6.0).all())        # (this stand-in records nothing: it adds)
    assert first.weight.data_ptr() != marks.weight.data_ptr() and first.weight.shape == marks.weight.shape
    assert first.position is marks.position and first.cache is s.cache


def test_a_recording_that_fails_leaves_marks_and_weights(recording, monkeypatch):    # noqa: F811
    s = _step(monkeypatch)
    marks = s.marks

    def run(*a):
        s.marks.weight.add_(5.0)
        raise b.PbsError("refused")

    monkeypatch.setattr(s, "run", run)
    with pytest.raises(b.PbsError, match="refused"):
        s.capture()
    assert s.marks is marks and bool((marks.weight == 1.0).all())


def test_marks_without_weights_are_used_as_they_are(recording, monkeypatch):         # noqa: F811
    s, seen = _step(monkeypatch, weights=False), []
    monkeypatch.setattr(s, "run", lambda *a: seen.append(s.marks))
    s.capture()
    assert seen == [s.marks, s.marks]
