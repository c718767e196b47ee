"""Marks that the pipeline cannot set are refused before it writes a row or starts a kernel (no GPU needed)."""
import pytest
import torch

from paper_2510_21270_amd import binding as b


@pytest.fixture
def path(monkeypatch):
    """A pipeline on the CPU whose calls only say that they have been made."""
    made = []
    monkeypatch.setattr(b, "_same_device", lambda *a: None)
    for name in ("cache_write", "key_scores", "segment_permute", "block_mask", "attn_fwd", "unpermute"):
        monkeypatch.setattr(b, name, lambda *a, _n=name, **kw: made.append(_n))
    monkeypatch.setattr(b, "_launch", lambda what, *a: made.append(what))
    cache = b.Cache.__new__(b.Cache)
    cache.K, cache.dev, cache.h_kv, cache.c = torch.zeros(40, 1, 16, 128, dtype=torch.bfloat16), 0, 1, None
    pipe = b.Pipeline(b.problem(batch=2, h_q=2, h_kv=1, n=256, d=128, block=128, segment=256, dtype="bf16", tau=0.9), device="cpu")
    Q, K = (torch.zeros(2, h, 256, 128, dtype=torch.bfloat16) for h in (2, 1))
    return made, pipe, cache, (Q, K, K)


def _marks(cache, weight=True, position=True):
    return b.CacheMarks(cache, torch.zeros(40, 1, 16) if weight else None, torch.zeros(40, 1, 16, dtype=torch.int32) if position else None)


SLOTS = torch.arange(512, dtype=torch.int32).view(2, 256)


def test_a_refused_run_has_written_nothing(path):
    made, pipe, cache, qkv = path
    other = b.Cache.__new__(b.Cache)
    other.__dict__.update(cache.__dict__)
    marks = _marks(cache)
    for kw in (dict(marks=marks), dict(marks=marks, positions=SLOTS[:1]), dict(marks=marks, positions=SLOTS.long()),
               dict(marks=marks, positions=torch.zeros(2, 512, dtype=torch.int32)[:, ::2]), dict(marks=_marks(other), positions=SLOTS)):
        with pytest.raises(b.PbsError, match="pbs_cache_mark"):
            pipe.run(*qkv, cache=cache, slots=SLOTS, **kw)
        assert made == [], kw
    with pytest.raises(b.PbsError, match="pbs_cache_mark"):
        pipe.run(*qkv, marks=marks, positions=SLOTS)
    with pytest.raises(b.PbsError, match="slots"):
        pipe.run(*qkv, cache=cache, slots=SLOTS[:1], marks=marks, positions=SLOTS)
    assert made == []


def test_positions_are_asked_for_where_the_marks_have_them(path):
    made, pipe, cache, qkv = path
    pipe.run(*qkv, cache=cache, slots=SLOTS, marks=_marks(cache, position=False))
    same = torch.arange(256, dtype=torch.int32).expand(2, 256)                 # (rows of one memory)
    pipe.run(*qkv, cache=cache, slots=SLOTS, marks=_marks(cache), positions=same)
    pipe.run(*qkv, cache=cache, slots=SLOTS, marks=_marks(cache, weight=False), positions=same)
    assert made == 3 * (["cache_write"] * 2 + ["key_scores"] + ["pbs_cache_mark"] * 2 + ["segment_permute", "block_mask", "attn_fwd", "unpermute"])
