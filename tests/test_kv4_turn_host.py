"""DecodeSession.turn refuses what it cannot take, before anything is enqueued (CPU)."""
from types import SimpleNamespace

import pytest
import torch


def test_turns_that_do_not_fit_are_refused():
    from paper_2606_31519_amd import pipeline
    B, Hq, Hkv, D = 2, 4, 2, 64
    win = torch.zeros(B, Hkv, 8, D)
    ses = SimpleNamespace(state=SimpleNamespace(B=B, Hq=Hq, Hkv=Hkv, D=D, cap=40), kv4=object(), K_win=win, V_win=win, window=8,
                          n=30, w=5)
    turn = lambda q, k, v: pipeline.DecodeSession.turn(ses, q, k, v)  # noqa: E731
    x = lambda T, H, **kw: torch.zeros(B, T, H, D, **kw)  # noqa: E731
    assert turn(x(0, Hq), x(0, Hkv), x(0, Hkv)).shape == (B, 0, Hq, D)
    for bad in ((x(3, Hq), x(2, Hkv), x(2, Hkv)), (x(3, Hkv), x(3, Hkv), x(3, Hkv)), (x(3, Hq), x(3, Hkv), x(2, Hkv)),
                (x(3, Hq)[:1], x(3, Hkv), x(3, Hkv)), (x(3, Hq), x(3, Hkv), x(3, Hkv, dtype=torch.bfloat16)),
                (x(3, Hq).bfloat16(), x(3, Hkv).bfloat16(), x(3, Hkv).bfloat16())):
        with pytest.raises(ValueError):
            turn(*bad)
    with pytest.raises(RuntimeError, match="exceed"):
        turn(x(6, Hq), x(6, Hkv), x(6, Hkv))
    ses.kv4 = None
    with pytest.raises(ValueError, match="kv4"):
        turn(x(3, Hq), x(3, Hkv), x(3, Hkv))
