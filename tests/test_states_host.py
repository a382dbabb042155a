"""A state's own bookkeeping, on the CPU: steps of every kind one after the other, with plain forms in the place of the library's calls, against the
model of tests/states_model.py."""
import pytest
import torch

from paper_2404_15949_amd import corm
from tests.states_model import Follower, plain_library, rows


def _follower(seed, cap=64 * 4, r=4, **wants):
    return Follower(torch.Generator().manual_seed(seed), 2, 4, 2, 64, cap, "f32", r=r, **wants)


def test_a_second_prompt_starts_with_empty_accounts(monkeypatch):
    plain_library(monkeypatch)
    f = _follower(1, want_weight=True)
    f.preload(40)
    for _ in range(3):
        f.weigh()
    f.preload(50)                    # longer, and (below) shorter than what the slots held
    assert not f.st.weight.any()
    for _ in range(3):
        f.weigh(budget=48)
    f.preload(20)
    assert not f.st.weight.any()
    f.weigh()


def test_a_second_prompt_has_no_dead_slots(monkeypatch):
    plain_library(monkeypatch)
    f = _follower(2)
    f.preload(40)
    q, args = f.token()
    f.st.step_lazy(*args, None)
    assert (f.st.live != -1).any()
    f.preload(50)
    assert (f.st.live == -1).all()
