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


def test_a_state_with_accounts_evicts_by_one_rule(monkeypatch):
    """CORM's steps move rows without their accounts, steps by weight without last_hit: the second kind is refused, before anything is done."""
    made = plain_library(monkeypatch)
    f = _follower(3, want_weight=True)
    f.preload(40)
    q, args = f.token()

    def corms():
        st = f.st
        return (lambda: st.step(*args, None), lambda: st.step_lazy(*args, None), lambda: st.step_attend(*args, None), lambda: st.step_evict())

    for rule in ("weight", "hits"):
        for first in (lambda: f.st.step_weigh(*args),) if rule == "weight" else corms()[:2]:
            f.preload(40)
            first()
            made.clear()
            for second in corms() if rule == "weight" else (lambda: f.st.step_weigh(*args), lambda: f.st.step_weigh(*args, 20)):
                with pytest.raises(RuntimeError, match="accounts"):
                    second()
            assert made == []
    f = _follower(3)                    # without accounts there is nothing to lose
    f.preload(40)
    f.st.step(*args, None)
    f.st.step_lazy(*args, None)


def test_a_refused_step_takes_no_rule(monkeypatch):
    plain_library(monkeypatch)

    def refuse(*a, **k):
        raise corm.CormError(corm.CORM_EINVAL, "no")

    monkeypatch.setattr(corm, "corm_decode_step", refuse)
    f = _follower(4, want_weight=True)
    f.preload(40)
    q, args = f.token()
    with pytest.raises(corm.CormError):
        f.st.step(*args, None)
    f.preload(40)
    f.weigh()


def test_accounts_are_empty_behind_a_seeded_prompt(monkeypatch):
    """Seeding evicts by hits and cannot move accounts: what was in them is another prompt's."""
    plain_library(monkeypatch)
    f = _follower(5, want_weight=True)
    f.preload(40)
    f.st.weight.fill_(3.0)
    f.st.prefill_seed(rows(f.g, "f32", 2, 4, 4, 64), None, None)
    f.adopt()
    f.weigh()
    f.weigh(budget=30)


def test_bounds_follow_every_step(monkeypatch):
    """The bounds of every block after a prompt, steps of other kinds that complete blocks, cuts and a second prompt: those of the rows that are there."""
    plain_library(monkeypatch)
    f = _follower(9, want_weight=True, want_bounds=True)
    f.preload(60)
    f.check_rows()
    f.blocks(2, 1)
    for _ in range(10):                  # over a block's end, without block steps between
        f.weigh()
    f.blocks(2, 1)
    f.weigh(budget=66)                   # rows move
    f.preload(130)
    f.check_rows()
    f.blocks(2, 1)


def test_bounds_follow_corms_steps(monkeypatch):
    plain_library(monkeypatch)
    f = _follower(10, want_bounds=True)
    f.preload(150)
    f.st.prefill_seed(rows(f.g, "f32", 2, 4, 4, 64), None, None)
    f.adopt()
    f.check_rows()
    for _ in range(3):
        f.st.step(*f.token()[1], None)
        f.adopt()
        f.check_rows()
    f.blocks(2, 1)


def test_steps_that_know_no_dead_slots_are_refused_behind_deferred_compaction(monkeypatch):
    """Attention over chosen blocks would read evicted keys, and the row it appends would be taken for dead."""
    made = plain_library(monkeypatch)
    f = _follower(11, want_bounds=True)
    f.preload(100)
    f.blocks(2, 1)
    f.st.step_lazy(*f.token()[1], None)
    made.clear()
    with pytest.raises(RuntimeError, match="dead"):
        f.st.step_blocks(*f.token()[1], 2)
    assert made == []
    f.preload(100)
    f.blocks(2, 1)


def test_a_row_of_a_block_step_starts_with_an_empty_account(monkeypatch):
    """Behind a cut the slots from the new length on hold accounts of keys that moved or went."""
    plain_library(monkeypatch)
    f = _follower(6, want_weight=True, want_bounds=True)
    f.preload(100)
    f.weigh()
    f.weigh(budget=70)
    f.st.renew_bounds()
    for _ in range(3):
        f.blocks(2, 1)
    f.weigh()
    f.weigh(budget=66)


def test_a_row_of_a_block_step_has_never_been_hit(monkeypatch):
    """... of a state that evicts by hits: the slot's last_hit."""
    plain_library(monkeypatch)
    for wants in (dict(want_bounds=True), dict(want_bounds=True, want_weight=True)):
        f = _follower(7, **wants)
        f.preload(100)
        q, args = f.token()
        f.st.step(*args, None)
        f.adopt()
        f.st.last_hit.fill_(50)
        f.st.renew_bounds()
        f.blocks(2, 1)
        assert (f.st.last_hit[:, :, 100] == 0).all() and (f.st.last_hit[:, :, 101] == 50).all()


def test_a_captured_block_step_may_be_replayed_behind_a_cut(monkeypatch):
    """What a graph holds cannot know of steps that come later: a block step captured on a state with accounts sets the new row's account."""
    plain_library(monkeypatch)
    monkeypatch.setattr(corm, "_capturing", lambda stream: True)
    f = _follower(8, want_weight=True, want_bounds=True)
    f.preload(100)
    f.st.renew_bounds()
    f.st.weight[:, :, 100:] = 5.0       # as a cut between capture and replay leaves it
    f.blocks(2, 1)
    with pytest.raises(RuntimeError, match="accounts"):
        f.st.step(*f.token()[1], None)


REFUSED_Q = (("shape", lambda q: q[:, :2]), ("type", lambda q: q.bfloat16()), ("strides", lambda q: q.transpose(0, 1)), ("none", lambda q: None),
             ("address", lambda q: torch.zeros(q.numel() + 1)[1:].view_as(q)))


def test_a_refused_step_leaves_the_state_as_it_was(monkeypatch):
    """Choice, budget and query are looked at before the row goes in: a caller that mends its call and repeats it has the token once."""
    made = plain_library(monkeypatch)
    f = _follower(12, want_weight=True, want_bounds=True)
    f.preload(100)
    q, args = f.token()
    rest, st = args[1:], f.st
    before = [x.clone() for x in (st.K, st.V, st.lens, st.pos, st.last_hit, st.weight, st.bounds)]
    made.clear()

    def refused(step, *a):
        with pytest.raises((ValueError, TypeError, corm.CormError)):
            step(*a)
        assert made == [] and all(torch.equal(x, y) for x, y in zip(before, (st.K, st.V, st.lens, st.pos, st.last_hit, st.weight, st.bounds))), a[3:]

    for nsel, nlast in ((0, 1), (-1, 1), (2, 0), (2, 3), (513, 1), (1 << 32, 1), (2, -(1 << 32) + 1), (2.0, 1), (None, 1), (2, None)):
        refused(st.step_blocks, *args, nsel, nlast)
    for budget in (0, f.r - 1, -1, 1 << 31, (1 << 32) + 50, 50.0):
        refused(st.step_weigh, *args, budget)
    for _, bad in REFUSED_Q:
        refused(st.step_blocks, bad(args[0]), *rest, 2, 1)
        refused(st.step_weigh, bad(args[0]), *rest)
    monkeypatch.setattr(corm, "corm_append", lambda *a, **k: corm._check(corm.CORM_EINVAL, "no"))
    refused(st.step_weigh, *args)
    monkeypatch.undo()
    made = plain_library(monkeypatch)
    assert st._rule is None
    st.step_blocks(*args, 512, 512)
    st.step_weigh(*f.token()[1], f.r)


def test_a_refused_step_leaves_the_8_bit_cache_as_it_was(monkeypatch):
    made = []
    for name in ("corm_q8_append", "corm_q8_attend", "corm_block_select"):
        monkeypatch.setattr(corm, name, lambda *a, name=name, **k: made.append(name))
    monkeypatch.setattr(corm, "_device", lambda: -1)
    states = [corm.Q8State(2, 4, 2, 64, 640, "f32", device="cpu", want_bounds=w) for w in (True, False)]
    q, k = torch.zeros(2, 4, 64), torch.zeros(2, 2, 64)
    for nsel, nlast in ((-1, 1), (2, 0), (2, 3), (513, 1), (2.0, 1), (2, None)):
        for call in (lambda: states[0].step(q, k, k, nsel, nlast), lambda: states[0].attend(q, nsel, nlast)):
            with pytest.raises((TypeError, corm.CormError)):
                call()
    for call in (lambda: states[1].step(q, k, k, 2), lambda: states[1].attend(q, 2)):
        with pytest.raises(RuntimeError, match="want_bounds"):
            call()
    for _, bad in REFUSED_Q:
        with pytest.raises((ValueError, corm.CormError)):
            states[0].step(bad(q), k, k)
    assert made == []
    states[0].step(q, k, k, 512, 512)
    states[1].step(q, k, k)
    assert made == ["corm_q8_append", "corm_block_select", "corm_q8_attend", "corm_q8_append", "corm_q8_attend"]


def test_steps_allocate_nothing(monkeypatch):
    """Memory taken within a step would belong to the current stream, whose earlier work may still be using it, and be written on the step's."""
    plain_library(monkeypatch)
    monkeypatch.setattr(corm, "corm_q8_append", lambda *a, **k: None)
    monkeypatch.setattr(corm, "corm_q8_attend", lambda *a, **k: None)
    f = _follower(13, want_weight=True, want_bounds=True)
    f.preload(100)
    q8 = corm.Q8State(2, 4, 2, 64, 256, "f32", device="cpu", want_bounds=True)
    tokens = [f.token()[1] for _ in range(5)]

    def none(*a, **k):
        raise AssertionError("an allocation")

    with monkeypatch.context() as m:
        for name in ("empty", "zeros", "empty_like", "zeros_like"):
            m.setattr(torch, name, none)
        for args, (nsel, nlast) in zip(tokens, ((1, 1), (3, 2), (512, 7), (2, 2))):
            f.st.step_blocks(*args, nsel, nlast)
            assert f.st.blocks.shape == (2, 2, nsel) and f.st.blocks.is_contiguous()
            q8.step(*args[:3], nsel, nlast)
            assert q8.blocks.shape == (2, 2, nsel) and q8.blocks.is_contiguous()
        f.st.step_weigh(*tokens[4], 60)


def test_the_choice_asks_for_its_workspace():
    """It has never done without one."""
    with pytest.raises(TypeError):
        corm.corm_block_select(corm.make_desc(2, 4, 2, 64, 256, 256, 4, 4, "f32"), 4096, 4096, 4096, 8, 2, 4096)


def test_layers_may_share_their_workspaces(monkeypatch):
    plain_library(monkeypatch)
    room = _room(corm.corm_blocks_workspace_bytes(corm.make_desc(2, 4, 2, 64, 256, 256, 4, 4, "f32")))
    layers = [_follower(15, want_bounds=True, want_weight=w, blocks_workspace=room) for w in (True, False)]
    for f in layers:
        assert f.st.blocks_workspace is room
        f.preload(100)
        f.blocks(2, 1)


def _room(nbytes):
    x = torch.empty(nbytes + 256, dtype=torch.uint8)
    x = x[-x.data_ptr() % 256:]
    return x[:nbytes]


def test_a_workspace_that_does_not_do_is_refused_where_it_is_given():
    """Not by the second call of a step, behind the row that the first one has put in."""
    args, small = (2, 4, 2, 64, 256), torch.empty(256, dtype=torch.uint8)
    desc = corm.make_desc(*args, 256, 4, 4, "f32")
    room = [_room(n(desc) + 256) for n in (corm.corm_workspace_bytes, corm.corm_blocks_workspace_bytes)]
    layer = dict(device="cpu", want_ring=False, want_bounds=True, want_weight=True)
    for bad in (small, room[1][16:], room[1][::2]):
        for make in (lambda: corm.LayerState(*args, 256, 4, 4, "f32", workspace=room[0], blocks_workspace=bad, **layer),
                     lambda: corm.Q8State(*args, "f32", device="cpu", workspace=bad)):
            with pytest.raises((ValueError, corm.CormError)):
                make()
    for bad in (small, room[0][16:], room[0][::2]):
        with pytest.raises((ValueError, corm.CormError)):
            corm.LayerState(*args, 256, 4, 4, "f32", workspace=bad, blocks_workspace=room[1], **layer)
    corm.LayerState(*args, 256, 4, 4, "f32", workspace=room[0], blocks_workspace=room[1], **layer)
    corm.Q8State(*args, "f32", device="cpu", workspace=room[1])
