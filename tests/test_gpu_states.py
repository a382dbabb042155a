"""A state's steps of every kind one after the other on the device, against the model of tests/states_model.py: eagerly, captured and replayed, and on a
stream that is not the current one."""
import pytest
import torch

from paper_2404_15949_amd import corm
from tests.states_model import Follower, rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _follower(seed, dtype="f32", cap=64 * 4, r=4, B=2, Hq=4, Hkv=2, d=64, **wants):
    return Follower(torch.Generator().manual_seed(seed), B, Hq, Hkv, d, cap, dtype, r=r, device=DEV, **wants)


def _mixed(f):
    """Steps by weight over a block's end, cuts, block steps before and behind them, a second prompt."""
    f.blocks(2, 1)
    for _ in range(8):
        f.weigh()
    f.blocks(2, 1)
    f.weigh(budget=66)
    f.blocks(2, 1)
    f.blocks(1, 1)
    f.weigh()
    f.weigh(budget=62)
    f.blocks(3, 2)


@pytest.mark.parametrize("dtype,Hq,d", [("f32", 4, 64), ("bf16", 8, 128), ("bf16", 2, 64)])
def test_steps_by_weight_and_block_steps_on_one_state(dtype, Hq, d):
    f = _follower(1, dtype, Hq=Hq, d=d, want_weight=True, want_bounds=True)
    f.preload(60)
    f.check_rows()
    _mixed(f)
    f.preload(130)
    f.check_rows()
    _mixed(f)
    f.preload(7)
    _mixed(f)


class _Replayed:
    """The state, but for steps that are copied into a captured graph's inputs and replayed (one graph for each step and its numbers)."""

    def __init__(self, st, like):
        self._st, self._graphs = st, {}
        self._in = [torch.zeros_like(x) for x in like]

    def __getattr__(self, name):
        return getattr(self._st, name)

    def _step(self, name, args, numbers):
        key = (name,) + numbers
        if key not in self._graphs:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                getattr(self._st, name)(*self._in, *numbers)
            self._graphs[key] = (g, getattr(self._st, "blocks", None))
        for x, y in zip(self._in, args):
            x.copy_(y)
        g, self.blocks = self._graphs[key]
        g.replay()
        torch.cuda.synchronize()

    def step_blocks(self, *args):
        self._step("step_blocks", args[:4], args[4:])

    def step_weigh(self, *args):
        self._step("step_weigh", args[:4], args[4:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_mixed_steps_captured_and_replayed(dtype):
    """Each kind of step is captured when it is first met and replayed from then on: nothing a later step needs hangs on the state's own flags."""
    warm = _follower(2, dtype, want_weight=True, want_bounds=True)
    warm.preload(60)
    warm.blocks(2, 1)
    warm.weigh(50)
    f = _follower(3, dtype, want_weight=True, want_bounds=True)
    f.preload(60)
    f.st = _Replayed(f.st, [x for x in _tokens(f)])
    _mixed(f)
    f.preload(100)
    f.check_rows()
    _mixed(f)


def _tokens(f):
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[f.dtype]
    return [torch.zeros(f.B, n, f.d, dtype=t, device=DEV) for n in (f.Hq, f.Hkv, f.Hkv)] + [torch.zeros(f.B, dtype=torch.int32, device=DEV)]


class _OnStream:
    """The state, with its steps on a stream of its own."""

    def __init__(self, st):
        self._st, self._s = st, torch.cuda.Stream()

    def __getattr__(self, name):
        return getattr(self._st, name)

    def _run(self, step, *args):
        self._s.wait_stream(torch.cuda.current_stream())
        step(*args, stream=self._s)
        self._s.synchronize()

    def step_blocks(self, *args):
        self._run(self._st.step_blocks, *args)

    def step_weigh(self, *args):
        self._run(self._st.step_weigh, *args)


def test_a_block_step_captured_on_a_given_stream_goes_by_accounts():
    """The stream a step is given is the one that tells whether it is captured, not the current one."""
    f = _follower(8, "f32", want_weight=True, want_bounds=True)
    f.preload(60)
    f.blocks(2, 1)
    inputs, s, main = _tokens(f), torch.cuda.Stream(), torch.cuda.current_stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        with torch.cuda.stream(main):
            f.st.step_blocks(*inputs, 2, 1, stream=s)
    f.weigh(budget=30)
    f.st = _Once(f.st, graph, inputs)
    f.blocks(2, 1)


class _Once:
    """The state, with a block step that is a graph's."""

    def __init__(self, st, graph, inputs):
        self._st, self._graph, self._in = st, graph, inputs

    def __getattr__(self, name):
        return getattr(self._st, name)

    def step_blocks(self, *args):
        for x, y in zip(self._in, args[:4]):
            x.copy_(y)
        self._graph.replay()
        torch.cuda.synchronize()


def test_mixed_steps_on_another_stream():
    f = _follower(4, "bf16", want_weight=True, want_bounds=True)
    f.preload(60)
    f.st = _OnStream(f.st)
    _mixed(f)


def test_bounds_follow_corms_steps():
    """Seeding, steps, and steps in two phases evict on the device: the bounds are those of the rows that stayed, and a block step chooses by them."""
    f = _follower(5, "f32", cap=64 * 6, r=8, w=4, tcap=512, want_bounds=True)
    f.preload(230)
    t, t_first = (torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(2))
    t.fill_(230)
    f.st.prefill_seed(rows(f.g, "f32", 2, 4, 4, 64, scale=2.0).to(DEV), t, t_first)
    f.adopt()
    f.check_rows()
    assert all(len(f.K[u]) < 230 for u in f.at)
    evicted = 0
    for i in range(5):
        before = {u: len(f.K[u]) for u in f.at}
        q, args = f.token()
        if i % 2:
            f.st.step_attend(*args, t_first)
            f.st.step_evict()
        else:
            f.st.step(*args, t_first)
        f.adopt()
        f.check_rows()
        evicted += sum(before[u] + 1 - len(f.K[u]) for u in f.at)
    assert evicted > 0
    f.blocks(2, 1)
    f.blocks(1, 1)


def test_accounts_behind_seeding_on_another_stream():
    f = _follower(6, "f32", r=8, w=4, tcap=512, want_weight=True)
    f.preload(100)
    f.weight = {u: torch.zeros(100, dtype=torch.float64) for u in f.at}
    f.st.weight.fill_(2.0)
    t, t_first = torch.full((2,), 100, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    f.st.prefill_seed(rows(f.g, "f32", 2, 4, 4, 64, scale=2.0).to(DEV), t, t_first, stream=s)
    s.synchronize()
    f.adopt()
    assert not f.st.weight.any()
    f.weigh()
    f.weigh(budget=20)
    with pytest.raises(RuntimeError, match="accounts"):
        f.st.step(*f.token()[1], t_first)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_a_refused_8_bit_step_leaves_the_token_out(code):
    g = torch.Generator().manual_seed(7)
    st = corm.Q8State(1, 2, 1, 64, 256, "f32", code, device=DEV, want_bounds=True)
    st.append(rows(g, "f32", 1, 1, 100, 64).to(DEV), rows(g, "f32", 1, 1, 100, 64).to(DEV))
    q, k, v = (rows(g, "f32", 1, n, 64).to(DEV) for n in (2, 1, 1))
    for a in ((q, k, v, -1), (q.bfloat16(), k, v), (q[:, :1], k, v), (q, k, v, 513), (q, k, v, 2, 3)):
        with pytest.raises((ValueError, corm.CormError)):
            st.step(*a)
    assert int(st.lens) == 100
    st.step(q, k, v, 2, 2)
    assert int(st.lens) == 101 and st.blocks.tolist() == [[[0, 1]]]
