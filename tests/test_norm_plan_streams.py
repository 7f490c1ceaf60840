"""Whose memory a norm plan's table is: work that is queued on another stream than the one that builds it must not write
it, and it must not be given away under a call on another stream (no GPU needed: who is waited for, and in which order;
the GPU test in test_gpu_norm_streams.py looks at the memory itself)."""
import types

import pytest
import torch

import paper_2606_25759_amd as nf
from paper_2606_25759_amd import binding

CURRENT, SIDE = 0x11, 0x22


class Stream:
    def __init__(self, handle, log):
        self.cuda_stream, self.log = handle, log

    def synchronize(self):
        self.log.append(("wait", self.cuda_stream))


class Tensor:
    """What the calls ask of a device tensor."""
    is_cuda, dtype, device, shape = True, torch.uint8, "cuda:0", (1,)

    def __init__(self, log, dtype=torch.uint8):
        self.log, self.dtype = log, dtype

    def get_device(self):
        return 0

    def data_ptr(self):
        return 0x10000

    def numel(self):
        return 1

    def is_contiguous(self):
        return True

    def record_stream(self, stream):
        self.log.append(("keep", stream.cuda_stream))


@pytest.fixture
def card(monkeypatch):
    log = []
    streams = {h: Stream(h, log) for h in (0, CURRENT, SIDE)}
    state = types.SimpleNamespace(log=log, streams=streams, current=CURRENT, capturing=False)

    def call(name):
        def fn(*args):
            handle = args[-1]
            log.append((name, handle))
            return 0
        return fn

    lib = types.SimpleNamespace(**{name: call(name) for name in ("nf_norm_table_init", "nf_grad_norm", "nf_grad_clip",
                                                                 "nf_grad_norm_clip")})

    def plan_init(entries, count, groups, plan):
        plan._obj.groups = groups
        return 0

    lib.nf_norm_plan_init = plan_init
    monkeypatch.setattr(binding, "load", lambda path=None: lib)
    monkeypatch.setattr(binding, "empty_workspace", lambda n, device="cuda": Tensor(log))
    monkeypatch.setattr(binding, "_raw_stream", lambda device: state.current)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: streams[state.current])
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: streams[0])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state.capturing)
    return state


def calls(plan, card, stream):
    norms, ws = Tensor(card.log, torch.float32), Tensor(card.log)
    return (lambda: nf.nf_grad_norm(plan, norms, ws, stream=stream),
            lambda: nf.nf_grad_clip(plan, norms, 1.0, stream=stream),
            lambda: nf.nf_grad_norm_clip(plan, 1.0, norms, ws, stream=stream))


def test_a_table_is_built_behind_what_its_memory_was_used_for(card):
    """The memory comes from the current stream, whose queued work may still write it when the copy is another's."""
    nf.norm_plan([], n_groups=1, stream=card.streams[SIDE])
    assert card.log == [("wait", CURRENT), ("nf_norm_table_init", SIDE)]
    del card.log[:]
    nf.norm_plan([], n_groups=1, stream=SIDE)
    assert card.log == [("wait", CURRENT), ("nf_norm_table_init", SIDE)]
    del card.log[:]
    nf.norm_plan([], n_groups=1)  # in order by itself
    nf.norm_plan([], n_groups=1, stream=card.streams[CURRENT])
    assert card.log == [("nf_norm_table_init", CURRENT)] * 2


@pytest.mark.parametrize("which", range(3))
def test_a_table_stays_while_another_stream_reads_it(card, which):
    for stream in (card.streams[SIDE], card.streams[0], 0):
        plan = nf.norm_plan([], n_groups=1)
        handle = getattr(stream, "cuda_stream", stream)
        del card.log[:]
        calls(plan, card, stream)[which]()
        assert ("keep", handle) in card.log
    plan = nf.norm_plan([], n_groups=1)
    del card.log[:]
    for stream in (None, card.streams[CURRENT]):  # the stream that the memory belongs to
        calls(plan, card, stream)[which]()
    assert not [e for e in card.log if e[0] == "keep"]
    card.current = SIDE  # another has become the current one
    calls(plan, card, None)[which]()
    assert ("keep", SIDE) in card.log
    del card.log[:]
    calls(plan, card, None)[which]()
    assert not [e for e in card.log if e[0] == "keep"]  # once is enough


@pytest.mark.parametrize("which", range(3))
def test_nothing_is_noted_in_a_capture(card, which):
    """A graph's replays are not the allocator's to see: a plan outlives the graphs that hold its calls."""
    plan = nf.norm_plan([], n_groups=1)
    del card.log[:]
    card.current, card.capturing = SIDE, True
    calls(plan, card, None)[which]()
    assert not [e for e in card.log if e[0] == "keep"]
    card.capturing = False
    calls(plan, card, None)[which]()
    assert ("keep", SIDE) in card.log


def test_another_librarys_stream(card):
    """An object that has a handle and is not torch's: taken as the handle."""
    plan = nf.norm_plan([], n_groups=1)
    plan.table.record_stream = lambda stream: (_ for _ in ()).throw(TypeError("not a stream"))
    del card.log[:]
    for call in calls(plan, card, types.SimpleNamespace(cuda_stream=SIDE)):
        call()
    assert [e[1] for e in card.log] == [SIDE] * 3
