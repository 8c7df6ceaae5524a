"""Where a call on a stream of the caller's takes its own memory: from that stream, never from the current one, whose queued work may still use
what it has freed.  The library and the allocator are stood in for, so no GPU is needed."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2306_09342_amd import binding as B

SIDE, OTHER = SimpleNamespace(cuda_stream=5, name="side"), SimpleNamespace(cuda_stream=6, name="other")
CURRENT = SimpleNamespace(cuda_stream=0, name="current")
VOCAB = B.make_vocab_cfg(6, 64, 40, "bf16", top_k=3)


def _vocab_inputs():
    X = torch.zeros(6, 64, dtype=torch.bfloat16)
    rows, top = torch.zeros(6), torch.zeros(6, 3)
    return dict(params=torch.zeros(40 * 65, dtype=torch.bfloat16), X=X, labels=rows.int(), rows=rows, idx=top.int(), logits=top, lse=torch.zeros(2, 6))


def _vocab_call(name, **more):
    i = _vocab_inputs()
    teacher = (i["idx"], i["logits"])
    if name == "rev_xent_forward":
        return B.rev_xent_forward(VOCAB, i["params"], i["X"], i["labels"], **more)
    if name == "rev_xent_backward":
        return B.rev_xent_backward(VOCAB, i["params"], i["X"], i["labels"], i["rows"], i["rows"], **more)
    if name == "rev_distill_forward":
        return B.rev_distill_forward(VOCAB, i["params"], i["X"], *teacher, labels=i["labels"], **more)
    return B.rev_distill_backward(VOCAB, i["params"], i["X"], *teacher, i["lse"], i["rows"], labels=i["labels"], dloss_ce=i["rows"], **more)


STACK = B.make_cfg(n_blocks=2, d_model=64, n_heads=2, d_mlp=128, seq_len=16, batch=1, mode="bf16")
MERGE = B.make_merge_cfg(1, 4, 4, 2, 32)


def _stack_call(name, stream=None, **more):
    x, p = torch.zeros(1, 16, 64), torch.zeros(8)
    key_len = (torch.ones(1).int(),) if name.endswith("_masked") else ()
    if "forward" in name:
        return getattr(B, name)(STACK, p, x, x, *key_len, stream=stream, **more)
    if "pareprop" in name:
        return getattr(B, name)(STACK, p, x, x, *key_len, x, x, OTHER, stream_grad=stream, want_inputs=True, **more)
    chain = (1,) if name.endswith("_chain") else ()
    return getattr(B, name)(STACK, p, x, x, *key_len, x, x, *chain, stream=stream, want_inputs=True, **more)


def _merge_call(name, **more):
    x, y, p = torch.zeros(16, 32), torch.zeros(4, 64), torch.zeros(8)
    return B.rev_merge_forward(MERGE, p, x, x, **more) if name == "rev_merge_forward" else B.rev_merge_backward(MERGE, p, x, x, y, y, **more)


CALLS = {n: _vocab_call for n in ("rev_xent_forward", "rev_xent_backward", "rev_distill_forward", "rev_distill_backward")}
CALLS.update({"rev_stack_" + n: _stack_call for n in ("forward", "forward_masked", "backward_reprop", "backward_reprop_masked", "backward_pareprop",
                                                      "backward_pareprop_masked", "backward_chain")})
CALLS.update({n: _merge_call for n in ("rev_merge_forward", "rev_merge_backward")})


@pytest.fixture
def memory(monkeypatch):
    """Every tensor that is allocated, with the stream whose memory it is and the streams it is kept for."""
    now, made = [CURRENT], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def watch(make):
        def made_by(*a, **k):
            t = make(*a, **k)
            made.append(SimpleNamespace(tensor=t, stream=now[-1].name, kept=[]))
            return t
        return made_by

    def keep(t, stream):
        next(m for m in made if m.tensor is t).kept.append(stream.name)

    class Library:
        def __getattr__(self, name):
            does = name.startswith(("rev_stack_forward", "rev_stack_backward_reprop", "rev_stack_backward_pareprop", "rev_stack_backward_chain")) or name in (
                "rev_merge_forward", "rev_merge_backward")
            return (lambda *a: 0) if does else getattr(real, name)

    real, library = B.lib(), Library()
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, watch(getattr(torch, name)))
    monkeypatch.setattr(torch.Tensor, "new_empty", watch(torch.Tensor.new_empty), raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream", keep, raising=False)
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_want", lambda *a: None)
    monkeypatch.setattr(B, "_vocab_call", lambda *a: None)
    return made


def _tensors(result):
    return [t for t in (result.values() if isinstance(result, dict) else result if isinstance(result, tuple) else [result]) if t is not None]


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_is_the_streams_own(name, memory):
    returned = _tensors(CALLS[name](name, stream=SIDE))
    assert returned and len(memory) > len(returned)              # and a workspace
    for m in memory:
        assert m.stream == "side"
        if any(m.tensor is t for t in returned):
            assert m.kept == ["current"]


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_of_the_current_stream(name, memory):
    returned = _tensors(CALLS[name](name))
    assert returned and len(memory) > len(returned) and all(m.stream == "current" and not m.kept for m in memory)
