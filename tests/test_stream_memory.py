"""Whose memory a call on a stream of its own gets.  The caching allocator orders the uses
of a block along the stream that it was allocated on: what a call on another stream than
the current one allocates has to be that stream's, or it may still be in use on the current
one.  Here with streams and tensors that only note what happens to them."""
import contextlib
import types

import pytest
import torch

HERE, SIDE = object(), object()


class Block:
    def __init__(self, stream):
        self.stream, self.recorded = stream, []
        self.shape, self.dtype, self.device = (2, 4, 64), torch.bfloat16, "fake"

    def record_stream(self, s):
        self.recorded.append(s)

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return 512

    def element_size(self):
        return 1

    def is_contiguous(self):
        return True

    def view(self, *a):
        return self


@pytest.fixture
def made(monkeypatch):
    """The blocks that calls allocate, in order."""
    from paper_2607_25422_amd import binding as b
    at, blocks = [HERE], []

    def new(*a, **kw):
        blocks.append(Block(at[-1]))
        return blocks[-1]

    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()
    for name in ("empty", "empty_like", "empty_strided"):
        monkeypatch.setattr(torch, name, new)
    for name in ("new_empty",):
        monkeypatch.setattr(Block, name, lambda self, *a, **kw: new(), raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: at[-1])
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(b, "_torch_stream", lambda s: at[-1] if s is None else s)
    b_made = types.SimpleNamespace(b=b, blocks=blocks)
    return b_made


def problem(b):
    p = b.make_problem("bf16", B=2, d=256, H=4, d_h=64, kept_offsets=[0, 1, 2])
    p.L_max = 4000
    return p


def calls(b, monkeypatch):
    """name -> call(stream): every call that allocates and takes a stream."""
    for low in ("skip_cache_append", "skip_cache_attn", "skip_cache_select",
                "skip_cache_attn_pages", "skip_quantize_passages"):
        monkeypatch.setattr(b, low, lambda *a, **kw: None)
    p, q = problem(b), Block(HERE)
    cache = types.SimpleNamespace(k=Block(HERE))
    odd = Block(HERE)
    odd.dtype = torch.float32
    store = types.SimpleNamespace(data=q)
    return {
        "append": lambda s: b.cache_append(p, cache, q, q, q, q, q, stream=s),
        "append of other rows": lambda s: b.cache_append(p, cache, odd, q, q, q, q, stream=s),
        "attn": lambda s: b.cache_attn(p, cache, q, q, q, stream=s),
        "select": lambda s: b.cache_select(p, cache, q, q, q, 4, stream=s),
        "attn_pages": lambda s: b.cache_attn_pages(p, cache, q, q, q, q, stream=s),
        "keys of a store": lambda s: b.quantize_passages(p, store, q, q, q, q, want_keys=True,
                                                         stream=s),
    }


NAMES = ("append", "append of other rows", "attn", "select", "attn_pages", "keys of a store")


@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_the_streams(made, monkeypatch, name):
    """Allocated on the call's stream, and recorded on the current one, whose program
    has them."""
    call = calls(made.b, monkeypatch)
    assert tuple(call) == NAMES
    # (a slice of the keys is what is returned)
    monkeypatch.setattr(Block, "__getitem__", lambda self, i: self, raising=False)
    call[name](SIDE)
    assert made.blocks and all(x.stream is SIDE for x in made.blocks)
    assert all(x.recorded == [HERE] for x in made.blocks)
    for same in (None, HERE):
        made.blocks.clear()
        call[name](same)
        assert made.blocks and all(x.stream is HERE and not x.recorded for x in made.blocks)


def test_workspaces_are_the_streams(made, monkeypatch):
    """They are used on the call's stream alone, and need no record."""
    b, p = made.b, problem(made.b)
    monkeypatch.setattr(b, "workspace_bytes", lambda p: 1000)
    monkeypatch.setattr(b, "_cache_bytes", lambda *a: 1000)
    monkeypatch.setattr(b, "_dptr", lambda t, *a: t.data_ptr())
    for make in (lambda s: b._fresh_workspace(1000, "fake", s), lambda s: b._ws(p, None, s),
                 lambda s: b._cache_ws(p, None, None, 0, False, False, "fake", s, 0)):
        for s, want in ((SIDE, SIDE), (HERE, HERE), (None, HERE)):
            made.blocks.clear()
            make(s)
            assert len(made.blocks) == 1 and made.blocks[0].stream is want
            assert not made.blocks[0].recorded
