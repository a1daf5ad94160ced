"""`stream=` means the same in every call of the cache, its attention and the
rotary axes: the given stream waits for the current one, then the call is
queued there.  On the host, with the library's entry points and the streams
replaced by records of what they were asked."""
import types

import pytest
import torch

from paper_2609_00865_amd import mv

BF = torch.bfloat16


class Stream:
    device = torch.device("cuda", 0)

    def __init__(self, handle):
        self.cuda_stream, self.waited = handle, []

    def wait_stream(self, other):
        self.waited.append(other)


@pytest.fixture
def calls(monkeypatch):
    """Every call that takes a stream, and the record of the handles they passed on."""
    handles, cur = [], Stream(11)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: cur)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None, raising=False)
    monkeypatch.setattr(mv, "_need", lambda *a, **k: None)
    monkeypatch.setattr(mv, "_device", lambda: 0)
    for name in ("mv_rope_axes", "mv_cache_reset", "mv_cache_status", "mv_cache_reserve",
                 "mv_cache_write", "mv_cache_fork", "mv_cache_compact", "mv_cache_free",
                 "mv_tree_attn", "mv_tree_mask"):
        monkeypatch.setattr(mv, name, lambda *a: handles.append(a[-1]) or 0)
    for name in ("mv_cache_compact_workspace_bytes", "mv_tree_attn_workspace_bytes"):
        monkeypatch.setattr(mv, name, lambda *a: 64)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    rows = lambda heads: torch.zeros(3, heads, 64, dtype=BF)
    c = types.SimpleNamespace(_args=lambda: (None, None), _refs=(None, None), _t=(i32(1),),
                              shape=mv.CacheShape(1, 8, 16, 2, 64, 4, 4), head_dim=64, k=rows(2))
    rope = mv.RopeAxes(64, [0] * 32)
    out = (rows(4), torch.zeros(4, 3))
    ws = torch.zeros(64, dtype=torch.uint8)
    todo = {
        "reset": lambda s: mv.PagedCache.reset(c, stream=s),
        "status": lambda s: mv.PagedCache.status(c, stream=s),
        "reserve": lambda s: mv.cache_reserve(c, i32(2), i32(3), 3, stream=s),
        "write": lambda s: mv.cache_write(c, 0, i32(3), rows(2), rows(2), stream=s),
        "write_rotated": lambda s: mv.cache_write(c, 0, i32(3), rows(2), rows(2), rope=rope,
                                                  pos=i32(1, 3), stream=s),
        "fork": lambda s: mv.cache_fork(c, i32(2), i32(2), stream=s),
        "fork_given": lambda s: mv.cache_fork(c, i32(2), i32(2), workspace=ws, stream=s),
        "compact": lambda s: mv.cache_compact(c, i32(2), i32(2), i32(3), i32(1, 2), stream=s),
        "compact_given": lambda s: mv.cache_compact(c, i32(2), i32(2), i32(3), i32(1, 2),
                                                    workspace=ws, stream=s),
        "free": lambda s: mv.cache_free(c, i32(2), stream=s),
        "mask": lambda s: mv.tree_mask(i32(3), i32(2), 3, stream=s),
        "attn": lambda s: mv.tree_attn(c, 0, rows(4), i32(1), i32(2), stream=s),
        "attn_given": lambda s: mv.tree_attn(c, 0, rows(4), i32(1), i32(2), out=out, workspace=ws,
                                             stream=s),
        "rope": lambda s: mv.rope_axes(rows(4), i32(1, 3), rope, stream=s),
        "rope_given": lambda s: mv.rope_axes(rows(4), i32(1, 3), rope, out=out[0], stream=s),
    }
    return todo, handles, cur


def test_a_given_stream_waits_for_the_current_one(calls):
    todo, handles, cur = calls
    for name, call in todo.items():
        side = Stream(22)
        call(side)
        assert side.waited == [cur], name
        assert handles[-1] == 22, name
    assert len(handles) == len(todo)


def test_on_the_current_stream_nothing_waits(calls):
    todo, handles, cur = calls
    for name, call in todo.items():
        call(None)
        call(cur)
        assert not cur.waited and handles[-2:] == [11, 11], name


def test_a_stream_of_another_device_is_refused(calls):
    """Kernels would run there, on pointers of the current device."""
    todo, handles, cur = calls
    for name, call in todo.items():
        side = Stream(22)
        side.device = torch.device("cuda", 1)
        with pytest.raises(ValueError, match="stream"):
            call(side)
        assert not side.waited and not handles, name


@pytest.mark.gpu
def test_a_side_stream_sees_what_was_queued():
    """Rows that are still being computed on the current stream, written and
    rotated on another one, read by the status and freed there."""
    gen = torch.Generator().manual_seed(1)
    n, heads, d = 48, 2, 64
    rope = mv.RopeAxes(d, [0] * 32, 1e4)
    c = mv.PagedCache(1, 8, 16, heads, d, 2, 4)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    x = torch.randn(n, heads, d, generator=gen).to(BF).cuda()
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    big = torch.randn(4096, 4096, generator=gen).cuda()
    ids, ptr = i32([1]), i32([0, n])
    side = torch.cuda.Stream()
    k, y, z = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    want = mv.rope_axes(x, pos, rope)
    torch.cuda.synchronize()
    for _ in range(20):
        big = (big @ big).clamp_(-1, 1)
    k.copy_(x + (big.sum() * 0).to(BF))
    slot, _ = mv.cache_reserve(c, ids, ptr, n)
    mv.cache_write(c, 0, slot, k, k, stream=side)
    mv.rope_axes(k, pos, rope, out=y, stream=side)
    assert c.status(stream=side)["free_pages"] == 5
    mv.rope_axes(y, pos, rope, inverse=True, out=z, stream=side)
    mv.cache_free(c, ids, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    place = slot.long()
    assert torch.equal(c.k[0, place // 16, :, place % 16], x)
    assert torch.equal(c.v[0, place // 16, :, place % 16], x)
    assert torch.equal(y, want)
    assert c.status()["free_pages"] == 8
