"""What the Python binding does around the library's calls, without a GPU: the library, the tensors' checks and torch's streams are stand-ins."""
import contextlib
import ctypes
import types

import pytest
import torch

import paper_2605_12471_amd as kv
from paper_2605_12471_amd import binding

HKV, D, CAPACITY = 2, 64, 100


class Streams:
    """torch's streams, by their handles: which is current, and which was at each allocation."""

    def __init__(self, monkeypatch, current=5):
        self.current, self.made, self.recorded = current, [], []
        empty = torch.empty

        @contextlib.contextmanager
        def within(stream):
            outer, self.current = self.current, stream.cuda_stream
            yield
            self.current = outer

        def spy(*shape, **kw):
            t = empty(*shape, **kw)
            self.made.append((t.data_ptr(), self.current))
            return t
        monkeypatch.setattr(torch, "empty", spy)
        monkeypatch.setattr(torch.cuda, "stream", within)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: types.SimpleNamespace(cuda_stream=handle))
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=self.current))
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: self.current + 100 * device, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)  # (the current device)
        monkeypatch.setattr(torch.Tensor, "is_cuda", True)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.recorded.append((t.data_ptr(), s.cuda_stream)))

    def of(self, address):
        return [s for a, s in self.made if a == address][-1]


def a_cache(monkeypatch, native):
    """A cache without a library behind it, and the calls of kvfold_cache_evict that it makes: (kept, workspace, stream)."""
    calls, cache = [], object.__new__(kv.KvFoldCache)
    cache.handle, cache._device, cache._hq, cache._hkv, cache._d, cache._capacity = ctypes.c_void_p(1), 0, 4, HKV, D, CAPACITY
    cache._check, cache.close = lambda *a, **k: None, lambda: None
    monkeypatch.setattr(binding, "kvfold_evict_workspace_bytes", lambda handle, n_keep: 1000)

    def plain(handle, layer, weights, n_keep, n_sink, n_recent, to, to_layer, to_weights, kept, workspace, n_bytes, stream):
        calls.append((kept, workspace, stream))
        return 0

    def fast(bound, layer, weights, n_keep, n_sink, n_recent, into, to_layer, to_weights, kept, workspace, stream):
        calls.append((kept.data_ptr(), workspace.data_ptr(), cache._stream(stream)))
        return 0
    cache._lib = types.SimpleNamespace(kvfold_cache_evict=plain)
    cache._bound_weights = object() if native else None
    monkeypatch.setattr(binding, "_native", types.SimpleNamespace(evict=fast))
    return cache, calls


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("stream", [None, 5, 7, 0])
@pytest.mark.parametrize("given", ["nothing", "kept", "workspace", "both"])
def test_what_an_eviction_takes_is_its_streams_own(monkeypatch, native, stream, given):
    """Memory of another stream's pool may be given to that stream's next tensor while the eviction still uses it, or be in use there still."""
    cache, calls = a_cache(monkeypatch, native)
    kept = torch.zeros((HKV, 10), dtype=torch.int32) if given in ("kept", "both") else None
    space = torch.zeros(1000, dtype=torch.uint8) if given in ("workspace", "both") else None
    streams = Streams(monkeypatch)
    rows = cache.evict(0, torch.zeros((HKV, CAPACITY)), 10, kept=kept, workspace=space, stream=stream)
    (at_kept, at_space, used), = calls
    assert used == (5 if stream is None else stream) and streams.current == 5
    assert rows is kept if kept is not None else rows.data_ptr() == at_kept
    for mine, address in ((kept, at_kept), (space, at_space)):
        assert address == mine.data_ptr() if mine is not None else streams.of(address) == used
    # what is handed out may be used, and let go, on the current stream
    assert streams.recorded == ([(at_kept, 5)] if kept is None and used != 5 else [])


@pytest.mark.parametrize("call", ["step", "noalloc", "rope", "window", "weigh", "evict"])
def test_the_current_stream_is_that_of_the_caches_device(monkeypatch, call):
    """A cache on another GPU than the current one: the stream that is current there (100 stands for its device in the handle)."""
    cache, calls = a_cache(monkeypatch, native=False)
    Streams(monkeypatch)
    cache._device, cache._bound, cache.dtype_name, cache.length = 1, None, "bf16", lambda layer: 0
    names = ("kvfold_step_ex", "kvfold_step_noalloc", "kvfold_step_rope", "kvfold_step_window", "kvfold_cache_weigh", "kvfold_cache_evict")
    cache._lib = types.SimpleNamespace(**{name: lambda *a: calls.append(a[-1]) for name in names})
    for name in names:
        monkeypatch.setattr(binding, name, lambda *a: calls.append(a[-1]))
    q, k = torch.zeros((3, 4, D), dtype=torch.bfloat16), torch.zeros((3, HKV, D), dtype=torch.bfloat16)
    angles = (torch.zeros((3, D // 2)), torch.zeros((3, D // 2)))
    if call == "weigh":
        cache.weigh(0, q, torch.zeros((4, 3)), torch.zeros((HKV, CAPACITY)))
    elif call == "evict":
        cache.evict(0, torch.zeros((HKV, CAPACITY)), 10)
    else:
        cache.step(0, q, k, k, torch.zeros_like(q), **{"step": {}, "noalloc": {"noalloc": True}, "rope": {"rope": angles}, "window": {"window": (1, 2)}}[call])
    assert calls == [105]


@pytest.mark.parametrize("native", [True, False])
def test_a_target_of_another_kind_is_refused(monkeypatch, native):
    """Its handle would be taken for a cache's."""
    cache, calls = a_cache(monkeypatch, native)
    Streams(monkeypatch)
    quant = object.__new__(kv.KvFoldQuantCache)
    quant.handle, quant._bound, quant.close = ctypes.c_void_p(2), None, lambda: None
    for to in (quant, 7):
        with pytest.raises(TypeError):
            cache.evict(0, torch.zeros((HKV, CAPACITY)), 10, to=to)
    assert not calls


def test_more_rows_than_there_are_take_no_memory(monkeypatch):
    """The library's answer, not that of an allocation of n_keep indices."""
    for native in (True, False):
        cache, calls = a_cache(monkeypatch, native)
        monkeypatch.setattr(binding, "kvfold_evict_workspace_bytes", lambda handle, n_keep: 0 if not 1 <= n_keep <= CAPACITY else 1000)
        cache._lib.kvfold_cache_evict = lambda *a: -3
        monkeypatch.setattr(binding._native, "evict", lambda *a: None if a[9].numel() != HKV * a[3] else -3)
        streams = Streams(monkeypatch)
        with pytest.raises(kv.KvFoldError) as e:
            cache.evict(0, torch.zeros((HKV, CAPACITY)), 1 << 40)
        assert e.value.status == -3
        monkeypatch.undo()


def test_strides_of_dimensions_of_size_one_mean_nothing(monkeypatch):
    """One row, or one KV head, of any view may be appended; strides that count have to be alike."""
    calls, cache = [], object.__new__(kv.KvFoldQuantCache)
    cache.handle, cache._device, cache._hq, cache._hkv, cache._d = ctypes.c_void_p(1), 0, 4, HKV, D
    cache._bf16, cache._f32, cache.close, cache._stream = torch.bfloat16, torch.float32, lambda: None, lambda s: 0
    cache._lib = types.SimpleNamespace(kvfold_qcache_append=lambda *a: calls.append(a[4:7]) or 0)
    monkeypatch.setattr(binding, "_expect", lambda name, t, *a, **k: t.data_ptr())
    rows = torch.zeros((5, HKV, D), dtype=torch.bfloat16)
    one = torch.zeros(2000, dtype=torch.bfloat16)
    cache.append(0, rows[:1], one.as_strided((1, HKV, D), (999, D, 1)), pos_offset=0)
    cache.append(0, one.as_strided((1, HKV, D), (999, D, 1)), rows[:1], pos_offset=0)
    cache._hkv = 1
    cache.append(0, rows[:, :1], one.as_strided((5, 1, D), (HKV * D, 7, 1)), pos_offset=0)
    cache.append(0, one.as_strided((1, 1, D), (5, 7, 1)), rows[:1, :1], pos_offset=0)
    assert [a[2] for a in calls] == [1, 1, 5, 1] and calls[2][0] == HKV * D
    assert all(s >= 0 and s % 8 == 0 for a in calls for s in a[:2]) and calls[0][1] == calls[1][1] == D
    cache._hkv = HKV
    for k, v in ((rows[:2], one.as_strided((2, HKV, D), (3 * D, D, 1))), (rows[:1], one.as_strided((1, HKV, D), (HKV * D, 2 * D, 1))),
                 (one.as_strided((1, HKV, D), (HKV * D, D, 2)), one.as_strided((1, HKV, D), (HKV * D, D, 2)))):
        with pytest.raises(ValueError):
            cache.append(0, k, v, pos_offset=0)
