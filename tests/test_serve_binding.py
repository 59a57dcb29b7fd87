"""What the binding of the paged cache hands to the library, on the CPU: the library's own host-side queries, a stand-in for its launch."""
import os

import pytest
import torch

from paper_2508_04711_amd import binding


class OnDevice(torch.Tensor):
    """A tensor in host memory that says it is on device 0."""
    is_cuda = True

    def get_device(self):
        return 0


def _on_device(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def calls(monkeypatch):
    """The attention calls that reach the library, as (new rows, workspace bytes given, workspace bytes needed)."""
    if not os.path.exists(binding.library_path()):
        from paper_2508_04711_amd import build
        build.build()
    lib, seen = binding.load_library(), []

    class Library:
        hstu_paged_attn_workspace_bytes = staticmethod(lib.hstu_paged_attn_workspace_bytes)
        hstu_attn_status_string = staticmethod(lib.hstu_attn_status_string)

        @staticmethod
        def hstu_paged_attn_fwd(params, cache, bias, q, q_stride, off, o, ws, size, stream):
            need = lib.hstu_paged_attn_workspace_bytes(params, cache)
            seen.append((binding._PAGED_PARAMS.unpack(params)[6], size, need))
            return -2 if need == 0 else (0 if need <= 256 or size >= need else -4)
    monkeypatch.setattr(binding, "load_library", lambda: Library)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream_of", lambda index: 0)
    return seen


def _cache(batch=5, pages=80, ps=64, d=128):
    return binding.HstuPagedCache(_on_device(pages, 4, ps, d), _on_device(pages, 4, ps, d),
                                  _on_device(batch, pages, dtype=torch.int32), _on_device(batch, dtype=torch.int32))


def _call(cache, rows, max_len=100, **kw):
    off = _on_device(cache.batch + 1, dtype=torch.int32)
    return binding.hstu_paged_attn_fwd(_on_device(rows, 4, 128), cache, off, max_len, 0.1, **kw)


def test_a_call_between_query_and_launch_does_not_change_the_workspace(calls, monkeypatch):
    """Another thread's call with another number of rows may run wherever the interpreter switches, here inside the store of what
    the query gave: both calls get the workspace that they need."""
    cache, store = _cache(), binding.HstuPagedCache.__setattr__
    others = [5, 600]

    def interrupted(self, name, value):
        store(self, name, value)
        if name == "_need" and others:
            _call(self, others.pop(0))
    monkeypatch.setattr(binding.HstuPagedCache, "__setattr__", interrupted)
    _call(cache, 600)
    _call(cache, 5)
    assert sorted(rows for rows, _, _ in calls) == [5, 5, 600, 600]
    assert all(size == need > 256 for _, size, need in calls), calls


@pytest.mark.parametrize("bad", [dict(max_len=0), dict(alpha=float("inf")), dict(out_dtype=torch.bfloat16)])
def test_a_refused_call_leaves_nothing_behind(calls, bad):
    """The library's query gives 0 for a call that it refuses: the next call of the same shape asks again."""
    dtype = torch.float32 if "out_dtype" in bad else torch.bfloat16
    cache = binding.HstuPagedCache(*(_on_device(80, 4, 64, 128, dtype=dtype) for _ in range(2)),
                                   _on_device(5, 80, dtype=torch.int32), _on_device(5, dtype=torch.int32))
    off, q = _on_device(6, dtype=torch.int32), _on_device(7, 4, 128, dtype=dtype)
    with pytest.raises(binding.HstuError) as e:
        binding.hstu_paged_attn_fwd(q, cache, off, bad.get("max_len", 100), bad.get("alpha", 0.1), out_dtype=bad.get("out_dtype"))
    assert e.value.status == -2
    binding.hstu_paged_attn_fwd(q, cache, off, 100, 0.1)
    assert calls[-1][0] == 7 and calls[-1][1] == calls[-1][2] > 256
