"""The cache object of the binding holds addresses: nothing that it was made from can be exchanged behind its back.  On the CPU, with the checks for a
GPU taken out and the calls of the library caught before they are made."""
import pytest
import torch

from paper_2403_02352_amd import binding

E4M3 = torch.float8_e4m3fn


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(binding, "_one_device", lambda first, *ts: first.device)
    monkeypatch.setattr(binding, "_check", lambda *ts: None)
    monkeypatch.setattr(binding, "_serve", lambda fn, dev, *args: made.append((fn.__name__, args)))
    return made


def empty(kind, n_pages=3):
    return binding.PagedCache.empty(n_pages, 2, 16, 64, E4M3 if kind == "e4m3" else torch.bfloat16, device="cpu")


def each_call(cache):
    """The three calls over one sequence of four tokens."""
    rows = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    args = (torch.zeros((1, 1), dtype=torch.int32), torch.tensor([4], dtype=torch.int32), torch.tensor([0, 4], dtype=torch.int32))
    yield lambda: binding.cache_write(cache, rows, rows, *args)
    yield lambda: binding.cache_read(cache, *args, out=(rows, rows.clone()))
    yield lambda: binding.attention_paged(rows, cache, *args)


@pytest.mark.parametrize("kind", ["same", "e4m3"])
@pytest.mark.parametrize("name", ["K", "V", "K_scale", "V_scale", "e4m3", "device", "n_pages", "kv_heads", "page_size", "d_h"])
def test_attributes_are_read_only(calls, kind, name):
    cache = empty(kind)
    held = getattr(cache, name)
    with pytest.raises(AttributeError):
        setattr(cache, name, getattr(empty(kind, 5), name))
    with pytest.raises(AttributeError):
        delattr(cache, name)
    assert getattr(cache, name) is held


@pytest.mark.parametrize("kind,names", [("same", ["K", "V"]), ("e4m3", ["K", "V", "K_scale", "V_scale"])])
def test_a_tensor_that_has_moved_is_refused(calls, kind, names):
    for name in names:
        cache = empty(kind)
        for call in each_call(cache):
            call()
        assert len(calls) == 3
        calls.clear()
        t = getattr(cache, name)
        # (larger, in memory of its own: what the tensor lay in before is free)
        t.set_(torch.zeros((30,) + tuple(t.shape[1:]), dtype=torch.uint8).view(t.dtype) if t.element_size() == 1 else torch.zeros((30,) + tuple(t.shape[1:]), dtype=t.dtype))
        for call in each_call(cache):
            with pytest.raises(ValueError):
                call()
        assert not calls


def test_a_cache_passes_what_it_holds(calls):
    cache = empty("e4m3")
    for call in each_call(cache):
        call()
    assert [n for n, _ in calls] == ["atp_cache_write", "atp_cache_read", "atp_attention_paged"]
    c = calls[0][1][0]
    assert (c.K, c.V, c.K_scale, c.V_scale) == tuple(t.data_ptr() for t in (cache.K, cache.V, cache.K_scale, cache.V_scale))
    assert (c.n_pages, c.kv_heads, c.page_size, c.d_h, c.type) == (3, 2, 16, 64, binding.ATP_CACHE_E4M3) == (cache.n_pages, cache.kv_heads, cache.page_size, cache.d_h, 1)
