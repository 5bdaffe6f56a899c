"""What the allocating calls start on a device (a page list's first state, a workspace's zeros)
runs on the device that was named, whichever is the current one (no GPU: the device guard,
the allocation and the library's calls are stand-ins)."""
import types

import pytest
import torch


@pytest.fixture()
def api(monkeypatch):
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    now = [torch.device("cuda", 0)]

    class Guard:
        def __init__(self, device):
            self.device = torch.device(device)

        def __enter__(self):
            now.append(self.device)

        def __exit__(self, *_):
            now.pop()

    def empty(shape, dtype=None, device=None):
        device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        where = now[-1] if device.index is None else device
        return types.SimpleNamespace(shape=shape, dtype=dtype, device=where, is_cuda=True)

    calls = []

    def started(*args, **_):
        calls.append((now[-1], [t.device for t in flat(args) if hasattr(t, "is_cuda")]))

    def flat(args):
        for t in args:
            yield from ((t.page_table, t.free, t.n_free) if isinstance(t, _api.PageList) else (t,))

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    for name in ("tgvkv_pages_init", "tgvkv_cache_workspace_init", "tgvkv_workspace_init"):
        monkeypatch.setattr(_api, name, started)
    return types.SimpleNamespace(api=_api, calls=calls, now=now)


@pytest.mark.parametrize("device,index", [(None, 0), ("cuda", 0), ("cuda:0", 0), ("cuda:1", 1),
                                          (torch.device("cuda", 3), 3)])
def test_what_an_allocation_starts_runs_on_its_device(api, device, index):
    a = api.api
    desc = a.make_desc(1, 4, 2, 64, 64, 32, 8)
    cache = a.make_cache_desc(2, 8, 2, 64, 16, 8, 4)
    for call in (lambda: a.alloc_pages(cache, device), lambda: a.new_cache_workspace(cache, device),
                 lambda: a.new_workspace(desc, device)):
        api.calls.clear()
        call()
        (current, tensors), = api.calls
        assert current == torch.device("cuda", index)
        assert tensors and all(d == current for d in tensors)
        assert api.now == [torch.device("cuda", 0)]        # as it was


def test_device_0_by_its_number_is_not_the_current_one(api):
    a = api.api
    api.now[0] = torch.device("cuda", 1)
    cache = a.make_cache_desc(2, 8, 2, 64, 16, 8, 4)
    for call in (a.alloc_pages, a.new_cache_workspace):
        for device, index in ((0, 0), (None, 1)):
            api.calls.clear()
            call(cache, device)
            (current, tensors), = api.calls
            assert current == torch.device("cuda", index) and all(d == current for d in tensors)
    for device, index in ((0, 0), (None, 1)):
        assert a.alloc_cache(cache, device).k.device == torch.device("cuda", index)


def test_other_devices(monkeypatch):
    from paper_2606_03075_gb300 import api as a
    cache = a.make_cache_desc(2, 8, 2, 64, 16, 8, 4)
    assert a.alloc_pages(cache, device="meta").free.device.type == "meta"    # nothing is started
    with pytest.raises(ValueError, match="CUDA"):
        a.new_cache_workspace(cache, device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        a.new_workspace(a.make_desc(1, 4, 2, 64, 64, 32, 8), device="cpu")
