"""A paged cache's views are on the device that holds it, whichever is current when they are asked for (no GPU: the
library and torch's device queries are stood in for)."""
import types

import torch


def test_views_name_the_device_of_the_cache(monkeypatch):
    import paper_2403_18647_gb300 as sd
    asked = []
    monkeypatch.setattr(sd, "_lib", lambda: types.SimpleNamespace(sdsat_kv_create_paged=lambda *a: 0, sdsat_kv_destroy=lambda *a: None))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch, "as_tensor", lambda data, device=None: asked.append((data, torch.device(device))) or torch.zeros(1, dtype=torch.int16))
    kv = sd.PagedKV(types.SimpleNamespace(handle=None, shape=types.SimpleNamespace(n_layers=2, n_heads=4, head_dim=64)), 2, 100, 7)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    kv.pages = lambda: (64, 128, 7, 2)
    kv.info = lambda: (256, 512, 1024, 2, 100)
    for view, address, shape in (("table", 64, (2, 2)), ("refs", 128, (7,)), ("lens", 1024, (2,)), ("k", 256, (2, 7, 4, 64, 64)),
                                 ("v", 512, (2, 7, 4, 64, 64))):
        getattr(kv, view)
        data, device = asked[-1]
        assert device == torch.device("cuda", 3), view
        assert data.__cuda_array_interface__["data"] == (address, False) and data.__cuda_array_interface__["shape"] == shape
        assert data.owner is kv
