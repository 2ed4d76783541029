"""Which stream the binding hands to the library; without a device."""
from types import SimpleNamespace

import torch

from paper_2410_05076_b200 import binding


def test_a_status_answers_for_the_stream_of_the_contexts_device(monkeypatch):
    """The block-sparse and page calls go to the current stream of the context's device, whichever device is current; so
    does the question what became of them."""
    asked = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: SimpleNamespace(cuda_stream=100 + (0 if device is None else device)))
    td = binding.Tidal.__new__(binding.Tidal)
    td.lib = SimpleNamespace(tidal_device_status=lambda ctx, stream: asked.append(stream) or binding.OK)
    td.ctx, td.device = binding.C.c_void_p(), 3
    assert td.device_status() == binding.OK and asked == [103]
