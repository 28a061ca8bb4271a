"""The binding's side of the serving calls, without a GPU."""
import ctypes

import pytest
import torch

from paper_2609_34866_gb300 import binding


def _any_device(monkeypatch):
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None, name="tensor": None if t is None else t.data_ptr())


def test_tensors_of_a_cache_cannot_be_exchanged(monkeypatch):
    """The calls go by addresses that were taken once: another tensor in their place would leave them behind."""
    _any_device(monkeypatch)
    cache = binding.KvCache(2, 64, 8, 16, 3, device="cpu")
    want = {"k_codes": cache.desc.k_codes, "v_codes": cache.desc.v_codes, "k_scales": cache.desc.k_scales, "v_scales": cache.desc.v_scales}
    for name, address in want.items():
        t = getattr(cache, name)
        assert t.data_ptr() == address
        with pytest.raises(AttributeError):
            setattr(cache, name, torch.zeros_like(t))
        assert getattr(cache, name) is t
    cache.k_scales += 2.0  # in place: the same tensor
    assert cache.k_scales.data_ptr() == want["k_scales"] and bool((cache.k_scales == 2).all())
    given = torch.ones((3, 2, 16, 64), dtype=torch.uint8)
    assert binding.KvCache(2, 64, 8, 16, 3, device="cpu", v_codes=given).v_codes is given


def test_current_stream_without_torch_internals(monkeypatch):
    """The handle of the current stream, from torch's short way if this torch has it, else from its public one."""
    class Stream:
        cuda_stream = 1234

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream())
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 1000 + device)
    assert binding._stream(None) == 1003
    monkeypatch.setattr(binding, "_raw_stream", None)
    assert binding._stream(None) == 1234
    assert binding._stream(Stream()) == 1234 and binding._stream(77) == 77


def test_numbers_of_tokens_past_64_bits_are_refused():
    """n_tokens * n_q_heads is bounded whatever the product does in 64 bits."""
    from paper_2609_34866_gb300 import build
    build.build()
    L = binding.lib()
    cache = binding._KvCacheDesc(2, 64, 8, 16, 4, 1 << 20, 1 << 20, 1 << 20, 1 << 20)
    fake = ctypes.c_void_p(1 << 20)  # never dereferenced
    for n in (1 << 30, 1 << 60, 1 << 62, (1 << 62) + 1, (1 << 63) - 1):
        assert L.jab_kv_attention_workspace_size(ctypes.byref(cache), 2, n, 4, 1, 64, 0) == 0
        assert L.jab_kv_attention(ctypes.byref(cache), 2, n, 4, fake, 0, 256, fake, fake, 4, fake, 1, 64, 0, 0, 0.0, fake, 256, None, fake,
                                  (1 << 64) - 1, None) == 2  # JAB_ERR_UNSUPPORTED
