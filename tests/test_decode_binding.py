"""The compiled marshalling of a decoding step's calls refuses, before the library sees them, what is no tensor, tensors in host
memory and a wrong number of arguments; each as an exception of the binding's own kinds."""
import os

import pytest
import torch


@pytest.fixture(scope="module")
def qii():
    from paper_2601_22813_amd import binding, build
    if not (os.path.exists(binding.LIB_PATH) and os.path.exists(binding.DECODE_PATH)):
        build.build(force=True)
    return binding


def test_host_memory_is_refused(qii):
    module = qii._decode()
    x, n = torch.zeros((2, 2, 16)), torch.zeros(2, dtype=torch.int32)
    cache = qii.KVCache.empty(qii.KV_BF16, 2, 2, 16, 16, device="cpu")
    pages = torch.zeros((2, 1), dtype=torch.int32)
    calls = [lambda: module.rotary(x, n, torch.zeros((4, 2, 8)), 0, x, False, 0),
             lambda: module.kv_append(x, x, n, cache, pages, n, None, 0, qii.RTN, 0),
             lambda: module.kv_read(cache, pages, n, x, x, n, 0),
             lambda: module.paged_attention(x, cache, pages, n, 4, 1.0, x, None, None, None, 0, None, 0, 0)]
    for call in calls:
        with pytest.raises(qii.QiiError, match="device memory"):
            call()


def test_what_is_no_tensor_is_refused(qii):
    module = qii._decode()
    with pytest.raises(TypeError):
        module.rotary(1, None, None, 0, None, False, 0)
    with pytest.raises(AttributeError):
        module.kv_append(None, None, None, 3, None, None, None, 0, 0, 0)
    cache = qii.KVCache(None, None)
    with pytest.raises(qii.QiiError):
        module.kv_read(cache, None, None, None, None, None, 0)
    for name, count in (("rotary", 7), ("kv_append", 10), ("kv_read", 7), ("paged_attention", 14)):
        with pytest.raises(TypeError, match=f"{count} arguments"):
            getattr(module, name)(*[None] * (count - 1))
