"""What the binding refuses before the library sees an address, on the CPU: memory of the wrong side, types and shapes."""
import os
import types

import numpy as np
import pytest
import torch

from paper_2307_02628_amd import _build, skd


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(skd.LIB_PATH):
        _build.build(force=True)


class NoCalls:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


def decoder(io):
    d = object.__new__(skd.Decoder)
    d.cfg, d._lib, d._h = types.SimpleNamespace(io_on_device=io, batch=3, vocab=50), NoCalls(), None
    return d


def test_columns_in_the_wrong_memory():
    host = torch.zeros(4, 3, dtype=torch.int32)
    for tokens in (host, host.numpy(), host.long(), host[:, :2], host.t(), host[0], host[0].numpy()):
        with pytest.raises(ValueError):
            decoder(1).decode_chunk_rc(5, tokens)
    for tokens in (torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32), np.zeros(3), torch.zeros(2, 4, dtype=torch.int32)):
        with pytest.raises(ValueError):
            decoder(0).decode_chunk_rc(5, tokens)


class OnDevice(torch.Tensor):
    is_cuda = True


def device(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def test_draws_in_the_wrong_memory():
    good = dict(u=device(3), temperature=device(3), top_k=device(3, dtype=torch.int32), top_p=device(3), min_p=device(3), tokens_out=device(3, dtype=torch.int32),
                logits_out=device(3, 50))
    with pytest.raises(AssertionError, match="skd_logits_sample_rows was called"):
        decoder(1).logits_sample_rows_device(**good)
    with pytest.raises(AssertionError, match="skd_logits_sample_rows was called"):
        decoder(1).logits_sample_rows_device(1 << 20, tokens_out=1 << 21)
    for name, t in good.items():
        other = torch.int32 if t.dtype == torch.float32 else torch.int64
        for bad in (torch.zeros(t.shape, dtype=t.dtype), np.zeros(t.shape), device(*t.shape, dtype=other), device(4, *t.shape[1:], dtype=t.dtype)):
            with pytest.raises(ValueError):
                decoder(1).logits_sample_rows_device(**{**good, name: bad})


def test_strides_of_dense_tokens():
    """Dimensions of one element may have any stride."""
    cache = skd.KvCache(torch.zeros(2, 32 * 256, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32), 1, 128, 32)
    place = lambda t, heads: cache._rows_of(skd.KvChunk(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), len(t), len(t), 0), heads, t, "torch.bfloat16")  # noqa: E731
    x = torch.zeros(1, 5, 128, dtype=torch.bfloat16)
    assert place(x.transpose(0, 1), 1) == (x.data_ptr(), 128)
    wide = torch.zeros(7, 1001, dtype=torch.bfloat16)
    assert place(wide[3:4, 16:144], 1) == (wide[3:4, 16:].data_ptr(), 128)
    assert place(wide[3:4, 16:528].view(1, 4, 128), 4)[1] == 512
    assert place(wide[:, 16:144], 1)[1] == 1001                       # (refused by the library: not a multiple of 8)
    two = torch.zeros(2, 5, 128, dtype=torch.bfloat16)
    for bad, heads in ((two.transpose(0, 1), 2), (wide[:, 16:272:2], 1), (two, 3), (wide[:5, :640].view(5, 5, 128).transpose(1, 0), 5)):
        with pytest.raises(ValueError):
            place(bad, heads)
