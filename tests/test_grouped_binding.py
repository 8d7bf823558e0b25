"""The binding of the separate products on the host: calls that enqueue nothing."""
import pytest
import torch

from paper_2509_17863_amd import eaas

BF16, I8, F32 = torch.bfloat16, torch.int8, torch.float32


@pytest.mark.parametrize("E", [1, 8])
def test_an_empty_batch_with_its_routing(E):
    """T = 0: the routing's arrays have one element at least, and no call minds."""
    T, k, H, I = 0, 2, 128, 256
    z = lambda *shape, dtype=BF16: torch.zeros(shape, dtype=dtype)  # noqa: E731
    r = eaas.alloc_routing(T, k, E, device="cpu")
    off, take = r["offsets"], dict(perm=r["perm"], k=k, stream=0)
    ws = eaas.alloc_grouped_workspace(0, E, 2 * I, H, device="cpu")
    eaas.eaas_grouped_matmul(z(0, H), off, z(E, 2 * I, H), z(0, 2 * I), ws, **take)
    eaas.eaas_grouped_matmul_int8(z(0, H, dtype=I8), z(0, dtype=F32), off,
                                  z(E, 2 * I, H, dtype=I8), z(E, 2 * I, dtype=F32), z(0, 2 * I),
                                  ws, **take)
    eaas.eaas_grouped_matmul_dw(z(0, 2 * I), z(0, H), off, z(E, 2 * I, H, dtype=F32), ws,
                                accumulate=True, **take)
    eaas.eaas_grouped_matmul_dx(z(0, 2 * I), off, z(E, 2 * I, H), z(0, H), ws, stream=0)
    eaas.eaas_quantize_rows_int8(z(0, H), z(0, H, dtype=I8), z(0, dtype=F32), stream=0)
    n = off[E:]
    eaas.eaas_swiglu(z(0, 2 * I), z(0, I), n_rows=n, stream=0)
    eaas.eaas_swiglu_int8(z(0, 2 * I), z(0, I, dtype=I8), z(0, dtype=F32), n_rows=n, stream=0)
    eaas.eaas_swiglu_backward(z(0, 2 * I), z(0, I), z(0, 2 * I), n_rows=n, stream=0)
    eaas.eaas_unpermute_combine_backward(z(0, H), z(0, H, dtype=F32), r, z(0, k, dtype=F32),
                                         z(0, H), z(0, k, dtype=F32), E, stream=0)
    with pytest.raises(ValueError):  # (the type still counts)
        eaas.eaas_grouped_matmul(z(0, H), off, z(E, 2 * I, H), z(0, 2 * I), ws,
                                 perm=r["perm"].long(), k=k, stream=0)


def test_the_current_stream_without_the_handle_function(monkeypatch):
    class Stream:
        cuda_stream = 42

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 40 + device,
                        raising=False)
    assert eaas._stream(None) == 43
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream)
    assert eaas._stream(None) == 42
    assert eaas._stream(7) == 7 and eaas._stream(Stream) == 42
