"""CPU-only: the binding of attention takes tensors of the current GPU alone, and says so before it calls the library.  Another
GPU's tensors are stood in for by objects that answer what the binding asks of them."""
import pytest
import torch

from paper_2407_01781_amd import binding as B


class On:
    """A tensor of a GPU, as far as the binding looks at it."""
    is_cuda = True

    def __init__(self, device, shape, dtype):
        self.device, self.dtype, self.shape = torch.device("cuda", device), dtype, torch.Size(shape)

    def get_device(self):
        return self.device.index

    def stride(self, i=None):
        all_ = tuple(int(torch.Size(self.shape[d + 1:]).numel()) for d in range(len(self.shape)))
        return all_ if i is None else all_[i]

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Seqs:
    rows, batch_size, _h = 6, 2, 1 << 20


class Reached(Exception):
    pass


@pytest.fixture(autouse=True)
def _no_library(monkeypatch):
    """Device 0 is current; a call that comes through to the library or to new memory ends there."""
    def reached(*_):
        raise Reached
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_new_heads", reached)
    monkeypatch.setattr(B, "_check", reached)
    monkeypatch.setattr(B, "_stream", lambda: None)

    class Lib:
        def __getattr__(self, name):
            return reached
    monkeypatch.setattr(B, "lib", Lib())


def _cache():
    return B.KVCache(On(0, (4, 1, 16, 32), torch.bfloat16), On(0, (4, 1, 16, 32), torch.bfloat16))


CALLS = {
    "attention_fwd": lambda on: B.attention_fwd(Seqs, on("q", (6, 2, 32)), on("k", (6, 1, 32)), on("v", (6, 1, 32))),
    "attention_bwd": lambda on: B.attention_bwd(Seqs, on("q", (6, 2, 32)), on("k", (6, 1, 32)), on("v", (6, 1, 32)), on("out", (6, 2, 32)), on("lse", (2, 6), torch.float32),
                                                on("grad_out", (6, 2, 32)), grad_lse=on("grad_lse", (2, 6), torch.float32)),
    "cache_write": lambda on: B.cache_write(_cache(), on("table", (2, 3), torch.int32), on("start", (2,), torch.int32), on("k", (2, 1, 32)), on("v", (2, 1, 32))),
    "attention_step": lambda on: B.attention_step(_cache(), on("table", (2, 3), torch.int32), on("lengths", (2,), torch.int32), on("q", (2, 2, 32)), out=on("out", (2, 2, 32)))}
NAMES = {"attention_fwd": "q k v", "attention_bwd": "q k v out lse grad_out grad_lse", "cache_write": "table start k v", "attention_step": "table lengths q out"}


@pytest.mark.parametrize("call", list(CALLS))
def test_the_current_gpu(call, monkeypatch):
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: On(0, shape, dtype))
    with pytest.raises(Reached):
        CALLS[call](lambda name, shape, dtype=torch.bfloat16: On(0, shape, dtype))


@pytest.mark.parametrize("call,name", [(c, n) for c in CALLS for n in NAMES[c].split()])
def test_another_gpu(call, name, monkeypatch):
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: On(0, shape, dtype))
    with pytest.raises(AssertionError, match=name if name != "table" else "current GPU"):
        CALLS[call](lambda n, shape, dtype=torch.bfloat16: On(int(n == name), shape, dtype))
