"""The binding of prompt and tree attention, forks and read-back takes fp16 (and int32) tensors on a device and nothing that merely has their size.
The library is replaced: what gets as far as a call is recorded, nothing is launched."""
import os

import pytest
import torch

import paper_2505_18610_amd as kq
from paper_2505_18610_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")


class OnDevice(torch.Tensor):  # host memory that says that it is a device's
    is_cuda = True


def tensor(*shape, dtype=torch.float16, device=True):
    t = torch.zeros(*shape, dtype=dtype)
    return torch.Tensor._make_subclass(OnDevice, t) if device else t


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or kq.KVQ_OK


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    return lib


def prompt(q=torch.float16, k=torch.float16, v=torch.float16, out=torch.float16, lse=torch.float32, device=True):
    kq.kvq_prompt_attention(tensor(5, 4, 128, dtype=q, device=device), tensor(5, 2, 128, dtype=k), tensor(5, 2, 128, dtype=v), tensor(5, 4, 128, dtype=out), [0, 5],
                            lse=tensor(4, 5, dtype=lse))


class Cache(kq.KvqCache):
    def __init__(self, lib):
        self.lib, self.cfg, self.handle = lib, kq.KvqConfig(1, 1, 4, 2, 64, page_tokens=32), None


def tree(lib, q=torch.float16, k=torch.float16, v=torch.float16, out=torch.float16, mask=torch.int32, device=True):
    Cache(lib).kvq_tree_attention(0, tensor(1, 4, 3, 128, dtype=q), tensor(1, 2, 3, 128, dtype=k), tensor(1, 2, 3, 128, dtype=v),
                                  tensor(3, 1, dtype=mask, device=device), tensor(1, 4, 3, 128, dtype=out))


def read(lib, out=torch.float16, device=True):
    Cache(lib).kvq_cache_read(0, 0, *(tensor(1, 2, 3, 128, dtype=out, device=device) for _ in range(2)))


def fork(lib, seq_map=torch.int32, device=True):
    kq.kvq_cache_fork(Cache(lib), Cache(lib), 0, tensor(1, dtype=seq_map, device=device))


def test_what_is_taken(lib):
    prompt()
    prompt(out=torch.float32)
    tree(lib)
    tree(lib, out=torch.float32, mask=torch.uint32)
    read(lib)
    read(lib, out=torch.float32)
    fork(lib)
    assert len(lib.calls) == 7


@pytest.mark.parametrize("call,bad", [
    (prompt, dict(q=torch.bfloat16)), (prompt, dict(k=torch.int16)), (prompt, dict(v=torch.bfloat16)), (prompt, dict(out=torch.bfloat16)),
    (prompt, dict(out=torch.float64)), (prompt, dict(out=torch.int32)), (prompt, dict(lse=torch.int32)), (prompt, dict(lse=torch.float16)), (prompt, dict(device=False)),
    (tree, dict(q=torch.bfloat16)), (tree, dict(k=torch.bfloat16)), (tree, dict(v=torch.int16)), (tree, dict(out=torch.bfloat16)), (tree, dict(out=torch.int32)),
    (tree, dict(mask=torch.float32)), (tree, dict(mask=torch.int64)), (tree, dict(device=False)), (read, dict(out=torch.bfloat16)), (read, dict(out=torch.float64)),
    (read, dict(out=torch.int32)), (read, dict(device=False)), (fork, dict(seq_map=torch.float32)), (fork, dict(seq_map=torch.int64)), (fork, dict(device=False))])
def test_what_is_refused(lib, call, bad):
    with pytest.raises(AssertionError):
        call(**bad) if call is prompt else call(lib, **bad)
    assert not lib.calls
