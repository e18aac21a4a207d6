"""The binding of the paged cache of 8-bit floating point takes tensors of the types that the library reads, on a device, and nothing that merely has their
size.  The library is replaced: what gets as far as a call is recorded, nothing is launched."""
import pytest
import torch

import paper_2505_18610_amd as kq
from paper_2505_18610_amd import binding
from test_binding_types_cpu import lib, tensor  # noqa: F401

I32, F16, F32 = torch.int32, torch.float16, torch.float32


def cache(codes=torch.uint8, words=I32, device=True, shape=(3, 2, 1, 2, 4096)):
    return kq.KvqPaged8(tensor(*shape, dtype=codes, device=device), tensor(3, 2, 2, dtype=words, device=device))


def batch(table=I32, lengths=I32, begin=I32, device=True, n=2):
    return kq.KvqPaged8Batch(tensor(2, 4, dtype=table, device=device), tensor(n, dtype=lengths, device=device), tensor(3, dtype=begin, device=device), 3)


def append(k=F16, v=F16, cs=F32, width=128, rows=5, device=True, heads=2):
    cache().kvq_paged8_append(batch(), tensor(5, heads, 128, dtype=k, device=device), tensor(5, 2, 128, dtype=v), tensor(rows, width, dtype=cs))


def read(k=F16, v=F16, device=True, channels=128):
    cache().kvq_paged8_read(batch(), tensor(5, 2, channels, dtype=k, device=device), tensor(5, 2, 128, dtype=v))


def attend(q=F16, out=F16, lse=F32, ws=torch.uint8, device=True, ws_device=True, rows=5):
    cache().kvq_paged8_attention(batch(), tensor(5, 4, 128, dtype=q, device=device), tensor(rows, 4, 128, dtype=out), lse=tensor(4, 5, dtype=lse),
                                 workspace=tensor(64, dtype=ws, device=ws_device))


def diff(q=F16, out=F16, lam=F32, weight=F32, heads=4, device=True, ws_device=True):
    cache().kvq_paged8_diff_attention(batch(), tensor(5, 4, 128, dtype=q, device=device), tensor(heads, dtype=lam), tensor(5, 4, 128, dtype=out),
                                      norm_weight=tensor(128, dtype=weight), workspace=tensor(64, dtype=torch.uint8, device=ws_device))


@pytest.mark.parametrize("call,good", [(append, [{}, dict(width=64)]), (read, [{}, dict(k=F32, v=F32)]), (attend, [{}, dict(out=F32)]), (diff, [{}, dict(out=F32)])])
def test_what_is_taken(lib, call, good):  # noqa: F811
    for x in good:
        call(**x)
    assert lib.calls == ["kvq_paged8_" + {"attend": "attention", "diff": "diff_attention"}.get(call.__name__, call.__name__)] * len(good)


@pytest.mark.parametrize("call,bad", [(c, x) for c, xs in (
    (cache, [dict(codes=I32), dict(words=F32), dict(words=torch.int64), dict(device=False), dict(shape=(3, 2, 1, 2, 2048)), dict(shape=(2, 2, 1, 2, 4096))]),
    (batch, [dict(table=torch.int64), dict(lengths=torch.int64), dict(begin=F32), dict(device=False), dict(n=3)]),
    (append, [dict(k=torch.bfloat16), dict(v=torch.bfloat16), dict(k=F32), dict(cs=F16), dict(width=96), dict(rows=4), dict(device=False), dict(heads=3)]),
    (read, [dict(k=torch.bfloat16, v=torch.bfloat16), dict(v=F32), dict(device=False), dict(channels=64)]),
    (attend, [dict(q=torch.bfloat16), dict(q=F32), dict(out=torch.bfloat16), dict(lse=F16), dict(device=False), dict(ws_device=False), dict(rows=4)]),
    (diff, [dict(q=torch.bfloat16), dict(out=torch.bfloat16), dict(lam=F16), dict(weight=F16), dict(heads=5), dict(device=False), dict(ws_device=False)]),
) for x in xs])
def test_what_is_not(lib, call, bad):  # noqa: F811
    with pytest.raises((AssertionError, ValueError)):
        call(**bad)
    assert lib.calls == []


def test_strides(lib):  # noqa: F811
    """Rows of any strides whose channels follow one another; what the library takes as one run of memory is one."""
    wide = tensor(5, 6, 256)
    cache().kvq_paged8_append(batch(), wide[:, :2, 128:], wide[:, 4:, :128])
    assert lib.calls == ["kvq_paged8_append"]
    for k in (wide[:, :2, ::2], tensor(5, 128, 2).transpose(1, 2)):
        with pytest.raises(AssertionError):
            cache().kvq_paged8_append(batch(), k, k)
    with pytest.raises(AssertionError):  # (every other angle)
        cache().kvq_paged8_append(batch(), wide[:, :2, 128:], wide[:, 4:, :128], tensor(5, 256, dtype=F32)[:, ::2])
    with pytest.raises(AssertionError):
        kq.KvqPaged8Batch(tensor(2, 8, dtype=I32)[:, ::2], tensor(2, dtype=I32))
    with pytest.raises(AssertionError):
        kq.KvqPaged8Batch(tensor(2, 8, dtype=I32), tensor(4, dtype=I32)[::2])
    assert lib.calls == ["kvq_paged8_append"] and binding._paged8_rows(wide[:, :2, 128:], 5, 2)._obj.row_stride == 6 * 256
