"""Blocks that go on behind a cut or a fork inside a page wider than the block, and reads on another stream."""
import pytest
import torch

import paper_2505_18610_amd as kq
from test_gpu_moves import exported, like, seq_map
from test_gpu_tree import D, MIXED, cached, make

pytestmark = pytest.mark.gpu


def new(batch, hq, hkv, int16=False):
    cfg = kq.KvqConfig(1, batch, hq, hkv, 1024, page_tokens=64, policy=kq.KVQ_POLICY_PAPER)
    arena = torch.full((kq.kvq_arena_bytes(cfg, 16 * 64 * batch * hkv * 576),), 0xff, dtype=torch.uint8, device="cuda")
    c = kq.KvqCache(cfg, [1 << 40], [2], arena=arena)
    if int16:
        c.kvq_cache_set_option(kq.KVQ_OPT_TIER16, kq.KVQ_TIER16_INT16)
    return c


@pytest.mark.parametrize("int16", [False, True])
@pytest.mark.parametrize("cut,width", [(129, 8), (150, 8), (160, 8), (193, 16), (230, 16), (100, 2)])
@pytest.mark.parametrize("way", ["append", "steps", "batch"])
@pytest.mark.parametrize("move", ["truncate", "fork"])
def test_appends_behind_a_cut(int16, cut, width, way, move):
    """The block is the one that appends of explicit widths make, and attends like it."""
    g = torch.Generator("cuda").manual_seed(cut)
    k, v = (torch.randn(2, 2, 320, D, generator=g, device="cuda").half() for _ in range(2))
    q = torch.randn(2, 8, D, generator=g, device="cuda").half()
    c, want = new(2, 8, 2, int16), new(2, 8, 2, int16)
    tiers, at = [(128, 2), (64, 8), (100, 16)], 0
    for n, bits in tiers:
        c.kvq_quantize_append(0, k[:, :, at:at + n].contiguous(), v[:, :, at:at + n].contiguous(), bits)
        m = min(n, cut - at)
        if m > 0:
            want.kvq_quantize_append(0, k[:, :, at:at + m].contiguous(), v[:, :, at:at + m].contiguous(), bits)
        at += n
    if move == "truncate":
        c.kvq_cache_truncate(0, cut)
    else:
        d = new(2, 8, 2, int16)
        kq.kvq_cache_fork(d, c, 0, n_tokens=cut)
        c = d
    more = 70 if way == "append" else 20
    nk, nv = (x[:, :, 320 - more:].contiguous() for x in (k, v))
    outs = [torch.empty(2, 8, D, device="cuda") for _ in range(2)]
    if way == "append":
        c.kvq_quantize_append(0, nk, nv)
    else:
        for i in range(more):
            one = nk[:, :, i:i + 1].contiguous(), nv[:, :, i:i + 1].contiguous()
            if way == "steps":
                c.kvq_append_decode_attention(0, *one, q, outs[0])
            else:
                kq.kvq_append_decode_attention_batch([c], 0, [one[0]], [one[1]], [q], [outs[0]])
    want.kvq_quantize_append(0, nk, nv, width)
    assert exported(c) == exported(want)
    for x, o in ((c, outs[0]), (want, outs[1])):
        x.kvq_cache_set_option(kq.KVQ_OPT_DETERMINISTIC, 1)
        x.kvq_decode_attention(0, q, o)
    assert torch.isfinite(outs[0]).all() and float((outs[0] - outs[1]).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_read_on_another_stream(dtype):
    """Behind a fork and a cut of the same stream: what is read is what they have left, all of it."""
    c, lam, g = make(2, 4, 2, MIXED)
    d = like(c, 2)
    m = seq_map([1, 0])
    k, v = (torch.full((2, 2, 400, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    kq.kvq_cache_fork(d, c, 0, m, stream=s)
    d.kvq_cache_truncate(0, 400, stream=s)
    d.kvq_cache_read(0, 0, k, v, stream=s)
    s.synchronize()
    for got, want in zip((k, v), cached(c)):
        want = want[[1, 0]][:, :, :400]
        # code * S + Z in 32 bits, rounded once more to fp16
        step = 2.0 ** -24 + (2.0 ** -11 if dtype == torch.float16 else 0)
        assert bool(((got.double() - want).abs() <= step * want.abs() + 2.0 ** -25).all())
