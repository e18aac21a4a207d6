"""kvq_cache_fork, kvq_cache_truncate and kvq_cache_read: bit for bit against what the caches export."""
import math

import numpy as np
import pytest
import torch

import paper_2505_18610_amd as kq
from test_gpu_tree import D, cached, make

pytestmark = pytest.mark.gpu
MIXED = [(128, 2), (192, 4), (64, 8), (77, 16)]


def exported(c, layer=0, seqs=None):
    """All runs of a block as arrays by sequence: [(bits, codes, S, Z), ...] for K and V."""
    got = []
    for i, (t0, t1, bits) in enumerate(c.kvq_cache_describe(layer)[0]):
        for which in (kq.KVQ_WHICH_K, kq.KVQ_WHICH_V):
            arrays = [None if x is None else (x if seqs is None else x[seqs]) for x in c.kvq_cache_export_segment(layer, i, which)]
            got.append(((t0, t1, bits), *[None if x is None else x.tobytes() for x in arrays]))
    return got


def like(c, batch, layers=1, **kw):
    f = c.cfg
    cfg = kq.KvqConfig(layers, batch, f.n_q_heads // 1, f.n_kv_heads, kw.pop("max_tokens", f.max_tokens), page_tokens=f.page_tokens,
                       policy=kw.pop("policy", f.policy), group=f.group, window=kw.pop("window", 0))
    payload = kw.pop("payload", (f.max_tokens // f.page_tokens + 20) * f.page_tokens * batch * f.n_kv_heads * 576)
    arena = torch.full((kq.kvq_arena_bytes(cfg, payload),), 0xff, dtype=torch.uint8, device="cuda")
    d = kq.KvqCache(cfg, [kw.pop("budget", 1 << 50)] * layers, [2] * layers, arena=arena)
    if getattr(c, "_tier16", 0):
        d.kvq_cache_set_option(kq.KVQ_OPT_TIER16, kq.KVQ_TIER16_INT16)
    return d


def seq_map(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("int16", [False, True])
@pytest.mark.parametrize("page", [32, 64, 192])
@pytest.mark.parametrize("batch,to", [(3, [2, 0, 0, 1, 2]), (4, [3]), (1, [0, 0, 0]), (2, [1, 1])])
def test_fork_into_another_cache(int16, page, batch, to):
    tiers = [(192, 2), (384, 4), (192, 8), (77, 16)]
    c, lam, g = make(batch, 8, 2, tiers, page=page, int16=int16, reparam=True, group=64)
    d = like(c, len(to))
    for _ in range(2):  # the second time over the pages of the first
        free = d.kvq_cache_arena_free_bytes()
        kq.kvq_cache_fork(d, c, 0, seq_map(to))
        assert exported(d) == exported(c, seqs=to)
        assert d.kvq_cache_describe(0)[0] == c.kvq_cache_describe(0)[0]
    assert d.kvq_cache_arena_free_bytes() == free
    q = torch.randn(len(to), 8, D, generator=g, device="cuda").half()
    want, got = torch.empty(batch, 8, D, device="cuda"), torch.empty(len(to), 8, D, device="cuda")
    d.kvq_decode_attention(0, q, got)
    for b, p in enumerate(to):  # the factors went along
        c.kvq_decode_attention(0, q[b].expand(batch, -1, -1).contiguous(), want)
        assert float((want[p] - got[b]).abs().max()) < 2e-3


@pytest.mark.parametrize("to", [[1, 0, 2], [0, 0, 0], [2, 2, 1]])
@pytest.mark.parametrize("n", [-1, 461, 384, 400, 33])
def test_sequences_change_places_in_place(to, n):
    tiers = MIXED if n in (-1, 461, 384, 400) else [(200, 16)]
    c, lam, g = make(3, 8, 2, tiers)
    before = exported(c, seqs=to)
    free = c.kvq_cache_arena_free_bytes()
    values = cached(c)
    kq.kvq_cache_fork(c, c, 0, seq_map(to), n)
    if n in (-1, 461):
        assert exported(c) == before and c.kvq_cache_arena_free_bytes() == free
    else:
        for x, y in zip(cached(c), values):
            assert torch.equal(x, y[to][:, :, :n])


def test_fork_of_long_tables():
    """More pages than ride in the arguments of one launch, in place and into another cache."""
    c, lam, g = make(2, 4, 1, [(32 * 300, 2), (32 * 150, 4), (50, 16)], page=32)
    before = exported(c, seqs=[1, 0])
    kq.kvq_cache_fork(c, c, 0, seq_map([1, 0]))
    assert exported(c) == before
    d = like(c, 3)
    kq.kvq_cache_fork(d, c, 0, seq_map([1, 0, 1]))
    assert exported(d) == exported(c, seqs=[1, 0, 1])


def test_entries_beyond_the_sequences_are_the_nearest():
    c, lam, g = make(2, 4, 1, [(70, 8)])
    d = like(c, 4)
    kq.kvq_cache_fork(d, c, 0, seq_map([-5, 7, 2 ** 31 - 1, -2 ** 31]))
    assert exported(d) == exported(c, seqs=[0, 1, 1, 0])


def test_fork_without_a_map():
    c, lam, g = make(1, 4, 2, MIXED)
    d = like(c, 3)
    kq.kvq_cache_fork(d, c, 0)
    assert exported(d) == exported(c, seqs=[0, 0, 0])
    e = like(d, 3)
    kq.kvq_cache_fork(e, d, 0)
    assert exported(e) == exported(d)


def test_large_scales_are_known_in_the_fork():
    """The attention kernels take another path where a V scale is 256 or more: the mark goes along."""
    c, lam, g = make(1, 4, 1, [])
    k = torch.randn(1, 1, 96, D, generator=g, device="cuda").half()
    v = (torch.randn(1, 1, 96, D, generator=g, device="cuda") * 9000).half()
    c.kvq_quantize_append(0, k, v, 4)
    d = like(c, 1)
    kq.kvq_cache_fork(d, c, 0)
    q = torch.randn(1, 4, D, generator=g, device="cuda").half()
    a, b = torch.empty(1, 4, D, device="cuda"), torch.empty(1, 4, D, device="cuda")
    for x in (c, d):
        x.kvq_cache_set_option(kq.KVQ_OPT_DETERMINISTIC, 1)
    c.kvq_decode_attention(0, q, a)
    d.kvq_decode_attention(0, q, b)
    assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("bits", [2, 4, 8, 16])
@pytest.mark.parametrize("int16", [False, True])
@pytest.mark.parametrize("n", [0, 1, 7, 31, 32, 33, 50, 64, 95, 130, 159])
@pytest.mark.parametrize("way", ["truncate", "fork"])
def test_cut_and_grown_again(bits, int16, n, way):
    """Tokens behind a cut leave no trace, whatever they were, and the block grows on as if they had never been."""
    f = kq.KvqConfig(1, 2, 4, 2, 400, page_tokens=96, policy=kq.KVQ_POLICY_PAPER)
    g = torch.Generator("cuda").manual_seed(n)
    k, v = (torch.randn(2, 2, 230, D, generator=g, device="cuda").half() for _ in range(2))

    def new():
        arena = torch.full((kq.kvq_arena_bytes(f, 10 * 96 * 4 * 576),), 0xff, dtype=torch.uint8, device="cuda")
        c = kq.KvqCache(f, [1 << 40], [2], arena=arena)
        if int16:
            c.kvq_cache_set_option(kq.KVQ_OPT_TIER16, kq.KVQ_TIER16_INT16)
        return c

    c, want = new(), new()
    bad_k, bad_v = k[:, :, :160].clone(), v[:, :, :160].clone()
    bad_k[:, :, n:], bad_v[:, :, n:] = math.nan, math.inf
    c.kvq_quantize_append(0, bad_k, bad_v, bits)
    if way == "truncate":
        c.kvq_cache_truncate(0, n)
    else:
        d = new()
        kq.kvq_cache_fork(d, c, 0, n_tokens=n)
        c = d
    if n:
        want.kvq_quantize_append(0, k[:, :, :n].contiguous(), v[:, :, :n].contiguous(), bits)
    assert c.kvq_cache_describe(0) == want.kvq_cache_describe(0)
    assert c.kvq_cache_arena_free_bytes() == want.kvq_cache_arena_free_bytes()
    q = torch.randn(2, 4, D, generator=g, device="cuda").half()
    for grown in (0, 70):
        if grown:
            for x in (c, want):
                x.kvq_quantize_append(0, k[:, :, 160:].contiguous(), v[:, :, 160:].contiguous(), bits)
        if n + grown:
            assert exported(c) == exported(want)
            a, b = torch.empty(2, 4, D, device="cuda"), torch.empty(2, 4, D, device="cuda")
            for x, o in ((c, a), (want, b)):
                x.kvq_cache_set_option(kq.KVQ_OPT_DETERMINISTIC, 1)
                x.kvq_decode_attention(0, q, o)
            assert torch.isfinite(a).all() and float((a - b).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("int16,group,reparam", [(False, 32, False), (True, 128, True), (False, 64, True)])
@pytest.mark.parametrize("begin,n", [(0, None), (5, None), (100, 1), (127, 130), (400, 61), (0, 0)])
def test_read(dtype, int16, group, reparam, begin, n):
    """The exact value rounded to the output's type; 32 bits: one fused step, and the factor's product."""
    c, lam, g = make(2, 6, 3, MIXED, int16=int16, group=group, reparam=reparam, layers=2)
    n = 461 - begin if n is None else n
    k, v = (torch.full((2, 3, n + 1, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    ko, vo = (x.flatten()[:2 * 3 * n * D].view(2, 3, n, D) for x in (k, v))
    c.kvq_cache_read(1, begin, ko, vo)
    K, V = cached(c, 1)
    if lam is not None:
        K = K * lam.double()[:, None, :]
    step = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -24
    for got, want, whole, x in ((ko, K, k, lam), (vo, V, v, None)):
        want = want[:, :, begin:begin + n]
        tol = want.abs() * (step + (0 if x is None else 2.0 ** -23)) + 2.0 ** -25
        if dtype == torch.float16:
            tol = tol + want.abs() * 2.0 ** -23
        assert bool(((got.double() - want).abs() <= tol).all())
        assert float((whole.flatten()[2 * 3 * n * D:] - 7).abs().max()) == 0
    if dtype == torch.float16 and not reparam and not int16 and n:  # the raw tier gives back what went in
        last = max(begin, 384) - begin
        assert torch.equal(vo[:, :, last:].double(), V[:, :, begin + last:begin + n])


def test_prompt_in_chunks_over_what_the_cache_holds():
    """A second chunk attends to the first as the cache holds it, read back."""
    c, lam, g = make(1, 8, 2, [(300, 8)])
    q, k, v = (torch.randn(h, 100, D, generator=g, device="cuda").half() for h in (8, 2, 2))
    K, V = (torch.empty(1, 2, 300, D, dtype=torch.float16, device="cuda") for _ in range(2))
    c.kvq_cache_read(0, 0, K, V)
    keys, values = torch.cat([K[0], k], 1), torch.cat([V[0], v], 1)
    out = torch.empty(8, 100, D, dtype=torch.float16, device="cuda")
    kq.kvq_prompt_attention(q.transpose(0, 1), keys.transpose(0, 1), values.transpose(0, 1), out.transpose(0, 1), [0, 100], [0, 400])
    tree = torch.empty(1, 8, 100, D, dtype=torch.float16, device="cuda")
    sees = torch.ones(100, 100).tril().bool()
    from test_gpu_tree import words
    c.kvq_tree_attention(0, q[None], k[None], v[None], words(sees), tree)
    assert float((tree[0].float() - out.float()).abs().max()) < 4e-3


def test_another_stream():
    c, lam, g = make(2, 4, 2, MIXED)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    d = like(c, 2)
    torch.cuda.synchronize()
    k, v = (torch.empty(2, 2, 461, D, dtype=torch.float16, device="cuda") for _ in range(2))
    kq.kvq_cache_fork(d, c, 0, seq_map([1, 0]), stream=s)
    d.kvq_cache_truncate(0, 400, stream=s)
    d.kvq_cache_read(0, 0, k[:, :, :400].contiguous(), v[:, :, :400].contiguous(), stream=s)
    s.synchronize()
    for x, y in zip(cached(d), cached(c)):
        assert torch.equal(x, y[[1, 0]][:, :, :400])
