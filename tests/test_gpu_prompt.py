"""kvq_prompt_attention against softmax attention in 64 bits."""
import math

import pytest
import torch

import paper_2505_18610_amd as kq

pytestmark = pytest.mark.gpu
D = 128


def reference(q, k, v, qb, kb, scale=None):
    """Outputs, the sums of probabilities times |v| that errors of the probabilities scale with, and log-sums, in 64 bits."""
    scale = scale or 1 / math.sqrt(D)
    g = q.shape[1] // k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    size, lse = torch.zeros_like(out), torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(len(qb) - 1):
        nq, nk = qb[i + 1] - qb[i], kb[i + 1] - kb[i]
        if not nq or not nk:
            continue
        hidden = torch.arange(nk, device="cuda")[None] > torch.arange(nq, device="cuda")[:, None] + (nk - nq)
        for h in range(q.shape[1]):
            kk, vv = k[kb[i]:kb[i + 1], h // g].double(), v[kb[i]:kb[i + 1], h // g].double()
            s = (q[qb[i]:qb[i + 1], h].double() @ kk.t()) * scale
            s[hidden] = -math.inf
            some = ~hidden.all(1)
            p = torch.zeros_like(s)
            p[some] = torch.softmax(s[some], -1)
            # what no row sees does not count, whatever it holds
            for to, x in ((out, vv), (size, vv.abs())):
                clean = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
                y = p @ clean
                for bad in (math.inf, -math.inf):
                    y = torch.where((p @ (x == bad).double()) > 0, torch.full_like(y, bad), y)
                nan = ((p @ torch.isnan(x).double()) > 0) | (((p @ (x == math.inf).double()) > 0) & ((p @ (x == -math.inf).double()) > 0))
                to[qb[i]:qb[i + 1], h] = torch.where(nan, torch.full_like(y, math.nan), y)
            lse[h, qb[i]:qb[i + 1]][some] = torch.logsumexp(s[some], -1)
    return out, size, lse


def inputs(seed, hq, hkv, rows_q, rows_k):
    g = torch.Generator("cuda").manual_seed(seed)
    return tuple(torch.randn(n, h, D, generator=g, device="cuda").half() for n, h in ((rows_q, hq), (rows_k, hkv), (rows_k, hkv)))


def begins(lengths):
    b = [0]
    for n in lengths:
        b.append(b[-1] + n)
    return b


def check(q, k, v, qb, kb, out_dtype=torch.float16, scale=0.0, workspace=True, out=None):
    """Probabilities are rounded to fp16 (2^-11 of each), scores and sums have 32 bits: 128 products of up to |q k| each for the score,
    whose error the exponential takes over (here less than 2^-12), and one step of the sums for each key."""
    out = torch.full(q.shape, 7.0, dtype=out_dtype, device="cuda") if out is None else out
    lse = torch.empty(q.shape[1], qb[-1], dtype=torch.float32, device="cuda")
    need = kq.kvq_prompt_workspace_bytes(q.shape[1], k.shape[1], qb, kb)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need and workspace else None
    kq.kvq_prompt_attention(q, k, v, out, qb, kb, softmax_scale=scale, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    want, size, want_lse = reference(q, k, v, qb, kb, scale)
    rows = slice(qb[0], qb[-1])
    want, size, got = want[rows], size[rows], out.double()[rows]
    longest = max(b - a for a, b in zip(kb, kb[1:]))
    tol = (2.0 ** -11 + 2.0 ** -12) * size + 2.0 ** -24 * longest * float(v[torch.isfinite(v)].abs().max() if v.numel() else 0)
    if out_dtype == torch.float16:
        tol = tol + 2.0 ** -11 * want.abs() + 2.0 ** -25
    whole = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~whole & ~torch.isnan(want)], want[~whole & ~torch.isnan(want)])
    bad = ((got - want).abs() > tol) & whole
    assert not bad.any(), (int(bad.sum()), float((got - want)[whole].abs().max()), bad.nonzero()[:4].tolist())
    some = torch.isfinite(want_lse[:, rows])
    assert torch.equal(torch.isfinite(lse[:, rows]), some)
    # a score is a sum of 128 products in 32 bits: one step of the sum of their sizes for each
    sizes = max([float((q[a:b].double().abs().amax((0, 1)) * k[c:d].double().nan_to_num(0).abs().amax((0, 1))).sum())
                 for a, b, c, d in zip(qb, qb[1:], kb, kb[1:]) if a < b and c < d] or [0.0])
    err = float((lse.double()[:, rows] - want_lse[:, rows])[some].abs().max() if some.any() else 0)
    assert err <= 2e-4 + 128 * 2.0 ** -24 * sizes * abs(scale or 1 / math.sqrt(D))
    return out


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 515])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (7, 1), (2, 2), (16, 1)])
def test_one_prompt(n, hq, hkv):
    q, k, v = inputs(n, hq, hkv, n, n)
    check(q, k, v, [0, n], [0, n])


@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 33), (1, 5000), (3, 1000), (5, 64), (16, 4097), (33, 700), (64, 2048), (130, 3001), (300, 301),
                                   (40, 7), (1, 0), (130, 100), (257, 1)])
@pytest.mark.parametrize("hq,hkv", [(5, 1), (16, 2)])
@pytest.mark.parametrize("out", [torch.float16, torch.float32])
def test_chunks_and_rows_without_keys(nq, nk, hq, hkv, out):
    q, k, v = inputs(nq + nk, hq, hkv, nq, max(nk, 1))
    a = check(q, k, v, [0, nq], [0, nk], out)
    b = check(q, k, v, [0, nq], [0, nk], out, workspace=False)
    assert torch.equal(a, check(q, k, v, [0, nq], [0, nk], out)), "equal calls give equal bits"
    assert float((a.float() - b.float()).abs().max()) < 5e-3


@pytest.mark.parametrize("seed", range(6))
def test_packed_sequences(seed):
    r = torch.Generator().manual_seed(seed)
    n = int(torch.randint(2, 100, (1,), generator=r))
    nk = [int(x) for x in torch.randint(0, 260, (n,), generator=r)]
    nq = [int(x * f) + (i % 7 == 3) for i, (x, f) in enumerate(zip(nk, torch.rand(n, generator=r).tolist()))]
    nk[0], nq[0] = 900, 900
    qb, kb = begins(nq), begins(nk)
    q, k, v = inputs(seed, 10, 2, qb[-1], kb[-1])
    check(q, k, v, qb, kb)


def test_rows_outside_the_sequences_are_left_alone():
    q, k, v = inputs(1, 4, 2, 300, 400)
    out = check(q, k, v, [50, 120, 250], [10, 90, 333])
    assert float((out[:50] - 7).abs().max()) == 0 and float((out[250:] - 7).abs().max()) == 0


def test_strides():
    q, k, v = inputs(2, 8, 2, 150, 150)
    plain = check(q, k, v, [0, 150], [0, 150])
    fused = torch.cat([q, k, v], 1)  # one projection's output
    out = check(fused[:, :8], fused[:, 8:10], fused[:, 10:], [0, 150], [0, 150])
    assert torch.equal(out, plain)
    heads = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    out = torch.empty(8, 150, D, dtype=torch.float16, device="cuda").transpose(0, 1)
    assert torch.equal(check(*heads, [0, 150], [0, 150], out=out), plain)
    one = k[:, :1]
    assert torch.equal(check(q, one.expand(-1, 2, -1), v, [0, 150], [0, 150]), check(q, one.repeat(1, 2, 1), v, [0, 150], [0, 150]))


@pytest.mark.parametrize("scale", [0.02, 0.5, -0.1])
def test_scales(scale):
    q, k, v = inputs(3, 4, 2, 100, 180)
    check(q, k, v, [0, 100], [0, 180], torch.float32, scale)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("n,at", [(20, 19), (20, 7), (70, 40), (200, 131), (400, 399), (400, 0)])
def test_keys_that_a_row_does_not_see_do_not_reach_it(bad, n, at):
    q, k, v = inputs(4, 4, 2, n, n)
    v[at, :, 5::16] = bad
    check(q, k, v, [0, n], [0, n])
    q, k, v = inputs(4, 4, 2, n, n)
    k[at] = math.nan  # of the keys: rows before it are as ever, those behind it NaN
    out = torch.empty(q.shape, dtype=torch.float16, device="cuda")
    kq.kvq_prompt_attention(q, k, v, out, [0, n])
    want, size, _ = reference(q[:at], k[:at], v[:at], [0, at], [0, at])
    assert torch.isnan(out[at:]).all()
    assert not at or float((out[:at].double() - want).abs().max()) < 5e-3


def test_scores_of_any_size():
    """Huge scores: one key takes all the weight; equal ones share it."""
    q, k, v = inputs(5, 4, 2, 90, 90)
    check(q * 30, k * 30, v, [0, 90], [0, 90], scale=1.0)
    check(torch.zeros_like(q), k, v, [0, 90], [0, 90])


def test_another_stream_and_a_graph():
    q, k, v = inputs(6, 8, 2, 40, 3000)
    qb, kb = [0, 40], [0, 3000]
    ws = torch.empty(kq.kvq_prompt_workspace_bytes(8, 2, qb, kb), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    want = torch.empty_like(q)
    kq.kvq_prompt_attention(q, k, v, want, qb, kb, workspace=ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = torch.zeros_like(q)
    s.wait_stream(torch.cuda.current_stream())
    kq.kvq_prompt_attention(q, k, v, out, qb, kb, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        kq.kvq_prompt_attention(q, k, v, out, qb, kb, workspace=ws, stream=s)
    for i in range(3):
        out.zero_()
        q.mul_(-1)
        g.replay()
        eager = torch.empty_like(q)
        torch.cuda.synchronize()
        kq.kvq_prompt_attention(q, k, v, eager, qb, kb, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_rows_beyond_4_gib():
    """Token strides as of a tensor of many heads: offsets of late rows pass 32 bits."""
    big = torch.zeros(3000, 6000, D, dtype=torch.float16, device="cuda")
    q, k, v = inputs(7, 2, 1, 70, 2990)
    big[:2990, 5000:5001], big[:2990, 5999:] = k, v
    out = check(q, big[:, 5000:5001], big[:, 5999:], [0, 70], [0, 2990])
    assert torch.equal(out, check(q, k, v, [0, 70], [0, 2990]))
