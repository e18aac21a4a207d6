"""Cases by which prompt attention, tree attention and the moving and reading of cached states are followed.

A case is a dict of plain values; `op` names the operator:

  prompt   kvq_prompt_attention: causal attention of packed sequences, `seqs` a list "queries:keys ..." (the queries are
           the last of the keys: a whole prompt, or a chunk of one behind the keys of the chunks before it)
  tree     KvqCache.kvq_tree_attention: the tokens of a drafted tree over a block's cache, one tree for every sequence
  fork     kvq_cache_fork: the sequences of a block continue as given by a list of parents (beams that are reordered,
           samples of one prompt).  The forked block's contents are what comes back, by kvq_cache_read
  read     KvqCache.kvq_cache_read: cached tokens back as values

Where `own` is false the same is computed with elementary torch operations in 32 bits from what stands in the cache: codes, scales
and zero points.  `exact` computes it in 64 bits from the definition.
"""
import math

import torch

own = False

D = 128
ROPE_BASE = 1.0e6


# ------------------------------------------------------------------------------------------------------------- cases
def _prompt(name, q, kv, seqs, out="fp16", lse=False, head_major=False):
    return dict(name=name, op="prompt", q=q, kv=kv, seqs=seqs, out=out, lse=lse, head_major=head_major)


def _tree(name, batch, q, kv, nodes, tiers, page, group=32, out="fp16", tier16="fp16", reparam=False, one_mask=False):
    return dict(name=name, op="tree", batch=batch, q=q, kv=kv, nodes=nodes, tiers=tiers, page=page, group=group, out=out,
                tier16=tier16, reparam=reparam, one_mask=one_mask)


def _fork(name, batch, to, kv, tiers, page, group=32, out="fp16", tier16="fp16", reparam=False):
    return dict(name=name, op="fork", batch=batch, to=to, kv=kv, tiers=tiers, page=page, group=group, out=out,
                tier16=tier16, reparam=reparam)


def _read(name, batch, kv, tiers, page, begin, group=32, out="fp16", tier16="fp16", reparam=False):
    return dict(name=name, op="read", batch=batch, kv=kv, tiers=tiers, page=page, begin=begin, group=group, out=out,
                tier16=tier16, reparam=reparam)


def listed():
    return [
        # the smallest call: a question of 37 tokens with the heads of the library's "tiny" workload
        _prompt("prompt_tiny", 8, 2, "37:37"),
        # continuous batching: sixteen 7B-shaped prompts of unequal length packed one after the other
        _prompt("prompt_packed", 28, 4, " ".join("%d:%d" % (n, n) for n in (
            41, 77, 128, 190, 255, 333, 512, 640, 700, 999, 1024, 1500, 2047, 2500, 4000, 4096)), lse=True),
        # the last chunk of 1,024 of two 32B-shaped prompts of 16,000 tokens, head-major tensors as the cache takes them
        _prompt("prompt_chunk", 40, 8, "1024:16000 1024:16000", head_major=True),
        # the largest: one 70B-shaped prompt of 32K tokens
        _prompt("prompt_long", 64, 8, "32768:32768"),
        # four drafted tokens over the "tiny" cache: all four widths, one short sequence
        _tree("tree_tiny", 1, 8, 2, 4, "1024:2 1024:4 1024:8 1024:16", 256),
        # one user of a 7B-shaped model, 16 drafted tokens over 9,001, the paper's group of 128, calibrated key factors
        _tree("tree_7b_one", 1, 28, 4, 16, "8448:4 553:16", 128, group=128, reparam=True),
        # the 32B-shaped configuration the library is benched on, 32K tokens x 4 sequences, with trees of 64 tokens
        _tree("tree_32b", 4, 40, 8, 64, "16384:2 8192:4 8064:8 128:16", 128),
        # 70B-shaped, 25 drafted tokens over one long generation of 128K
        _tree("tree_70b_128k", 1, 64, 8, 25, "81920:2 40960:4 7168:8 1024:16", 1024),
        # beam search: eight 14B-shaped beams of 2,500 tokens go on from their parents
        _fork("fork_beams", 8, 8, 8, "2432:8 68:16", 64),
        # sixteen samples of one 7B-shaped prompt of 32K tokens
        _fork("fork_samples", 1, 16, 4, "32256:4 512:16", 256),
        # the cached prefix of an ordinary chat, from its 129th token on, with calibrated key factors
        _read("read_chat", 1, 8, "2432:8 68:16", 128, 128, reparam=True),
        # a whole 32B-shaped block of four sequences at all four widths
        _read("read_32b", 4, 8, "16384:2 8192:4 8064:8 128:16", 128, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn_tiers(rng, page, most):
    tokens = _log(rng, 40, most)
    newest = min(tokens, rng.randrange(1, 1025))
    whole = (tokens - newest) // page
    tiers, left = [], whole
    for bits in sorted(rng.sample([2, 4, 8], rng.randrange(1, 4))):
        take = min(left, _log(rng, 1, max(1, whole)))
        if take:
            tiers.append("%d:%d" % (take * page, bits))
        left -= take
    tiers.append("%d:16" % (newest + left * page))
    return " ".join(tiers)


def draw(rng):
    op = rng.choice(["prompt", "prompt", "tree", "tree", "tree", "fork", "read"])
    kv = rng.choice([2, 4, 8])
    q = kv * rng.choice([1, 4, 5, 7, 8])
    out = "fp16" if op in ("prompt", "tree") else rng.choice(["fp16", "fp16", "fp32"])
    if op == "prompt":
        n = rng.choice([1, 2, 4, 9, 16])
        seqs = []
        for _ in range(n):
            keys = _log(rng, 1, 20000 if n <= 4 else 5000)
            seqs.append("%d:%d" % (keys if rng.random() < 0.6 else _log(rng, 1, keys), keys))
        c = _prompt("", q, kv, " ".join(seqs), out, rng.random() < 0.3, rng.random() < 0.5)
    else:
        batch, page = rng.choice([1, 1, 2, 4, 8]), rng.choice([32, 64, 128, 256])
        tiers = _drawn_tiers(rng, page, min(131072, (1000000 if op == "tree" else 500000) // (batch * kv)))
        kind = dict(group=rng.choice([32, 64, 128]), out=out, tier16=rng.choice(["fp16", "fp16", "int16"]),
                    reparam=rng.random() < 0.3)
        if op == "tree":
            c = _tree("", batch, q, kv, _log(rng, 1, 64), tiers, page, one_mask=rng.random() < 0.3, **kind)
        elif op == "fork":
            c = _fork("", batch, max(1, batch * rng.randrange(1, 9) // 4), kv, tiers, page, **kind)
        else:
            total = sum(n for n, _ in _tiers(dict(tiers=tiers)))
            c = _read("", batch, kv, tiers, page, rng.choice([0, rng.randrange(total)]), **kind)
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------------------------------------------------ inputs
def _gen(seed, stream):
    return torch.Generator("cuda").manual_seed(int(seed) * 1009 + stream)


def _rotate(x, positions):
    """Rotary embedding, pairs (i, i + 64), on fp32 [..., n, 128]."""
    i = torch.arange(D // 2, device="cuda", dtype=torch.float64)
    ang = positions.double()[:, None] * (ROPE_BASE ** (-2.0 * i / D))[None, :]
    c, s = ang.cos().float(), ang.sin().float()
    a, b = x[..., :64], x[..., 64:]
    return torch.cat([a * c - b * s, a * s + b * c], -1)


def _states(seed, stream, heads, n, gain=None, first=0):
    """fp16 [heads, n, 128]: unit normals, rotated at positions first, first + 1, ... where channel gains are given (keys)
    or first is not None (queries)."""
    x = torch.randn(heads, n, D, generator=_gen(seed, stream), device="cuda")
    if gain is not None:
        x = x * gain[:, None, :]
    return (x if first is None else _rotate(x, torch.arange(first, first + n, device="cuda"))).half()


def _gains(seed, kv):
    """Key channels: four of every head are 20 times as large."""
    g = _gen(seed, 1)
    gain = torch.ones(kv, D, device="cuda")
    for h in range(kv):
        gain[h, torch.randperm(D, generator=g, device="cuda")[:4]] = 20.0
    return gain


def _tiers(case):
    return [tuple(int(x) for x in t.split(":")) for t in case["tiers"].split()]


def _seqs(case):
    return [tuple(int(x) for x in s.split(":")) for s in case["seqs"].split()]


def _total(case):
    return sum(n for n, _ in _tiers(case))


def _cached(case, seed):
    """Keys and values of the cached tokens, fp16 [batch, kv, T, 128], and the block's key factors (or None)."""
    gain, n = _gains(seed, case["kv"]), _total(case)
    k = torch.stack([_states(seed, 100 + b, case["kv"], n, gain) for b in range(case["batch"])])
    v = torch.stack([_states(seed, 200 + b, case["kv"], n, None, None) for b in range(case["batch"])])
    lam = None
    if case["reparam"]:  # as a calibration gives them: some channels several times the others
        lam = (1.0 + 3.0 * torch.rand(case["kv"], D, generator=_gen(seed, 2), device="cuda")).contiguous()
    return k, v, lam


def _packed(case, seed):
    """Queries, keys and values of the packed sequences, fp16 [tokens, heads, 128]."""
    gain, q, k, v = _gains(seed, case["kv"]), [], [], []
    for i, (nq, nk) in enumerate(_seqs(case)):
        q.append(_states(seed, 300 + 3 * i, case["q"], nq, None, nk - nq))
        k.append(_states(seed, 301 + 3 * i, case["kv"], nk, gain))
        v.append(_states(seed, 302 + 3 * i, case["kv"], nk, None, None))
    q, k, v = (torch.cat(x, 1) for x in (q, k, v))
    if case["head_major"]:
        return tuple(x.contiguous().transpose(0, 1) for x in (q, k, v))
    return tuple(x.transpose(0, 1).contiguous() for x in (q, k, v))


def _drafts(case, seed):
    """A drafted tree: queries, keys, values of its nodes and which node sees which, int32 words of 32 nodes."""
    n, T, B = case["nodes"], _total(case), case["batch"]
    gain, g = _gains(seed, case["kv"]), _gen(seed, 3)
    q = torch.stack([_states(seed, 400 + b, case["q"], n, None, T) for b in range(B)])
    k = torch.stack([_states(seed, 500 + b, case["kv"], n, gain, T) for b in range(B)])
    v = torch.stack([_states(seed, 600 + b, case["kv"], n, None, None) for b in range(B)])
    trees = 1 if case["one_mask"] else B
    draws = torch.rand(trees, n, generator=g, device="cuda").cpu()
    words = torch.zeros(trees, n, (n + 31) // 32, dtype=torch.int64)
    for t in range(trees):
        for i in range(n):
            parent = int(draws[t, i] * (i + 1)) - 1  # -1: the cache's last token
            if parent >= 0:
                words[t, i] = words[t, parent]
            words[t, i, i // 32] |= 1 << (i % 32)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).cuda()
    return q, k, v, words[0] if case["one_mask"] else words


def _parents(case, seed):
    return torch.randint(0, case["batch"], (case["to"],), generator=_gen(seed, 4), device="cuda", dtype=torch.int32)


def _dtype(case):
    return torch.float32 if case["out"] == "fp32" else torch.float16


def _bytes_of(bits, group, int16):
    """Bytes of one cached token of one KV head, K and V, scales and zero points included."""
    return 2 * D * bits // 8 + (2 * (D // group) * 4 if bits < 16 or int16 else 0)


def _cache(case, batch):
    """An empty cache of one block for `batch` sequences."""
    import paper_2505_18610_amd as kq

    units, page, int16 = batch * case["kv"], case["page"], case["tier16"] == "int16"
    cfg = kq.KvqConfig(1, batch, case.get("q", case["kv"]), case["kv"], _total(case) + 1, page_tokens=page, policy=kq.KVQ_POLICY_OLDEST_FIRST,
                       group=case["group"])
    payload = sum(-(-n // page) * page * units * _bytes_of(b, 32, int16) for n, b in _tiers(case))
    arena = torch.empty(kq.kvq_arena_bytes(cfg, int(payload * 1.05) + 16 * 512 * page * units), dtype=torch.uint8, device="cuda")
    cache = kq.KvqCache(cfg, [1 << 60], [2], arena=arena)
    if int16:
        cache.kvq_cache_set_option(kq.KVQ_OPT_TIER16, kq.KVQ_TIER16_INT16)
    return cache


def _filled(case, k, v, lam):
    cache = _cache(case, case["batch"])
    if lam is not None:
        cache.kvq_cache_set_reparam(0, lam)
    t = 0
    for n, bits in _tiers(case):
        cache.kvq_quantize_append(0, k[:, :, t:t + n].contiguous(), v[:, :, t:t + n].contiguous(), bits)
        t += n
    return cache


def _stored(x, bits, case):
    """What the cache holds of x: the values themselves, or codes with a scale and a zero point for each group (Eq. 1-2)."""
    if bits == 16 and case["tier16"] == "fp16":
        return x
    g = x.float().unflatten(-1, (D // case["group"], case["group"]))
    zero, levels = g.amin(-1, keepdim=True), (1 << bits) - 1
    # quotients of 32 bits that are rounded further: formed in 64 and rounded, so that a border stays one
    scale = ((g.amax(-1, keepdim=True) - zero).double() / levels).float().half()
    code = ((g - zero).double() / scale.double()).float().round().clamp(0, levels)
    code = torch.where(scale == 0, torch.zeros_like(code), code)
    return code.to(torch.uint8 if bits <= 8 else torch.int32), scale, zero.half()


def _plain_block(case, k, v, lam):
    """The tiers of a block as the plain form holds them, oldest first: (stored keys, stored values)."""
    if lam is not None:
        k = (k.float() * (1.0 / lam)[:, None, :]).half()
    got, t = [], 0
    for n, bits in _tiers(case):
        got.append((_stored(k[:, :, t:t + n], bits, case), _stored(v[:, :, t:t + n], bits, case)))
        t += n
    return got


def prepare(case, seed):
    st = {"case": case}
    if case["op"] == "prompt":
        st["q"], st["k"], st["v"] = _packed(case, seed)
        st["q_begin"], st["k_begin"] = [0], [0]
        for nq, nk in _seqs(case):
            st["q_begin"].append(st["q_begin"][-1] + nq)
            st["k_begin"].append(st["k_begin"][-1] + nk)
        if own:
            import paper_2505_18610_amd as kq

            st["out"] = torch.empty_like(st["q"], dtype=_dtype(case))
            st["lse"] = torch.empty(case["q"], st["q"].shape[0], dtype=torch.float32, device="cuda") if case["lse"] else None
            need = kq.kvq_prompt_workspace_bytes(case["q"], case["kv"], st["q_begin"], st["k_begin"])
            st["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        torch.cuda.synchronize()
        return st
    k, v, st["lam"] = _cached(case, seed)
    if own:
        st["cache"] = _filled(case, k, v, st["lam"])
    else:
        st["block"] = _plain_block(case, k, v, st["lam"])
    if case["op"] == "tree":
        st["q"], st["k"], st["v"], st["mask"] = _drafts(case, seed)
        if own:
            st["out"] = torch.empty(st["q"].shape, dtype=_dtype(case), device="cuda")
            need = st["cache"].kvq_tree_workspace_bytes(case["nodes"])
            st["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    elif case["op"] == "fork":
        st["parents"] = _parents(case, seed)
        if own:
            st["to"] = _cache(case, case["to"])
    if own and case["op"] in ("fork", "read"):
        shape = (case.get("to", case["batch"]), case["kv"], _total(case) - case.get("begin", 0), D)
        st["k_out"], st["v_out"] = (torch.empty(shape, dtype=_dtype(case), device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    return st


# -------------------------------------------------------------------------------------------------------------- pass
def run(st):
    return (_run_own if own else _run_plain)(st, st["case"])


def _run_own(st, case):
    import paper_2505_18610_amd as kq

    if case["op"] == "prompt":
        kq.kvq_prompt_attention(st["q"], st["k"], st["v"], st["out"], st["q_begin"], st["k_begin"], lse=st["lse"],
                                workspace=st["workspace"])
        return (st["out"], st["lse"]) if case["lse"] else st["out"]
    if case["op"] == "tree":
        st["cache"].kvq_tree_attention(0, st["q"], st["k"], st["v"], st["mask"], st["out"], workspace=st["workspace"])
        return st["out"]
    if case["op"] == "fork":
        kq.kvq_cache_fork(st["to"], st["cache"], 0, seq_map=st["parents"])
        st["to"].kvq_cache_read(0, 0, st["k_out"], st["v_out"])
        return st["k_out"], st["v_out"]
    st["cache"].kvq_cache_read(0, case["begin"], st["k_out"], st["v_out"])
    return st["k_out"], st["v_out"]


def _softmax_product(s, v):
    """softmax(s) v in 32 bits and the log of the sum of exponentials; rows of nothing but -inf give zeros and -inf."""
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(s - m)
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v) / torch.where(total == 0, torch.ones_like(total), total), (m + torch.log(total))[..., 0]


def _values(stored):
    """The values that stored keys or values stand for, 32 bits."""
    if torch.is_tensor(stored):
        return stored.float()
    code, scale, zero = stored
    return (code.float() * scale.float() + zero.float()).flatten(-2)


def _run_plain(st, case):
    g = case.get("q", case["kv"]) // case["kv"]
    scale = 1.0 / math.sqrt(D)
    if case["op"] == "prompt":
        out = torch.empty(st["q"].shape, dtype=_dtype(case), device="cuda")
        lse = torch.empty(case["q"], st["q"].shape[0], device="cuda")
        for i, (nq, nk) in enumerate(_seqs(case)):
            q0, k0 = st["q_begin"][i], st["k_begin"][i]
            for h in range(case["kv"]):
                k = st["k"][k0:k0 + nk, h].float().t().contiguous()
                v = st["v"][k0:k0 + nk, h].float()
                for a in range(0, nq, 1024):
                    b = min(nq, a + 1024)
                    seen = nk - nq + b  # keys that the last of these rows sees
                    q = st["q"][q0 + a:q0 + b, h * g:(h + 1) * g].float().transpose(0, 1)
                    hidden = torch.arange(seen, device="cuda")[None, :] > torch.arange(a, b, device="cuda")[:, None] + (nk - nq)
                    s = (torch.matmul(q, k[:, :seen]) * scale).masked_fill_(hidden, -math.inf)
                    o, l = _softmax_product(s, v[:seen])
                    out[q0 + a:q0 + b, h * g:(h + 1) * g] = o.transpose(0, 1).to(out.dtype)
                    lse[h * g:(h + 1) * g, q0 + a:q0 + b] = l
        return (out, lse) if case["lse"] else out
    block = st["block"]
    if case["op"] == "fork":
        block = [tuple(x[st["parents"].long()] if torch.is_tensor(x) else tuple(y[st["parents"].long()] for y in x) for x in tier)
                 for tier in block]
    if case["op"] in ("fork", "read"):
        k, v = (torch.cat([_values(tier[w]) for tier in block], 2)[:, :, case.get("begin", 0):] for w in (0, 1))
        if st["lam"] is not None:
            k = k * st["lam"][:, None, :]
        return k.to(_dtype(case)).contiguous(), v.to(_dtype(case)).contiguous()
    # the nodes of a tree over the cached tokens and among themselves
    B, kv = st["q"].shape[0], case["kv"]
    q = st["q"].reshape(B, kv, -1, D).float()
    to_cache = q if st["lam"] is None else (q * st["lam"][:, None, :]).half().float()
    s = [torch.matmul(to_cache, _values(k).transpose(2, 3).contiguous()) for k, _ in block]
    v = [_values(x) for _, x in block]
    n = case["nodes"]
    j = torch.arange(n, device="cuda")
    sees = (st["mask"][..., j // 32] >> (j % 32)) & 1
    sees = sees.expand(B, n, n)[:, None, None]
    among = torch.matmul(q, st["k"].float().transpose(2, 3).contiguous()).reshape(B, kv, g, n, n)
    s.append(among.masked_fill(sees == 0, -math.inf).reshape(B, kv, g * n, n))
    v.append(st["v"].float())
    o, _ = _softmax_product(torch.cat(s, -1) * scale, torch.cat(v, 2))
    return o.reshape(st["q"].shape).to(_dtype(case))


# ------------------------------------------------------------------------------------------------- the same, exactly
def _exact_rows(q, k, v, hidden=None):
    """q [r, 128], k, v [t, 128] in 64 bits; hidden [r, t]: pairs that do not meet."""
    s = (q @ k.t()) / D ** 0.5
    if hidden is not None:
        s[hidden] = -math.inf
    l = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(l == -math.inf, torch.zeros_like(l), l)[:, None])
    return p @ v, l


def _exact_stored(x, bits, case):
    """x [n, 128] as the cache gives it back, 64 bits: codes by Eq. 1, scale and zero point in 16 bits by Eq. 2."""
    if bits == 16 and case["tier16"] == "fp16":
        return x.double()
    G, top = case["group"], 2 ** bits - 1
    y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, D, G):
        part = x[:, c:c + G].float()
        lo, hi = part.min(1, keepdim=True).values, part.max(1, keepdim=True).values
        S = ((hi - lo).double() / top).float().half().double()
        ratio = ((part - lo).double() / S.clamp_min(1e-30)).float()  # the quotient has 32 bits, ties go to even
        code = torch.clamp(torch.round(ratio), 0, top).double() * (S > 0)
        y[:, c:c + G] = code * S + lo.double()
    return y


def _exact_unit(case, k, v, h, lam):
    """Cached keys (as they stand in the cache, divided by their factors) and values of one KV head."""
    if lam is not None:
        k = (k.float() * (1.0 / lam[h])).half()
    ks, vs, t = [], [], 0
    for n, bits in _tiers(case):
        ks.append(_exact_stored(k[t:t + n], bits, case))
        vs.append(_exact_stored(v[t:t + n], bits, case))
        t += n
    return torch.cat(ks), torch.cat(vs)


def exact(case, seed):
    if case["op"] == "prompt":
        q, k, v = _packed(case, seed)
        out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
        lse = torch.empty(case["q"], q.shape[0], dtype=torch.float64, device="cuda")
        q0 = k0 = 0
        for nq, nk in _seqs(case):
            for h in range(case["q"]):
                u = h * case["kv"] // case["q"]
                kk, vv = k[k0:k0 + nk, u].double(), v[k0:k0 + nk, u].double()
                for a in range(0, nq, 4096):
                    rows = torch.arange(a, min(nq, a + 4096), device="cuda")
                    last = nk - nq + int(rows[-1]) + 1
                    hidden = torch.arange(last, device="cuda")[None, :] - rows[:, None] > nk - nq
                    o, l = _exact_rows(q[q0 + a:q0 + a + len(rows), h].double(), kk[:last], vv[:last], hidden)
                    out[q0 + a:q0 + a + len(rows), h], lse[h, q0 + a:q0 + a + len(rows)] = o, l
            q0, k0 = q0 + nq, k0 + nk
        return (out, lse) if case["lse"] else out
    k, v, lam = _cached(case, seed)
    kv = case["kv"]
    if case["op"] in ("fork", "read"):
        source = _parents(case, seed).tolist() if case["op"] == "fork" else range(case["batch"])
        begin = case.get("begin", 0)
        k_out, v_out = (torch.empty(len(source), kv, _total(case) - begin, D, dtype=torch.float64, device="cuda") for _ in range(2))
        for h in range(kv):
            for p in sorted(set(source)):
                kk, vv = _exact_unit(case, k[p, h], v[p, h], h, lam)
                if lam is not None:
                    kk = kk * lam[h].double()
                for b, parent in enumerate(source):
                    if parent == p:
                        k_out[b, h], v_out[b, h] = kk[begin:], vv[begin:]
        return k_out, v_out
    g = case["q"] // kv
    q, dk, dv, mask = _drafts(case, seed)
    n, T = case["nodes"], _total(case)
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    words = (mask if mask.dim() == 3 else mask[None].expand(case["batch"], -1, -1)).tolist()
    for b in range(case["batch"]):
        hidden = torch.zeros(n, T + n, dtype=torch.bool)
        for i in range(n):
            for j in range(n):
                hidden[i, T + j] = not (words[b][i][j // 32] >> (j % 32)) & 1
        hidden = hidden.cuda()
        for u in range(kv):
            kk, vv = _exact_unit(case, k[b, u], v[b, u], u, lam)
            vv = torch.cat([vv, dv[b, u].double()])
            for h in range(u * g, (u + 1) * g):
                qq = q[b, h]
                qc = qq if lam is None else (qq.float() * lam[u]).half()
                s = torch.cat([qc.double() @ kk.t(), qq.double() @ dk[b, u].double().t()], 1) / D ** 0.5
                s[hidden] = -math.inf
                out[b, h] = torch.softmax(s, -1) @ vv
    return out


# -------------------------------------------------------------------------------------------------------------- work
def work(case):
    wide = 4 if case["out"] == "fp32" else 2
    if case["op"] == "prompt":
        seqs = _seqs(case)
        nq, nk = sum(a for a, _ in seqs), sum(b for _, b in seqs)
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in seqs)
        return {"bytes": case["q"] * nq * (D * (2 + wide) + (4 if case["lse"] else 0)) + 2 * case["kv"] * nk * D * 2,
                "flops": 4 * D * case["q"] * pairs}
    int16 = case["tier16"] == "int16"
    token = [(n, _bytes_of(b, case["group"], int16)) for n, b in _tiers(case)]
    held = sum(n * size for n, size in token)
    if case["op"] == "tree":
        n, B = case["nodes"], case["batch"]
        io = B * n * D * (case["q"] * (2 + wide) + 2 * case["kv"] * 2)
        return {"bytes": io + B * case["kv"] * held, "flops": 4 * D * B * case["q"] * n * (_total(case) + n)}
    t, read, begin, batch = 0, 0, case.get("begin", 0), case.get("to", case["batch"])
    for n, size in token:
        read += size * max(0, t + n - max(t, begin))
        t += n
    rows = batch * case["kv"] * (_total(case) - begin)
    # a fork: one parent is read at least, every sequence written
    moved = case["kv"] * held * (1 + batch) if case["op"] == "fork" else 0
    return {"bytes": moved + batch * case["kv"] * read + rows * 2 * D * wide, "flops": 2 * 2 * D * rows}
