"""kvq_prompt_attention of sequences of very different lengths in one call: those of few rows go with the launch of the others or have one of their
own, blocks are cut into ranges of keys or not."""
import pytest
import torch

import paper_2505_18610_amd as kq
from test_gpu_prompt import begins, check, inputs

pytestmark = pytest.mark.gpu

CALLS = {  # query heads, KV heads, [(queries, keys)]
    "few rows beside prompts": (8, 2, [(146, 146), (18, 3372), (6, 6), (1, 1), (256, 256), (4, 884), (235, 235), (1, 0), (0, 7), (17, 17)]),
    "decode steps beside a prompt": (14, 2, [(1, 40 * i + 1) for i in range(20)] + [(700, 700)]),
    "decode steps over more keys than the prompt's": (14, 2, [(1, 3000), (2, 2500), (300, 300), (1, 299), (9, 301)]),
    "too many decode steps to go along": (16, 8, [(1, 1900 + i) for i in range(80)] + [(130, 2000)]),
    "small ones among themselves": (10, 2, [(1, 900), (5, 800), (10, 1000), (3, 60), (1, 1)]),
    "uneven: in two": (4, 4, [(3, 3), (3273, 3273), (428, 428), (4279, 4279), (2, 2), (512, 512)]),
    "uneven, most of a filling": (8, 8, [(5300, 5300)]),
}


@pytest.mark.parametrize("name", CALLS)
def test_mixed_lengths(name):
    hq, hkv, seqs = CALLS[name]
    qb, kb = begins([a for a, _ in seqs]), begins([b for _, b in seqs])
    q, k, v = inputs(len(seqs), hq, hkv, qb[-1], kb[-1])
    a = check(q, k, v, qb, kb)
    assert torch.equal(a, check(q, k, v, qb, kb)), "equal calls give equal bits"
    b = check(q, k, v, qb, kb, torch.float32, workspace=False)
    assert float((a.float() - b).abs().max()) < 5e-3
    # a workspace that holds the partial results of some launches only, with a guard behind it
    need = kq.kvq_prompt_workspace_bytes(hq, hkv, qb, kb)
    if need:
        guard = torch.full((need // 2 + 4096,), 77, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        kq.kvq_prompt_attention(q, k, v, out, qb, kb, workspace=guard[:need // 2 // 16 * 16])
        assert float((out.float() - a.float()).abs().max()) < 5e-3 and bool((guard[need // 2 // 16 * 16:] == 77).all())
