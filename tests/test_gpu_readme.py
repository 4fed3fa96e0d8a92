"""The README's verification step with a forward of the caller's own runs as it stands there, step after step, and carries no token's
weight over to another."""
import math
import os
import re

import pytest
import torch

import paper_2407_09722_b200 as M

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def example():
    text = open(README).read()
    block = re.search(r"A verification step with a forward of your own, over pages:\n\n((?:    .*\n)+)", text).group(1)
    return "\n".join(line[4:] for line in block.splitlines())


def test_the_readme_example_step_after_step():
    code = example()
    for was, now in (("window=4096", "window=40"), ("keep=8192", "keep=24"), ("recent=1024", "recent=8")):
        assert was in code
        code = code.replace(was, now)
    B, Hq, Hkv, hd, gamma, V, page = 3, 4, 2, 64, 3, 101, 16
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *d: torch.randn(*d, device="cuda", generator=gen)  # noqa: E731
    k_pages, v_pages = (torch.zeros(12, Hkv, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ns = dict(torch=torch, math=math, gamma=gamma, k_pages=k_pages, v_pages=v_pages, table=torch.arange(12, dtype=torch.int32, device="cuda").view(B, 4),
              lens=torch.tensor([0, 9, 20], dtype=torch.int32, device="cuda"), weights=torch.zeros(B, Hkv, 4 * page, device="cuda"),
              result=M.ResultBuffers(B, gamma, gamma), rest_of_the_decoder=lambda y: rand(B, gamma + 1, V))
    ns["pos"] = ns["lens"].clone()
    evicted = 0
    for _ in range(20):
        x = rand(B, gamma + 1, Hq + 2 * Hkv, hd).bfloat16()
        ns["q"], ns["k"], ns["v"] = x.split([Hq, Hkv, Hkv], 2)
        ns["draft_tok"] = torch.randint(0, V, (B, gamma), device="cuda", dtype=torch.int32)
        ns["draft_logq"] = -4.0 * torch.arange(1, gamma + 1, device="cuda").float().expand(B, gamma).contiguous()
        ns["uniforms"] = torch.rand(B, V, device="cuda", generator=gen).clamp_(1e-6, 1 - 1e-6)
        before = ns["lens"].clone()
        exec(code, ns)
        out = ns["result"].n_out
        assert not ns["result"].status.any() and bool((out >= 1).all())
        assert torch.equal(ns["lens"], (before + out).clamp(max=24))
        evicted += int((before + out > 24).sum())
        free = torch.arange(4 * page, device="cuda") >= ns["lens"][:, None, None]
        assert not bool(ns["weights"][free.expand_as(ns["weights"])].any())          # what the next tokens' slots start from
        assert bool((ns["weights"][~free.expand_as(ns["weights"])] > 0).all())
    assert evicted > 3
