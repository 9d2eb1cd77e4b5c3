"""The README's step of several continuations, as it stands there, in a loop."""
import os
import re

import pytest
import torch

from paper_2405_03133_amd import binding as lb
from test_attn_gpu import gen, rnd

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_continuations_snippet_of_the_readme_in_a_loop():
    """Every step goes on from the rows that the one before it chose: the cache of every row against a copy of its own."""
    text = open(os.path.join(ROOT, "README.md")).read()
    code = compile(re.search(r"^Several continuations.*?```python\n(.*?)```", text, re.S | re.M).group(1), "README.md", "exec")
    B, beams, page, W, pages, Hkv, D, V = 2, 3, 4, 8, 60, 2, 8, 50
    R, g = B * beams, gen(3)
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
    k_cache, v_cache = (torch.zeros(pages, Hkv, page, D, device="cuda") for _ in range(2))
    s = dict(lb=lb, beams=beams, page=page, pages=pages, k_cache=k_cache, v_cache=v_cache, score=torch.zeros(B, beams, device="cuda"),
             free=torch.arange(pages, dtype=torch.int32, device="cuda"), count=i32(1) + pages, count_new=i32(1), lens=i32(R), lens_new=i32(R),
             table=i32(R, W) - 1, table_new=i32(R, W) - 1, copies=i32(3, R), status=i32(1))
    add, cu, positions, slots = i32(R) + 1, i32(R + 1), i32(R), torch.zeros(R, dtype=torch.int64, device="cuda")
    dense, moved = [torch.zeros(2, Hkv, 0, D, device="cuda") for _ in range(R)], 0
    for step in range(3 * page + 2):
        lb.lory_kv_plan(s["lens"], add, s["table"], s["free"], s["count"], page, s["lens_new"], cu, positions, slots, s["count_new"], s["status"])
        assert s["status"].item() == 0
        for n in ("lens", "count"):
            s[n], s[n + "_new"] = s[n + "_new"], s[n]
        new = rnd(g, 2, R, Hkv, D)
        for x, y in zip((k_cache, v_cache), new):
            x[slots // page, :, slots % page] = y
        s["logits"] = rnd(g, R, V)
        exec(code, s)
        assert s["status"].item() == 0
        dense = [torch.cat([dense[b], new[:, b, :, None]], 2) for b in range(R)]
        parents = s["parent"].view(-1).tolist()
        moved += parents != list(range(R))
        dense = [dense[p] for p in parents]
        assert s["lens"].tolist() == [step + 1] * R
        for b in range(R):
            at = s["table"][b, :-(-(step + 1) // page)].long()
            row = torch.stack([x[at].transpose(0, 1).flatten(1, 2)[:, :step + 1] for x in (k_cache, v_cache)])
            assert torch.equal(row, dense[b]), (step, b)
    assert moved > 3
