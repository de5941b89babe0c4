"""Plans where some of what is written is in place and some apart, and two plans at once on streams of their own."""

import numpy as np
import pytest
import torch

from paper_2407_17678_amd import binding as B
from tests.test_gpu_kv_plan import _ints, random_plan

pytestmark = pytest.mark.gpu


def _tensors(p):
    return dict(table=_ints(p.table), ring=_ints(p.ring), state=_ints(p.state), lens=_ints(p.lens), new=_ints(p.new),
                ws=torch.full((B.s2_kv_plan_workspace_bytes(len(p.lens), p.table.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda"))


def _same(out, want):
    return all(np.array_equal(out[k].cpu().numpy(), np.array(want[k])) for k in ("table", "ring", "state"))


@pytest.mark.parametrize("in_place", [(), ("table",), ("ring",), ("state",), ("table", "ring"), ("ring", "state"), ("table", "state")])
def test_partly_in_place(in_place):
    for seed, pages in ((1, 9000), (2, 700)):  # (of the second the pages run short)
        p = random_plan(seed, 16, 5, 9, 70, pages)
        t = _tensors(p)
        out = {k: t[k] if k in in_place else torch.full_like(t[k], 77) for k in ("table", "ring", "state")}
        B.s2_kv_plan_paged(p.params, t["table"], t["lens"], t["new"], t["ring"], t["state"], out["table"], out["ring"], out["state"], t["ws"])
        torch.cuda.synchronize()
        assert _same(out, p.oracle())


def test_two_at_once():
    plans = [random_plan(s, 32, 8, 12, 60, 12000) for s in (3, 4)]
    made, streams = [_tensors(p) for p in plans], [torch.cuda.Stream() for _ in plans]
    outs = [{k: torch.full_like(t[k], 77) for k in ("table", "ring", "state")} for t in made]
    torch.cuda.synchronize()
    for _ in range(20):
        for p, t, o, st in zip(plans, made, outs, streams):
            B.s2_kv_plan_paged(p.params, t["table"], t["lens"], t["new"], t["ring"], t["state"], o["table"], o["ring"], o["state"], t["ws"], stream=st)
    torch.cuda.synchronize()
    for p, o in zip(plans, outs):
        assert _same(o, p.oracle())


@pytest.mark.parametrize("max_blocks", [511, 512, 513, 1024, 1300])
@pytest.mark.parametrize("in_place", [False, True])
def test_lines_longer_than_are_loaded_at_once(max_blocks, in_place):
    random_plan(5, 16, 2, 3, max_blocks, 9000).check(in_place=in_place)
    random_plan(6, 64, 3, 2, max_blocks, 1500, with_from=True).check(in_place=in_place)
