"""libra_append_attn_rotary in each form of the chunk launch (whole units, both halves of units,
listed halves, split keys) with each way its queries are turned: half pairing by R / 32, interleaved
pairing, any other R.

As in test_gpu_append_rotary.py, whose bounds these are: the cache holds libra_rotary_apply's bits,
outputs are those of float64 attention of the exactly turned queries, and rounded queries give the
bits of the two calls."""
import pytest
import torch

import gpu_harness as H
from test_gpu_append_rotary import NAN, Step, same
from test_gpu_rotary import Handle, randn
from test_launched_forms import driver, forms, line, pytestmark as needs_compiler  # noqa: F401

BATCHES = {  # lens, news, hq, hkv, CUs, form, whether keys are split
    "units": ([1400, 900, 300], [700, 520, 300], 16, 2, 4, "units", False),
    "halves": ([700, 520], [700, 300], 8, 2, 4, "halves", False),
    "listed": ([900, 700], [260, 33], 32, 2, 2, "listed", False),
    "tiles": ([2900, 900], [32, 20], 8, 2, 4, "tiles", True),
}
ROPES = [dict(rdim=128), dict(rdim=96, amplitude=1.25), dict(rdim=64), dict(rdim=32),
         dict(rdim=128, interleaved=True), dict(rdim=80, interleaved=True),
         dict(rdim=64, interleaved=True), dict(rdim=16, interleaved=True), dict(rdim=112),
         dict(rdim=72), dict(rdim=20), dict(rdim=22, interleaved=True), dict(rdim=104, interleaved=True)]


@needs_compiler
def test_batches_take_the_forms_they_are_for(driver):  # noqa: F811
    got = forms(driver, [line(*b[:5]) for b in BATCHES.values()])
    assert [(f["form"], f["parts"] > 1) for f in got] == [b[5:] for b in BATCHES.values()]


@pytest.mark.gpu
@pytest.mark.parametrize("kw", ROPES, ids=str)
@pytest.mark.parametrize("name", list(BATCHES))
def test_form_and_turn(name, kw):
    lens, news, hq, hkv, cus = BATCHES[name][:5]
    H.say(f"[case] append rotary form {name} {kw}")
    s = Step(lens, news, hq, hkv, seed=90, shift=77, num_cus=cus)
    rope = Handle(**kw)
    s.check(rope, s.one_step(rope), f"{name} {kw}")
    s.reset()
    rounded = s.one_step(rope, round_queries=True)
    s.reset()
    same(rounded, s.turned_first(rope), f"{name} {kw} rounded")
    rope.close()
    s.close()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv", [(28, 4), (16, 1)])
def test_rounded_single_rows_replay_from_a_graph(hq, hkv):
    """Each replay has other projections, positions and a cache whose last tokens are the former
    replay's, and gives the bits of the two calls."""
    H.say(f"[case] append rotary graph of rounded single rows {hq}/{hkv}")
    s = Step([600, 1, 16, 17, 5000], [1] * 5, hq, hkv, seed=91, shift=3, num_cus=64)
    rope = Handle(rdim=96)
    out, lse = s.outputs()
    s.call(rope, out, lse, round_queries=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.call(rope, out, lse, round_queries=True)
    for i in range(3):
        s.qkv.copy_(randn(s.qkv.shape, torch.bfloat16, 92 + i))
        s.pd.add_(500)
        out.fill_(NAN)
        lse.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), s.cache.k.clone(), s.cache.v.clone()
        same(s.one_step(rope, round_queries=True), got, f"replay {i}, eager")
        same(s.turned_first(rope), got, f"replay {i}")
    del g
    rope.close()
    s.close()
