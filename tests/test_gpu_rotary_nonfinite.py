"""Infinite keys under single-token rows of libra_append_attn_rotary.

Rounded to bf16, queries give the bits of libra_rotary_apply and libra_append_attn, also over keys
that a program masks with an infinite channel."""
import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra
from paper_2606_03077_amd import workloads as wl

import gpu_harness as H
from test_gpu_append_rotary import BF16, Step, same
from test_gpu_rotary import Handle

pytestmark = pytest.mark.gpu

LENS = [700, 33, 90, 2]               # the first row is split, the others are not
GROUPS = [(8, 2), (16, 2), (18, 2), (16, 1)]


def step(hq, hkv, seed):
    s = Step(LENS, [1] * len(LENS), hq, hkv, seed=seed, num_cus=8, min_split_pages=16)
    assert 0 < libra.libra_plan_get_info(s.plan)["n_merge_groups"] < len(LENS) * hkv
    return s


def set_keys(s, places, channels, value):
    """Cached keys at (sequence, index) get value in some channels, for every KV head."""
    k, v = s.cache.unpack()
    for b, at in places:
        k[int(s.batch.block_table[b, at // 16]), :, at % 16, channels] = value
    libra.libra_kv_pack_pages(s.cache.layout, H.u16_to_dev(k), H.u16_to_dev(v), 0, s.cache.num_pages)
    torch.cuda.synchronize()
    s.k0, s.v0 = s.cache.k.clone(), s.cache.v.clone()


def bits(x):
    return wl.f32_to_bf16_bits(np.float32(x))


@pytest.mark.parametrize("hq,hkv", GROUPS)
@pytest.mark.parametrize("rdim,channels", [(64, [100]), (64, [3]), (64, [64, 127]), (128, [70]),
                                           (20, [21]), (20, [4])])
def test_rounded_queries_over_masked_keys(hq, hkv, rdim, channels):
    """-inf in channels that are copied (masks, as every query holds 1 there) or turned (whatever
    the sign gives): in every case what the two calls give."""
    H.say(f"[case] rounded over masked keys {hq}/{hkv} R={rdim} channels={channels}")
    s = step(hq, hkv, 80)
    s.q[:, :, channels] = 1.0
    set_keys(s, [(0, i) for i in range(100, 400)] + [(1, 5), (1, 31), (2, 0)], channels, bits(-np.inf))
    rope = Handle(rdim=rdim)
    got = s.one_step(rope, round_queries=True)
    s.reset()
    want = s.turned_first(rope)
    same(got, want, "rounded over masked keys")
    if min(channels) >= rdim:
        assert bool(torch.isfinite(got[0].view(BF16)).all()) and bool(torch.isfinite(got[1]).all())
    rope.close()
    s.close()
