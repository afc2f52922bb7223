"""Infinite and NaN keys and queries under libra_append_attn_rotary.

Rounded to bf16, queries give the bits of libra_rotary_apply and libra_append_attn, also over keys
that a program masks with an infinite channel.  In 16 bits a row that sees such a key has what the
unrounded query has, or is NaN (its LSE -inf), whether its keys are split or not; rows that do not
see it keep their results."""
import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra
from paper_2606_03077_amd import workloads as wl

import gpu_harness as H
from test_gpu_append_rotary import BF16, Step, same
from test_gpu_rotary import Handle, f64

pytestmark = pytest.mark.gpu

LENS = [700, 33, 90, 2]               # the first row is split, the others are not
GROUPS = [(8, 2), (16, 2), (18, 2), (16, 1)]


def step(hq, hkv, seed, news=(1, 1, 1, 1)):
    s = Step(LENS, list(news), hq, hkv, seed=seed, num_cus=8, min_split_pages=16)
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


@pytest.mark.parametrize("hq,hkv", GROUPS)
@pytest.mark.parametrize("channel", [3, 100])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("news", [(1, 1, 1, 1), (1, 20, 60, 2)])
def test_a_key_that_is_not_finite(hq, hkv, channel, value, news):
    H.say(f"[case] key of {value} in channel {channel}, {hq}/{hkv}, new tokens {news}")
    s = step(hq, hkv, 81, news)
    rope = Handle(rdim=64)
    clean = s.one_step(rope)
    s.reset()
    set_keys(s, [(0, 650), (2, 7)], [channel], wl.BF16_NAN if np.isnan(value) else bits(value))
    out, lse, _, _ = s.one_step(rope)
    q = torch.from_numpy(rope.turn(f64(s.q), s.pos)).cuda()
    got, glse = out.view(BF16).double(), lse.double()
    r0 = finite = 0
    for b, ((k, v), n, c) in enumerate(zip(s.tokens(), LENS, news)):
        rows = slice(r0, r0 + c)
        r0 += c
        if b not in (0, 2):
            # (near, as the chunk kernel's maxima are a wave's, and its rows other sequences')
            H.assert_parity(got[rows].cpu().numpy(), glse[rows].cpu().numpy(),
                            clean[0][rows].view(BF16).double().cpu().numpy(),
                            clean[1][rows].double().cpu().numpy(), label=f"sequence {b}")
            continue
        seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - c, n, device="cuda")[:, None]
        for h in range(hq):
            z = (q[rows, h] @ k[:, h // (hq // hkv)].double().t()) * s.batch.scale
            z.masked_fill_(~seen, -np.inf)
            L = torch.logsumexp(z, dim=1)
            o = torch.exp(z - L[:, None]) @ v[:, h // (hq // hkv)].double()
            none = got[rows, h].isnan().any(dim=1)
            assert bool(got[rows, h][none].isnan().all()) and bool((glse[rows, h][none] == -np.inf).all())
            assert not bool((o.isnan().any(dim=1) & ~none).any()), (b, h)
            if bool((~none).any()):
                finite += int((~none).sum())
                H.assert_parity(got[rows, h][~none][:, None].cpu().numpy(), glse[rows, h][~none][:, None].cpu().numpy(),
                                o[~none][:, None].cpu().numpy(), L[~none][:, None].cpu().numpy(),
                                label=f"sequence {b}, head {h}")
    H.say(f"[case] {finite} of the rows that see it stay finite")
    assert finite == 0 or not np.isnan(value)
    rope.close()
    s.close()


@pytest.mark.parametrize("hq,hkv", GROUPS)
def test_a_query_that_is_not_finite_makes_its_row_nan(hq, hkv):
    """All of a row's splits are NaN then, and nothing finite is left to merge."""
    H.say(f"[case] query of NaN, {hq}/{hkv}")
    s = step(hq, hkv, 82)
    rope = Handle(rdim=64)
    clean = s.one_step(rope)
    s.reset()
    s.q[0, 3, 90] = s.q[2, 1, 5] = float("nan")
    out, lse, _, _ = s.one_step(rope)
    o = out.view(BF16)
    bad = torch.zeros((s.rows, s.hq), dtype=torch.bool, device="cuda")
    bad[0, 3] = bad[2, 1] = True
    assert bool(o[bad].isnan().all()) and bool((lse[bad] == -np.inf).all())
    assert torch.equal(out[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])
    rope.close()
    s.close()
