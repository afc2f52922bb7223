"""libra_append_attn_rotary on the GPU, in every launched form (decode units, wide and narrow
chunk tiles, split keys).

Where nothing turns (frequencies of zero) it gives libra_append_attn's bits, and with queries
rounded to bf16 those of libra_rotary_apply and libra_append_attn.  Turned, the cache
holds libra_rotary_apply's bits, and outputs are those of float64 attention of the exactly turned
queries over that cache: queries enter the scores as two bf16 parts, so what is left of them is
2^-17 of each channel (two halvings of 2^-8 and the turn's own error), and a score, a sum of 128
float32 products, is within scale |q| |k| (2^-17 + 128 * 2^-24) of exact."""
import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra
from paper_2606_03077_amd import workloads as wl

import gpu_harness as H
from test_gpu_rotary import Handle, f64, randn

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
NAN = 0x7FC0


class Step:
    """A batch's cache, projections and plan."""

    def __init__(self, lens, news, hq, hkv, seed=1, shift=None, **params):
        self.lens, self.news, self.hq, self.hkv = lens, news, hq, hkv
        self.batch = wl.custom_batch(lens, news, num_q_heads=hq, num_kv_heads=hkv, seed=seed,
                                     append=True)
        self.cache = H.DeviceCache(self.batch)
        self.rows = sum(news)
        self.qkv = torch.empty((self.rows, hq + 2 * hkv, 128), dtype=BF16, device="cuda")
        self.q, self.k, self.v = self.qkv.split([hq, hkv, hkv], dim=1)
        for dst, src in ((self.q, self.batch.q), (self.k, self.batch.k_new), (self.v, self.batch.v_new)):
            dst.copy_(H.u16_to_dev(src).view(BF16))
        at = np.concatenate([np.arange(n - c, n) for n, c in zip(lens, news)]).astype(np.int32)
        self.pos = at if shift is None else (at + shift).astype(np.int32)
        self.pd = torch.from_numpy(self.pos).cuda()
        self.given = None if shift is None else self.pd
        self.params = params
        self.plan = H.plan_for(self.batch, **params)
        self.ws = libra.alloc_workspace(self.plan)
        self.k0, self.v0 = self.cache.k.clone(), self.cache.v.clone()

    def outputs(self):
        return (torch.full((self.rows, self.hq, 128), NAN, dtype=torch.int16, device="cuda"),
                torch.full((self.rows, self.hq), float("nan"), device="cuda"))

    def reset(self):
        self.cache.k.copy_(self.k0)
        self.cache.v.copy_(self.v0)

    def call(self, rope, out, lse, ws=None, stream=None, round_queries=False):
        libra.libra_append_attn_rotary(
            self.cache.layout, self.plan, rope.h, self.given, self.q, self.k, self.v, self.cache.bt,
            self.cache.bt_stride, len(self.lens), self.hq, self.batch.scale,
            self.ws if ws is None else ws, out, lse, stream=stream, round_queries=round_queries)

    def unturned(self):
        """libra_append_attn on the projections as they are."""
        out, lse = self.outputs()
        libra.libra_append_attn(self.cache.layout, self.plan, self.q.contiguous(),
                                self.k.contiguous(), self.v.contiguous(), self.cache.bt,
                                self.cache.bt_stride, len(self.lens), self.hq, self.batch.scale,
                                self.ws, out, lse)
        torch.cuda.synchronize()
        return out, lse, self.cache.k.clone(), self.cache.v.clone()

    def turned_first(self, rope):
        """libra_append_attn on projections that libra_rotary_apply has turned."""
        q, k = (torch.empty(t.shape, dtype=BF16, device="cuda") for t in (self.q, self.k))
        libra.libra_rotary_apply(rope.h, self.q, self.pd, q)
        libra.libra_rotary_apply(rope.h, self.k, self.pd, k)
        out, lse = self.outputs()
        libra.libra_append_attn(self.cache.layout, self.plan, q, k, self.v.contiguous(), self.cache.bt,
                                self.cache.bt_stride, len(self.lens), self.hq, self.batch.scale,
                                self.ws, out, lse)
        torch.cuda.synchronize()
        return out, lse, self.cache.k.clone(), self.cache.v.clone()

    def one_step(self, rope, **kw):
        out, lse = self.outputs()
        self.call(rope, out, lse, **kw)
        torch.cuda.synchronize()
        return out, lse, self.cache.k.clone(), self.cache.v.clone()

    def tokens(self):
        """[sequence] -> (K, V), [length, hkv, 128] as cached, bf16."""
        k, v = torch.empty_like(self.cache.k), torch.empty_like(self.cache.v)
        libra.libra_kv_unpack_pages(self.cache.layout, k, v, 0, self.cache.num_pages)
        k, v = (t.view(BF16).view(-1, self.hkv, 16, 128) for t in (k, v))
        for b, n in enumerate(self.lens):
            ids = self.cache.bt[b, :(n + 15) // 16].long()
            yield [t[ids].transpose(1, 2).reshape(-1, self.hkv, 128)[:n] for t in (k, v)]

    def check(self, rope, got, label):
        """The cache and the outputs after a call."""
        out, lse = H.bf16_dev_to_f64(got[0]), got[1].double().cpu().numpy()
        turned = torch.empty((self.rows, self.hkv, 128), dtype=BF16, device="cuda")
        libra.libra_rotary_apply(rope.h, self.k, self.pd, turned)
        q = torch.from_numpy(rope.turn(f64(self.q), self.pos)).cuda()
        G, r0, worst, rms = self.hq // self.hkv, 0, 0.0, []
        ro, rl = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
        for (k, v), n, c in zip(self.tokens(), self.lens, self.news):
            rows = slice(r0, r0 + c)
            assert torch.equal(k[n - c:], turned[rows]) and torch.equal(v[n - c:], self.v[rows]), label
            seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - c, n, device="cuda")[:, None]
            for h in range(self.hq):
                z = (q[rows, h] @ k[:, h // G].double().t()) * self.batch.scale
                z.masked_fill_(~seen, -np.inf)
                rl[rows, h] = torch.logsumexp(z, dim=1)
                ro[rows, h] = torch.exp(z - rl[rows, h][:, None]) @ v[:, h // G].double()
            size = self.batch.scale * q[rows].norm(dim=-1).max() * k.double().norm(dim=-1).max()
            # ... and float32 exponentials and logarithm of a sum.
            tol = float(size) * (2.0 ** -17 + 2.0 ** -17) + 2.0 ** -20 * (4 + np.abs(rl[rows].cpu().numpy()))
            err = np.abs(lse[rows] - rl[rows].cpu().numpy())
            worst = max(worst, float((err / tol).max()))
            rms.append(err.ravel() ** 2)
            r0 += c
        rms = float(np.sqrt(np.concatenate(rms).mean()))
        H.say(f"[parity] {label}: lse error {worst:.3f} of its bound, rms {rms:.2e}")
        assert worst <= 1.0, label
        # Independent parts: 2^-18 / sqrt(3) of scores of size 1 to 2, and float32's roundings.
        assert rms <= 1e-5, label
        H.assert_parity(out, lse, ro.cpu().numpy(), rl.cpu().numpy(), label=label)

    def close(self):
        libra.libra_plan_destroy(self.plan)
        self.cache.close()


def same(a, b, label):
    for x, y, what in zip(a, b, ("out", "lse", "k", "v")):
        x, y = (t.view(torch.int32) if t.dtype == torch.float32 else t for t in (x, y))
        assert torch.equal(x, y), f"{label}: {what} differs"


CASES = [
    # lens, news, hq, hkv, plan parameters
    ("decode rows", [1, 2, 17, 300, 5000, 64], [1] * 6, 28, 4, dict(num_cus=64)),
    ("one decode row", [700], [1], 40, 8, {}),
    ("prompt of one page", [16], [16], 4, 2, {}),
    ("first tokens", [1, 2, 3], [1, 2, 3], 8, 8, {}),
    ("mixed", [70, 300, 45, 2200, 33], [1, 100, 45, 1, 2], 32, 8, dict(num_cus=32, units_per_cu=1,
                                                                     min_split_pages=2)),
    ("one head a group", [600, 90], [333, 1], 4, 4, {}),
    ("three heads a group", [600, 90], [333, 70], 12, 4, {}),
    ("seven heads a group", [1000, 50], [400, 20], 14, 2, {}),
    ("sixteen heads a group", [300, 1500], [50, 200], 32, 2, {}),
    ("split keys", [2900, 700], [32, 1], 8, 2, dict(num_cus=4)),
    ("wide tiles", [2100, 1500, 900], [2100, 700, 900], 40, 8, dict(num_cus=16)),
    ("long prior", [70000], [40], 10, 2, {}),
    ("decode, eight heads a group", [1, 16, 17, 900, 4097], [1] * 5, 16, 2, dict(num_cus=32, min_split_pages=2)),
    ("decode, nine heads a group", [1, 16, 17, 900], [1] * 4, 18, 2, dict(num_cus=32, min_split_pages=2)),
    ("decode, sixteen heads a group", [1, 700, 33, 48], [1] * 4, 16, 1, {}),
    ("decode beside a chunk, sixteen heads", [700, 150], [1, 90], 32, 2, dict(num_cus=32)),
]
ROPES = [dict(), dict(rdim=64, interleaved=True), dict(rdim=20), dict(rdim=96, amplitude=1.25),
         dict(interleaved=True), dict(rdim=32), dict(rdim=2, interleaved=True), dict(rdim=112)]


def still():
    """A rotary that turns nothing."""
    r = Handle(rdim=44)
    libra.libra_rotary_destroy(r.h)
    r.theta = np.zeros(22, np.longdouble)
    r.h = libra.libra_rotary_create(rotary_dim=44, frequencies=np.zeros(22))
    return r


@pytest.mark.parametrize("shift", [None, 100000])
@pytest.mark.parametrize("case", range(len(CASES)), ids=[c[0] for c in CASES])
def test_cases(case, shift):
    name, lens, news, hq, hkv, params = CASES[case]
    s = Step(lens, news, hq, hkv, seed=case, shift=shift, **params)
    plain = s.unturned()
    s.reset()
    rope = still()
    same(s.one_step(rope), plain, f"{name}, still")
    rope.close()
    for j in range(2):
        kw = ROPES[(case + 3 * j + 5 * (shift is not None)) % len(ROPES)]
        H.say(f"[case] append rotary {name} shift={shift} {kw}")
        rope = Handle(**kw)
        s.reset()
        s.check(rope, s.one_step(rope), f"{name} {kw}")
        s.reset()
        rounded = s.one_step(rope, round_queries=True)
        s.reset()
        same(rounded, s.turned_first(rope), f"{name} {kw} rounded")
        rope.close()
    s.close()


@pytest.mark.parametrize("seed", range(8))
def test_random_batches(seed):
    rng = np.random.default_rng(300 + seed)
    hkv, G, B = int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 2, 4, 5, 7, 8])), int(rng.integers(1, 12))
    news = [int(rng.choice([1, 1, 2, 15, 16, 17, 64, 300])) for _ in range(B)]
    lens = [c + int(rng.choice([0, 1, 15, 31, 500, 2000])) for c in news]
    params = dict(num_cus=int(rng.choice([4, 16, 64, 256])), min_split_pages=int(rng.choice([1, 4, 16])))
    s = Step(lens, news, G * hkv, hkv, seed=seed, shift=int(rng.integers(0, 5000)), **params)
    rope = Handle(rdim=2 * int(rng.integers(1, 65)), interleaved=bool(rng.integers(2)))
    H.say(f"[case] append rotary random {seed}: G={G} hkv={hkv} lens={lens} news={news} R={rope.rdim}")
    s.check(rope, s.one_step(rope), f"random {seed}")
    s.reset()
    rounded = s.one_step(rope, round_queries=True)
    s.reset()
    same(rounded, s.turned_first(rope), f"random {seed} rounded")
    rope.close()
    s.close()


@pytest.mark.parametrize("lens,news,hq,hkv", [([900, 1500], [1, 1], 8, 2), ([1500, 700], [400, 90], 10, 2),
                                              ([3000], [20], 8, 2)])
def test_scores_whose_maximum_moves(lens, news, hq, hkv):
    """Scores of size 16, so that running maxima move by far more than a product's exponent."""
    H.say(f"[case] append rotary large scores {lens} {news}")
    s = Step(lens, news, hq, hkv, seed=60, num_cus=4)
    s.qkv[:, :hq + hkv] *= 4
    s.cache.k.view(BF16).mul_(4)
    rope = Handle(rdim=96)
    out, lse, _, _ = s.one_step(rope)
    o, l = H.bf16_dev_to_f64(out), lse.double().cpu().numpy()
    q = torch.from_numpy(rope.turn(f64(s.q), s.pos)).cuda()
    G, r0 = hq // hkv, 0
    for (k, v), n, c in zip(s.tokens(), lens, news):
        seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - c, n, device="cuda")[:, None]
        for h in range(hq):
            z = (q[r0:r0 + c, h] @ k[:, h // G].double().t()) * s.batch.scale
            z.masked_fill_(~seen, -np.inf)
            L = torch.logsumexp(z, dim=1)
            p = torch.exp(z - L[:, None])
            want = (p @ v[:, h // G].double()).cpu().numpy()
            # A score is off by at most eps = scale |q| |k| (2^-17 + 2^-17), a probability by
            # that and by bf16's 2^-8, the output by its own 2^-8.
            eps = float(s.batch.scale * q[r0:r0 + c, h].norm(dim=-1).max() *
                        k[:, h // G].double().norm(dim=-1).max()) * 2.0 ** -16
            size = (p @ v[:, h // G].double().abs()).cpu().numpy()
            assert (np.abs(o[r0:r0 + c, h] - want) <= (2 * eps + 2.0 ** -8) * size + 2.0 ** -8 * np.abs(want)).all()
            L = L.cpu().numpy()
            assert (np.abs(l[r0:r0 + c, h] - L) <= eps + 2.0 ** -20 * (4 + np.abs(L))).all()
        r0 += c
    rope.close()
    s.close()


@pytest.mark.parametrize("rdim,interleaved", [(128, False), (128, True), (20, False)])
def test_other_rows_do_not_see_a_rows_infinities(rdim, interleaved):
    """A query that is infinite, NaN, or turns past bf16's largest value, and a NaN new key: only
    its own row, or its own sequence's rows that see it, go wrong.  The chunk kernel's running
    maxima move by a vote of a wave's 32 rows, so that the others' probabilities are rounded to
    bf16 against another maximum, which is 2^-8 of each, twice, and of the outputs."""
    H.say(f"[case] append rotary non-finite R={rdim}")
    s = Step([300, 200, 90], [1, 60, 40], 8, 2, seed=61)
    rope = Handle(rdim=rdim, interleaved=interleaved, amplitude=2.0)
    clean = s.one_step(rope)
    q0 = s.qkv.clone()
    most = max(float(v.abs().max()) for _, v in s.tokens())

    def near(got, clean, keep):
        a, b = (t[0].view(BF16).float()[keep] for t in (got, clean))
        assert bool(((a - b).abs() <= 2 * 2.0 ** -8 * most + 2 * 2.0 ** -8 * b.abs()).all())
        a, b = (t[1][keep] for t in (got, clean))
        assert bool(((a - b).abs() <= 2.0 ** -20 * (4 + b.abs())).all())

    for value in (float("inf"), float("nan"), 3.3e38):
        s.qkv.copy_(q0)
        s.qkv[0, 3, 1] = s.qkv[7, 5, 0] = s.qkv[30, 0, 9] = value
        s.reset()
        got = s.one_step(rope)
        keep = torch.ones((s.rows, s.hq), dtype=torch.bool, device="cuda")
        keep[0, 3] = keep[7, 5] = keep[30, 0] = False
        near(got, clean, keep)
    s.qkv.copy_(q0)
    s.qkv[1 + 25, s.hq, 2] = float("nan")              # sequence 1, new token 25, KV head 0
    s.reset()
    got = s.one_step(rope)
    keep = torch.ones((s.rows, s.hq), dtype=torch.bool, device="cuda")
    keep[1 + 25:61, :4] = False
    near(got, clean, keep)
    assert not torch.isfinite(got[0][26:61, :4].view(BF16)).any()
    rope.close()
    s.close()


def test_smaller_workspace_other_stream_and_no_lse():
    H.say("[case] append rotary workspace and stream")
    s = Step([2900, 700], [32, 1], 8, 2, num_cus=4)
    rope = Handle()
    two = s.one_step(rope)
    s.reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    small = torch.empty(H.plain_workspace(s.plan), dtype=torch.uint8, device="cuda")
    out, lse = s.outputs()
    torch.cuda.synchronize()
    s.call(rope, out, lse, ws=small, stream=side)
    torch.cuda.synchronize()
    H.assert_parity(H.bf16_dev_to_f64(out), lse.double().cpu().numpy(), H.bf16_dev_to_f64(two[0]),
                    two[1].double().cpu().numpy(), label="whole tiles against split ones")
    out2, _ = s.outputs()
    s.call(rope, out2, None, ws=small)
    torch.cuda.synchronize()
    assert torch.equal(out, out2)
    rope.close()
    s.close()


def test_replays_from_a_graph_with_new_positions():
    H.say("[case] append rotary graph")
    s = Step([600, 1500, 300, 2200], [1, 200, 64, 1], 32, 8, shift=7, num_cus=32, units_per_cu=1,
             min_split_pages=2)
    rope = Handle(rdim=64)
    out, lse = s.outputs()
    s.call(rope, out, lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.call(rope, out, lse)
    for i in range(3):
        s.pd.add_(1000)
        torch.cuda.synchronize()
        s.reset()
        out.fill_(NAN)
        lse.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), s.cache.k.clone(), s.cache.v.clone()
        s.reset()
        same(s.one_step(rope), got, f"replay {i}")
    del g
    rope.close()
    s.close()


def test_single_rows_replay_from_a_graph():
    """A step of single rows is one launch (and a merge): the units write the new tokens.  Each
    replay has other projections, and the page it writes still holds the last replay's token."""
    H.say("[case] append rotary graph of single rows")
    s = Step([600, 1, 16, 17, 5000], [1] * 5, 28, 4, shift=3, num_cus=64)
    rope = Handle()
    out, lse = s.outputs()
    s.call(rope, out, lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.call(rope, out, lse)
    for i in range(3):
        s.qkv.copy_(randn(s.qkv.shape, BF16, 40 + i))
        out.fill_(NAN)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), s.cache.k.clone(), s.cache.v.clone()
        s.check(rope, got, f"replay {i}")
        same(s.one_step(rope), got, f"replay {i}")
    del g
    rope.close()
    s.close()


def test_launches_of_a_step():
    """Per-kernel timing sees one decode launch for single rows, a cache write beside chunks."""
    H.say("[case] append rotary launches")
    rope = Handle()
    for news, kinds in (([1, 1], {"decode"}), ([1, 40], {"cache_write", "decode", "chunk"})):
        s = Step([300, 200], news, 8, 2, num_cus=8, min_split_pages=64)
        s.one_step(rope)
        libra.libra_profile_enable(True)
        try:
            libra.libra_profile_collect()
            s.one_step(rope)
            libra.libra_rotary_apply(rope.h, s.k, s.pd, torch.empty_like(s.k))
            seen = libra.libra_profile_collect()
        finally:
            libra.libra_profile_enable(False)
        assert {k for k, (_, n) in seen.items() if n} == kinds | {"rotary"}, seen
        s.close()
    rope.close()


def test_two_streams_share_plan_and_rotary():
    """Calls of one plan and one rotary at once, on two streams, each with its own cache,
    workspace and outputs."""
    H.say("[case] append rotary two streams")
    lens, news = [600, 1500, 300], [1, 200, 64]
    a, b = (Step(lens, news, 8, 2, seed=70 + i, num_cus=32) for i in (0, 1))
    rope = Handle(rdim=64)
    want = [s.one_step(rope) for s in (a, b)]
    for s in (a, b):
        s.reset()
    libra.libra_plan_destroy(b.plan)
    b.plan, streams = a.plan, [torch.cuda.Stream() for _ in range(2)]
    outs = [s.outputs() for s in (a, b)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, st in zip((a, b), outs, streams):
            s.call(rope, *o, stream=st)
    torch.cuda.synchronize()
    for s, o, w, label in zip((a, b), outs, want, "ab"):
        same((*o, s.cache.k, s.cache.v), w, label)
    rope.close()
    b.cache.close()
    a.close()


def test_stale_nan_behind_the_last_token():
    """Slots behind a sequence's end hold NaN: nothing of them comes out."""
    H.say("[case] append rotary stale slots")
    s = Step([37, 100], [5, 1], 8, 2)
    rope = Handle()
    clean = s.one_step(rope)
    s.reset()
    k, v = s.cache.unpack()
    for b, n in enumerate(s.lens):
        page, slot = int(s.batch.block_table[b, (n - 1) // 16]), (n - 1) % 16 + 1
        k[page, :, slot:] = NAN
        v[page, :, slot:] = NAN
    libra.libra_kv_pack_pages(s.cache.layout, H.u16_to_dev(k), H.u16_to_dev(v), 0, s.cache.num_pages)
    dirty = s.one_step(rope)
    same(dirty[:2], clean[:2], "stale")
    rope.close()
    s.close()
