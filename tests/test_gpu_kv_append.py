"""libra_kv_append on the GPU: every cache element against the oracle's turned keys and the
given values, untouched slots bit for bit; then decode over what it wrote."""
import numpy as np
import pytest
import torch

import oracle
from oracle import rotary as ref
from paper_2606_03077_amd import libra
from paper_2606_03077_amd import workloads as wl

import gpu_harness as H
from test_gpu_rotary import Handle, f64, randn

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


class Cache:
    def __init__(self, pages, hkv, seed=1):
        self.pages, self.hkv = pages, hkv
        self.k = torch.empty(pages * hkv * 2048, dtype=BF16, device="cuda")
        self.v = torch.empty_like(self.k)
        self.layout = libra.libra_kv_layout_create(self.k, self.v, pages, hkv)
        self.k0, self.v0 = (randn((pages, hkv, 16, 128), BF16, seed + i) for i in (0, 1))
        libra.libra_kv_pack_pages(self.layout, self.k0, self.v0, 0, pages)

    def logical(self):
        """[slots, hkv, 128] of K and of V."""
        k, v = torch.empty_like(self.k0), torch.empty_like(self.v0)
        libra.libra_kv_unpack_pages(self.layout, k, v, 0, self.pages)
        torch.cuda.synchronize()
        return [t.transpose(1, 2).reshape(-1, self.hkv, 128) for t in (k, v)]

    def initial(self):
        return [t.transpose(1, 2).reshape(-1, self.hkv, 128).clone() for t in (self.k0, self.v0)]

    def close(self):
        libra.libra_kv_layout_destroy(self.layout)


def runs(pattern, rng, pages):
    """Slots of a pattern's rows: lists of distinct slots, -1 and others for padding."""
    perm = rng.permutation(pages)
    if pattern == "one":
        return [int(perm[0]) * 16 + 7]
    if pattern == "singles":                       # decode rows
        return [int(p) * 16 + int(rng.integers(16)) for p in perm[:45]]
    if pattern == "aligned":                       # a chunk from a page's begin, ragged end
        return [int(perm[i // 16]) * 16 + i % 16 for i in range(16 * 5 + 9)]
    if pattern == "middle":                        # a chunk that begins inside a page
        return [int(perm[i // 16]) * 16 + i % 16 for i in range(5, 16 * 6 + 3)]
    if pattern == "late":                          # ... in a page's last slot
        return [int(perm[i // 16]) * 16 + i % 16 for i in range(15, 16 * 4)]
    if pattern == "next_page":                     # consecutive pages, consecutive slots
        return list(range(16 * 3 + 2, 16 * 8 + 1))
    if pattern == "backward":
        return list(range(16 * 7, 16 * 2, -1))
    if pattern == "padded":                        # padding inside and behind, of every kind
        s = list(range(16 * 2, 16 * 4)) + [-1] + list(range(16 * 5 + 1, 16 * 6)) + [-5, -1, 16 * 9]
        return s + [pages * 16, pages * 16 + 3, -2 ** 40, 2 ** 40] + list(range(16, 32)) + [-1] * 40
    if pattern == "all_padding":
        return [-1] * 70
    assert pattern == "mixed"                      # chunks and single rows, as a step has them
    out, page = [], 0
    while page + 6 < pages:
        n = int(rng.choice([1, 1, 1, 2, 15, 16, 17, 33, 64]))
        first = int(rng.integers(16))
        out += [int(perm[page + (first + i) // 16]) * 16 + (first + i) % 16 for i in range(n)]
        page += (first + n + 15) // 16
    return out


PATTERNS = ["one", "singles", "aligned", "middle", "late", "next_page", "backward", "padded",
            "all_padding", "mixed"]
ROPES = [dict(), dict(rdim=64, interleaved=True), dict(rdim=20), dict(rdim=2, interleaved=True),
         dict(rdim=96, amplitude=1.25), dict(rdim=22, interleaved=True), dict(rdim=72)]


def check_cache(cache, rope, slots, pos, k, v, label):
    """The cache holds k turned (k itself without a rope) and v at the live slots, and nothing
    else has changed."""
    slots = np.asarray(slots)
    live = (slots >= 0) & (slots < 16 * cache.pages)
    at = torch.from_numpy(slots[live]).cuda()
    gk, gv = cache.logical()
    k0, v0 = cache.initial()
    lm = torch.from_numpy(live).cuda()
    if rope is not None:
        if live.any():
            rope.check(f64(gk[at]), f64(k[lm]), pos[live], BF16, label=label)
        k0[at] = gk[at]
    else:
        k0[at] = k[lm]
    v0[at] = v[lm]
    assert torch.equal(gk, k0), f"{label}: keys outside the new slots changed"
    assert torch.equal(gv, v0), f"{label}: values differ"


@pytest.mark.parametrize("hkv,hq", [(1, 0), (3, 6), (8, 40)])
@pytest.mark.parametrize("pattern", PATTERNS)
def test_patterns_of_slots(pattern, hkv, hq):
    rng = np.random.default_rng(PATTERNS.index(pattern))
    cache = Cache(60, hkv)
    slots = runs(pattern, rng, 60)
    rows = len(slots)
    rope = Handle(**ROPES[(PATTERNS.index(pattern) + hkv) % len(ROPES)])
    H.say(f"[case] kv append {pattern} rows={rows} hkv={hkv} hq={hq} R={rope.rdim}")
    pos = rng.integers(0, 200000, size=rows).astype(np.int32)
    qkv = randn((rows, hq + 2 * hkv + 1, 128), BF16, 5)      # one head of something else between
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv + 1:]
    q_out = torch.full((rows + 2, hq, 128), 5.0, dtype=BF16, device="cuda")
    libra.libra_kv_append(cache.layout, rope.h, torch.from_numpy(pos).cuda(),
                          torch.tensor(slots, dtype=torch.int64, device="cuda"), q if hq else None,
                          k, v, q_out[:rows] if hq else None)
    check_cache(cache, rope, slots, pos, k, v, pattern)
    if hq:
        live = (np.asarray(slots) >= 0) & (np.asarray(slots) < 16 * cache.pages)
        lm = torch.from_numpy(live).cuda()
        if live.any():
            rope.check(f64(q_out[:rows][lm]), f64(q[lm]), pos[live], BF16, label="q")
        assert bool((q_out[:rows][~lm] == 5.0).all()) and bool((q_out[rows:] == 5.0).all())
    rope.close()
    cache.close()


@pytest.mark.parametrize("rope_kw", ROPES)
def test_keys_and_queries_have_rotary_applys_bits(rope_kw):
    H.say(f"[case] kv append bits {rope_kw}")
    rng = np.random.default_rng(3)
    cache, rope = Cache(40, 2), Handle(**rope_kw)
    slots = runs("mixed", rng, 40)
    rows = len(slots)
    pos = torch.from_numpy(rng.integers(-100, 40960, size=rows).astype(np.int32)).cuda()
    q, k, v = randn((rows, 5, 128), BF16, 6), randn((rows, 2, 128), BF16, 7), randn((rows, 2, 128), BF16, 8)
    want_q, want_k = torch.empty_like(q), torch.empty_like(k)
    libra.libra_rotary_apply(rope.h, q, pos, want_q)
    libra.libra_rotary_apply(rope.h, k, pos, want_k)
    at = torch.tensor(slots, dtype=torch.int64, device="cuda")
    libra.libra_kv_append(cache.layout, rope.h, pos, at, q, k, v, q)        # q in place
    gk, gv = cache.logical()
    assert torch.equal(q, want_q) and torch.equal(gk[at], want_k) and torch.equal(gv[at], v)
    rope.close()
    cache.close()


@pytest.mark.parametrize("pattern", ["singles", "middle", "padded", "mixed"])
def test_without_rotation_keys_are_copied(pattern):
    """Any bits, NaN payloads among them, and no positions."""
    H.say(f"[case] kv append copy {pattern}")
    rng = np.random.default_rng(4)
    cache = Cache(40, 3)
    slots = runs(pattern, rng, 40)
    bits = torch.from_numpy(rng.integers(-32768, 32768, size=(2, len(slots), 3, 128)).astype(np.int16)).cuda()
    libra.libra_kv_append(cache.layout, None, None,
                          torch.tensor(slots, dtype=torch.int64, device="cuda"), None, bits[0], bits[1], None)
    live = (np.asarray(slots) >= 0) & (np.asarray(slots) < 16 * 40)
    at, lm = torch.tensor(np.asarray(slots)[live], device="cuda"), torch.from_numpy(live).cuda()
    for got, before, new in zip(cache.logical(), cache.initial(), bits):
        want = before.view(torch.int16)
        want[at] = new[lm]
        assert torch.equal(got.view(torch.int16), want)
    cache.close()


def test_slots_past_32_bits_of_elements():
    """A cache of more than 2^31 elements, rows in its last pages."""
    hkv, pages = 8, 140000                        # 2.3e9 elements, 4.6 GB each side
    H.say("[case] kv append far pages")
    k = torch.empty(pages * hkv * 2048, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    lay = libra.libra_kv_layout_create(k, v, pages, hkv)
    slots = torch.arange(16 * pages - 40, 16 * pages, device="cuda")
    rope = Handle()
    kn, vn = randn((40, hkv, 128), BF16, 9), randn((40, hkv, 128), BF16, 10)
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    libra.libra_kv_append(lay, rope.h, pos, slots, None, kn, vn, None)
    ko, vo = (torch.empty((3, hkv, 16, 128), dtype=BF16, device="cuda") for _ in range(2))
    libra.libra_kv_unpack_pages(lay, ko, vo, pages - 3, 3)
    gk, gv = (t.transpose(1, 2).reshape(48, hkv, 128)[8:] for t in (ko, vo))
    rope.check(f64(gk), f64(kn), np.arange(40, dtype=np.int32), BF16)
    assert torch.equal(gv, vn)
    libra.libra_kv_layout_destroy(lay)
    rope.close()


def test_rows_of_several_launches():
    """With 1,024 KV heads a launch takes 65,536 rows.  Only the rows around that are not
    padding, so that only their projections exist."""
    H.say("[case] kv append several launches")
    hkv, per_launch, rows = 1024, 65536, 65536 + 50
    cache, rope = Cache(8, hkv), Handle()
    first = per_launch - 21                                 # a run across the two launches
    k, v = randn((71, hkv, 128), BF16, 12), randn((71, hkv, 128), BF16, 13)
    slots = np.full(rows, -1, np.int64)
    slots[first:first + 71] = np.arange(5, 76)
    pos = np.arange(rows, dtype=np.int32)
    sd, pd = torch.from_numpy(slots).cuda(), torch.from_numpy(pos).cuda()
    at = first * hkv * 128 * 2                              # the rows before are never read
    status = libra.load().libra_kv_append(
        cache.layout, rope.h, pd.data_ptr(), sd.data_ptr(), rows, None, 0, 0, k.data_ptr() - at,
        hkv * 128, v.data_ptr() - at, hkv * 128, hkv, None, torch.cuda.current_stream().cuda_stream)
    assert status == 0
    check_cache(cache, rope, slots[first:first + 71], pos[first:first + 71], k, v, "launches")
    rope.close()
    cache.close()


def test_refusals_of_the_binding(monkeypatch):
    """Wrong heads in rows far enough apart to pass by their stride, lengths, and a device that is
    not the current one; the cache stays as it was."""
    hkv, rows = 2, 4
    cache, rope = Cache(3, hkv), Handle()
    saved = cache.k.clone(), cache.v.clone()
    qkv = randn((rows, 10, 128), BF16, 31)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    slots = pos.long()

    def call(q=qkv[:, :4], k=qkv[:, 4:6], v=qkv[:, 6:8], q_out=None, p=pos, s=slots):
        libra.libra_kv_append(cache.layout, rope.h, p, s, q, k, v,
                              torch.empty(rows, 4, 128, dtype=BF16, device="cuda") if q_out is None else q_out)

    for bad in (dict(k=qkv[:, 4:5], v=qkv[:, 6:7]), dict(k=qkv[:, 4:7], v=qkv[:, 7:10]),
                dict(v=qkv[:, 6:7]), dict(k=qkv[:3, 4:6]), dict(q=qkv[:3, :4]), dict(p=pos[:3]),
                dict(s=slots[:3]), dict(p=slots), dict(s=pos), dict(k=qkv[:, 4:6, :64]),
                dict(q_out=qkv[:, 6:10]), dict(q_out=qkv[:, 6:8].contiguous()),
                dict(k=qkv[:, 4:8:2]), dict(v=qkv[:, 6:8].cpu())):
        with pytest.raises((ValueError, libra.LibraError)):
            call(**bad)
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="current device"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(cache.k, saved[0]) and torch.equal(cache.v, saved[1])
    rope.close()
    cache.close()


def _decode(cache, plan, q, table, batch, hq, scale, ws):
    out = torch.full((batch, hq, 128), 0x7FC0, dtype=torch.int16, device="cuda")
    lse = torch.full((batch, hq), float("nan"), device="cuda")
    libra.libra_decode_attn(cache.layout, plan, q, table, table.shape[1], batch, hq, scale, ws, out, lse)
    torch.cuda.synchronize()
    return H.bf16_dev_to_f64(out), lse.double().cpu().numpy()


def test_append_then_decode_in_a_replayed_graph():
    """A captured step: keys and queries turned, the cache written, decode attention over it.
    Each replay takes another position and slot for every request (padded to the graph's rows)
    and is compared with the eager calls, and the eager ones with the oracle."""
    lens, hq, hkv, pages = [40, 17, 100, 3], 8, 2, 40
    H.say("[case] kv append + decode graph")
    rng = np.random.default_rng(5)
    cache, rope = Cache(pages, hkv), Handle()
    B, rows = len(lens), 6                         # two rows of padding
    table = rng.permutation(pages)[:4 * 7].reshape(4, 7).astype(np.int32)
    td = torch.from_numpy(table).cuda()
    scale = 0.0883
    plan = libra.libra_splitkv_plan(libra.LIBRA_MODE_DECODE, B, hq, hkv, lens, None, num_cus=8,
                                    min_split_pages=1)
    ws = libra.alloc_workspace(plan)
    libra.libra_plan_upload(plan, ws)
    q_out = torch.zeros((rows, hq, 128), dtype=BF16, device="cuda")
    qkv = randn((rows, hq + 2 * hkv, 128), BF16, 11)
    pos, slots = (torch.zeros(rows, dtype=t, device="cuda") for t in (torch.int32, torch.int64))
    out = torch.empty((B, hq, 128), dtype=torch.int16, device="cuda")
    lse = torch.empty((B, hq), device="cuda")

    def step():
        q, k, v = qkv.split([hq, hkv, hkv], dim=1)
        libra.libra_kv_append(cache.layout, rope.h, pos, slots, q, k, v, q_out)
        libra.libra_decode_attn(cache.layout, plan, q_out[:B], td, 7, B, hq, scale, ws, out, lse)

    def fill(i):
        # The new token overwrites one of the last tokens of each sequence.
        at = np.array([max(0, n - 1 - i) for n in lens])
        p = np.zeros(rows, np.int32)
        s = np.full(rows, -1, np.int64)
        p[:B] = at + 1000 * i
        s[:B] = table[np.arange(B), at // 16].astype(np.int64) * 16 + at % 16
        pos.copy_(torch.from_numpy(p))
        slots.copy_(torch.from_numpy(s))
        qkv.copy_(randn(qkv.shape, BF16, 20 + i))
        return p, s

    fill(0)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(1, 4):
        p, s = fill(i)
        saved = cache.k.clone(), cache.v.clone()
        out.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, cache.k, cache.v, q_out)]
        cache.k.copy_(saved[0])
        cache.v.copy_(saved[1])
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, lse, cache.k, cache.v, q_out)):
            assert torch.equal(a, b), i
        lk, lv = (t.view(-1, 16, hkv, 128).transpose(1, 2).contiguous() for t in cache.logical())
        rope.check(f64(q_out[:B]), f64(qkv[:B, :hq]), p[:B], BF16, label=f"replay {i}")
        ro, rl = oracle.decode_ref(H.dev_to_u16(q_out[:B].view(torch.int16)),
                                   H.dev_to_u16(lk.view(torch.int16)), H.dev_to_u16(lv.view(torch.int16)),
                                   table, np.array(lens), scale)
        H.assert_parity(H.bf16_dev_to_f64(out), lse.double().cpu().numpy(), ro, rl, label=f"replay {i}")
    del g
    libra.libra_plan_destroy(plan)
    rope.close()
    cache.close()
