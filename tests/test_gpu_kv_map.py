"""libra_kv_map and libra_kv_accept on the GPU against the oracle, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import drafts as ref
from paper_2606_03077_amd import libra

from test_gpu_kv_append import Cache

pytestmark = pytest.mark.gpu
I32 = torch.int32


def dev(a, dtype=I32):
    return torch.as_tensor(np.asarray(a), dtype=dtype).cuda()


class Tables:
    """A call's arrays; `in_place`: held_out and num_free_out are the inputs."""

    def __init__(self, prior, new, held, table, free, num_free, rows, depths=None, in_place=False):
        self.host = dict(prior=prior, new=new, held=held, table=np.asarray(table), free=free,
                         num_free=num_free, rows=rows, depths=depths)
        B = len(prior)
        self.prior, self.new, self.held = dev(prior), dev(new), dev(held)
        self.table = dev(table).reshape(B, np.shape(table)[1])
        self.free, self.num_free = dev(free), dev([num_free])
        self.depths = None if depths is None else dev(depths)
        junk = lambda n, dtype=I32: torch.full((n,), -77, dtype=dtype, device="cuda")
        self.slots, self.positions = junk(rows, torch.int64), junk(rows)
        self.starts, self.refused = junk(B + 1), junk(B)
        self.held_out = self.held if in_place else junk(B)
        self.num_out = self.num_free if in_place else junk(1)

    def call(self, stream=None):
        libra.libra_kv_map(self.prior, self.new, self.held, self.table, self.table.shape[1], self.free,
                           self.num_free, self.depths, self.slots, self.positions, self.starts,
                           self.held_out, self.num_out, self.refused, stream=stream)

    def check(self, want=None):
        torch.cuda.synchronize()
        want = want or ref.kv_map(**self.host)
        got = dict(table=self.table, free=self.free, held=self.held_out, num_free=self.num_out,
                   refused=self.refused, starts=self.starts, slots=self.slots, positions=self.positions)
        for name, t in got.items():
            w = np.asarray(want[name]).reshape(tuple(t.shape))
            assert np.array_equal(t.cpu().numpy(), w), name


def random_tables(seed, batch, hi, new_hi, spare, rows_off=0, depths=False, gone=0.1, in_place=False):
    rng = np.random.default_rng(seed)
    prior = rng.integers(0, hi, size=batch, endpoint=True)
    new = rng.integers(0, new_hi, size=batch, endpoint=True)
    held = -(-prior // 16) + (rng.random(batch) < 0.2) * rng.integers(0, 3, size=batch)
    away = rng.random(batch) < gone
    prior[away], new[away] = 0, 0
    columns = int(max(held.max(initial=0), (-(-(prior + new) // 16)).max(initial=0), 1))
    used = int(held.sum())
    perm = rng.permutation(used + spare)
    table, at = np.full((batch, columns), -5), 0
    for b in range(batch):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.full(used + spare, -9)
    free[:spare] = perm[used:]
    rows = max(0, int(new.sum()) + rows_off)
    d = rng.integers(0, 9, size=rows) if depths else None
    return Tables(prior, new, held, table, free, spare, rows, d, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,hi,new_hi,spare", [
    (1, 0, 1, 3), (1, 100, 40, 0), (3, 15, 2, 1), (64, 2000, 1, 40), (64, 2000, 1, 0), (255, 300, 64, 300),
    (1023, 90, 3, 50), (1024, 90, 3, 500), (1025, 90, 3, 5000), (2500, 200, 5, 100), (40, 9000, 700, 900)])
def test_random_requests(batch, hi, new_hi, spare, in_place):
    t = random_tables(batch * 7 + spare, batch, hi, new_hi, spare, 11, batch % 2 == 0, in_place=in_place)
    t.call()
    t.check()


@pytest.mark.parametrize("rows_off", [-5, 0, 1, 5000])
def test_rows_cut_and_padded(rows_off):
    t = random_tables(5, 50, 400, 20, 100, rows_off, True)
    t.call()
    t.check()


def test_rows_whose_sums_pass_32_bits():
    """900 requests in one pass, each of which might have all of three million rows."""
    t = random_tables(6, 900, 90, 3, 500, 3_000_000)
    t.call()
    t.check()


def test_no_requests_and_no_rows():
    t = Tables([], [], [], np.zeros((0, 1)), [1, 2, 3], 2, 4)
    t.call()
    t.check()
    t = random_tables(1, 30, 100, 0, 10, 0)
    assert t.slots.numel() == 0
    t.call()
    t.check()


def test_everything_ends():
    t = random_tables(9, 200, 3000, 5, 0, 3, gone=1.0)
    t.call()
    t.check()
    assert int(t.num_out) == t.free.numel()


@pytest.mark.parametrize("what,value", [("prior", -1), ("new", -3), ("held", -1), ("held", 99),
                                        ("new", 16 * 99), ("prior", 2 ** 31 - 1), ("new", 2 ** 31 - 1)])
def test_bad_requests_are_refused_and_left_alone(what, value):
    t = random_tables(3, 20, 200, 20, 200, 7)
    t.host[what] = np.array(t.host[what])
    t.host[what][6] = value
    setattr(t, what, dev(t.host[what]))
    rows = t.host["rows"]
    want = ref.kv_map(**t.host) if t.host["new"].sum() < 10 ** 6 else None
    t.call()
    torch.cuda.synchronize()
    assert t.refused[6] == 1 and t.held_out[6] == int(t.host["held"][6])
    assert (t.starts <= rows).all()
    if want is not None:
        t.check(want)


@pytest.mark.parametrize("num_free", [-4, 1 << 30])
def test_heights_outside_the_stack(num_free):
    t = random_tables(4, 10, 60, 20, 50)
    t.num_free.fill_(num_free)
    t.host["num_free"] = num_free
    t.host["free"] = t.free.cpu().numpy()
    t.call()
    t.check()


def test_replayed_steps_follow_the_lengths():
    """One captured call, in place, serves a run of drafted steps: grow, accept some, shrink, end."""
    rng = np.random.default_rng(2)
    B, columns, pool, rows = 37, 30, 37 * 25, 37 * 9 + 5
    prior = rng.integers(0, 200, size=B)
    t = Tables(prior, np.zeros(B, int), np.zeros(B, int), np.zeros((B, columns)), np.arange(pool), pool, rows,
               in_place=True)
    t.call()                                          # pages for what is there
    t.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.call()
    state = ref.kv_map(**t.host)
    for step in range(12):
        new = rng.integers(0, 9, size=B) if step % 2 == 0 else np.zeros(B, int)
        if step % 2:
            prior = prior + rng.integers(0, 5, size=B)
            prior[rng.random(B) < 0.1] = 0
        t.prior.copy_(dev(prior)), t.new.copy_(dev(new))
        g.replay()
        state = ref.kv_map(prior, new, state["held"], state["table"], state["free"], state["num_free"], rows)
        t.check(state)
        assert torch.ones(4, device="cuda").sum().item() == 4
    held = int(t.held.sum())
    assert held + int(t.num_free) == pool
    used = [int(p) for b in range(B) for p in t.table[b, :int(t.held[b])]]
    assert sorted(used + t.free[:int(t.num_free)].tolist()) == list(range(pool))  # no page twice


def test_on_another_stream():
    s = torch.cuda.Stream()
    t = random_tables(8, 64, 500, 9, 100)
    torch.cuda.synchronize()
    t.call(stream=s)
    s.synchronize()
    t.check()


# --- accepted tokens -------------------------------------------------------------------------

def run_accept(prior, accepted, counts, hkv=2, columns=None, break_table=None):
    accepted = np.asarray(accepted).reshape(len(prior), -1)
    nodes = int(accepted.max(initial=0)) + 1
    need = [-(-(p + nodes) // 16) for p in prior]
    pages = sum(need) + 2
    cache = Cache(pages, hkv)
    rng = np.random.default_rng(1)
    perm, at = rng.permutation(pages), 0
    columns = columns or max(need)
    table = np.full((len(prior), columns), perm[-1])
    for b, n in enumerate(need):
        table[b, :min(n, columns)] = perm[at:at + n][:columns]
        at += n
    if break_table is not None:
        table[break_table] = pages if break_table[1] % 2 else -1
    libra.libra_kv_accept(cache.layout, dev(prior), dev(accepted), dev(counts), dev(table), columns)
    got = [x.view(torch.int16).cpu().numpy() for x in cache.logical()]
    want = [x.view(torch.int16).cpu().numpy().copy() for x in cache.initial()]
    for w in want:
        for b, p in enumerate(prior):
            tokens = np.arange(columns * 16)
            slots = table[b, tokens // 16] * 16 + tokens % 16
            inside = (slots >= 0) & (slots < pages * 16)
            rows = np.where(inside[:, None, None], w[np.clip(slots, 0, pages * 16 - 1)], 0)
            moved = rows.copy()
            for i in range(min(counts[b], accepted.shape[1])):
                to, of = p + i, p + accepted[b, i]
                if accepted[b, i] > i and of < len(tokens) and inside[to] and inside[of]:
                    moved[to] = rows[of]
            w[slots[inside]] = moved[inside]
    for g, w in zip(got, want):
        assert np.array_equal(g, w)
    cache.close()


@pytest.mark.parametrize("prior,accepted,counts", [
    ([0], [[0]], [1]), ([5], [[3]], [1]), ([14], [[1, 2, 3, 4]], [4]),      # overlapping: each moves down one
    ([31, 7], [[0, 2, 5], [1, 3, 4]], [3, 2]), ([100], [[4, 9, 12]], [0]),
    ([0, 16, 33], [[0, 1, 2]] * 3, [3, 3, 3]),                              # all in place
    ([9], [list(range(1, 41))], [40]),                                      # more than one turn of 16
    ([3], [list(range(2, 200, 3))], [66]), ([3, 4], [[2, 5], [3, 6]], [9, -1])])
@pytest.mark.parametrize("hkv", [1, 8])
def test_accepted_paths(prior, accepted, counts, hkv):
    run_accept(prior, accepted, counts, hkv)


def test_accept_random_paths():
    rng = np.random.default_rng(4)
    B, most = 50, 16
    accepted = np.sort(np.array([rng.permutation(64)[:most] for _ in range(B)]), axis=1)
    run_accept(rng.integers(0, 90, size=B).tolist(), accepted, rng.integers(0, most + 1, size=B).tolist())


def test_accept_skips_what_lies_outside():
    run_accept([10, 20], [[3, 30], [1, 40]], [2, 2], columns=2)             # past the table
    run_accept([10, 20], [[3, 30], [1, 40]], [2, 2], break_table=(0, 2))    # a page of -1
    run_accept([10, 20], [[3, 30], [1, 40]], [2, 2], break_table=(1, 1))    # one past the cache
