"""The coded cache of the tree attention's long tests (no GPU): its exact attention is the plain formula's, and
a single page that is read wrongly anywhere shows."""
import numpy as np
import pytest

import tree_codes
from oracle import drafts as ref

SCALE = float(np.float32(1 / np.sqrt(128)))


def request(seed, prior, nodes, heads=2, b=3, g=1):
    q = np.random.default_rng(seed).standard_normal((nodes, heads, 128))
    key_code, value_code = tree_codes.codes(b, g, -(-(prior + nodes) // 16))
    return q, key_code, value_code


@pytest.mark.parametrize("prior,nodes", [(0, 1), (15, 3), (333, 5)])
def test_attention_by_pages(prior, nodes):
    q, key_code, value_code = request(1, prior, nodes)
    page = np.arange(prior + nodes) // 16
    k = tree_codes.KEY * (key_code[page][:, None, None] == np.arange(128))
    v = tree_codes.VALUE * (value_code[page][:, None, None] == np.arange(128))
    want, want_lse, _, _ = ref.tree_attention(q, k, v, prior, np.tril(np.ones((nodes, nodes), bool)), SCALE)
    out, lse, _ = tree_codes.attention(q, prior, key_code, value_code, SCALE)
    assert np.allclose(out, want, rtol=1e-12, atol=1e-12) and np.allclose(lse, want_lse, rtol=1e-12)


@pytest.mark.parametrize("prior", [1000, 15000, 30000, 50000])
@pytest.mark.parametrize("what", ["value of another page", "value of another head", "key of another page",
                                  "a step twice", "a step not at all"])
def test_a_wrong_page_shows(prior, what):
    """In each of 50 steps of 32 keys (two pages), by more than the tolerances."""
    rng = np.random.default_rng(prior)
    q, key_code, value_code = request(2, prior, 2)
    want, want_lse, score = tree_codes.attention(q, prior, key_code, value_code, SCALE)
    tol, lse_tol = tree_codes.tolerances(want, prior + 2, score)
    other_k, other_v = tree_codes.codes(3, 2, len(key_code))
    steps = rng.integers(0, len(key_code) // 2 - 1, size=50)
    for s in steps:
        at, far = slice(2 * s, 2 * s + 2), slice(2 * ((s + 7) % (len(key_code) // 2 - 1)), None)
        kc, vc = key_code.copy(), value_code.copy()
        if what == "value of another page":
            vc[at] = value_code[far][:2]
        elif what == "value of another head":
            vc[at] = other_v[at]
        elif what == "key of another page":
            kc[at] = key_code[far][:2]
        elif what == "a step twice":  # in the place of the one after it
            kc[2 * s + 2:2 * s + 4], vc[2 * s + 2:2 * s + 4] = (c[at][:len(c[2 * s + 2:2 * s + 4])] for c in (kc, vc))
        keep = np.ones(len(kc), bool)
        if what == "a step not at all":
            keep[at] = False
            got, got_lse, _ = tree_codes.attention(q, prior - 32, kc[keep], vc[keep], SCALE)
        else:
            got, got_lse, _ = tree_codes.attention(q, prior, kc, vc, SCALE)
        shows = np.abs(got - want) > tol
        assert shows.any() or (np.abs(got_lse - want_lse) > lse_tol).any(), s
