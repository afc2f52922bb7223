"""A cache whose pages carry codes, and the exact attention over it (helpers of the tree attention's tests).

Page j of (request b, KV head g) holds the same key and the same value in all its slots: key and value are
zero but for one channel each, the page's key code and value code.  A page that is read in another's place, or
twice, or not at all then moves a channel of the output by its 16 tokens' whole share."""
import numpy as np

KEY, VALUE = 8.0, 64.0


def codes(b, g, pages):
    """(key code, value code) of a request's pages under a KV head."""
    j = np.arange(pages)
    return (7 * j + 5 * (j // 128) + 29 * b + 11 * g) % 128, (j + 3 * (j // 128) + 41 * b + 17 * g) % 128


def attention(q, prior, key_code, value_code, scale):
    """q [nodes, heads, 128] float64, a chain behind `prior` tokens: (out, lse, largest score), by pages."""
    nodes = q.shape[0]
    seen = np.clip((prior + 1 + np.arange(nodes))[:, None] - 16 * np.arange(len(key_code))[None], 0, 16)
    z = scale * KEY * q[:, :, key_code]                       # [nodes, heads, pages]
    m = np.where(seen[:, None] > 0, z, -np.inf).max(axis=-1, keepdims=True)
    w = seen[:, None] * np.exp(np.minimum(z - m, 0))
    total = w.sum(axis=-1)
    out = w @ (VALUE * (value_code[:, None] == np.arange(128)))
    return out / total[..., None], m[..., 0] + np.log(total), np.abs(z).max(axis=-1)


def tolerances(want, keys, score):
    """(of the output, of the log-sum-exp): products and sums in float32, probabilities and the result in bf16.
    Values are not negative, so that sum p |v| is the output itself."""
    e = 140 * 2.0 ** -24 * score
    sums = (keys / 32 + 60) * 2.0 ** -24
    return (2 * 2.0 ** -8 * 1.01 + 2 * e + sums + 2.0 ** -20)[..., None] * want, e + sums + 2.0 ** -21 * 16
