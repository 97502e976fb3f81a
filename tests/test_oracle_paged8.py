"""The 8-bit cache's oracle against torch's own 8-bit type and short loops."""
import numpy as np
import pytest
import torch

import oracle
from oracle import paged8 as o8


def test_codes_are_torchs():
    rng = np.random.default_rng(0)
    b = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(b.copy()).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(o8.VALUES)) and np.array_equal(t[~np.isnan(t)], o8.VALUES[~np.isnan(t)])
    ok = np.sort(o8.VALUES[:127])
    x = np.concatenate([ok, (ok[1:] + ok[:-1]) / 2, rng.uniform(0, 448, 4000), 2.0 ** rng.uniform(-14, 9, 4000).clip(max=8.8)])
    x = np.concatenate([x, -x]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(o8.codes(x, 0), want)
    assert (o8.codes([np.nan, np.inf, -np.inf], 3) == 127).all() and o8.codes(1e9, 0) == 126


@pytest.mark.parametrize("top,e", [(0, -117), (448, 0), (448.001, 1), (449, 1), (224, -1), (1e-40, -117), (3e38, 119),
                                   (448 * 2.0 ** -117, -117), (448.1 * 2.0 ** -117, -116), (2.0 ** 127.9, 119)])
def test_exponents(top, e):
    assert o8.exponent(top) == e


def _rows(rng, n, Hkv, scale=1.0):
    return rng.standard_normal((n, Hkv, 128)) * scale


def test_writes_and_rows():
    rng = np.random.default_rng(1)
    pool = rng.integers(0, 256, (4, 2, o8.PAGE_BYTES)).astype(np.uint8)
    k, v = _rows(rng, 100, 2), _rows(rng, 100, 2, 30.0)
    table = np.array([2, 0])
    pos = np.arange(100)
    slot = table[pos // 64] * 64 + pos % 64
    after = o8.write(pool, k, v, slot)
    rk, rv, there = o8.rows(after, table, 100)
    assert there.all()
    for x, y in ((k, rk), (v, rv)):
        for a in range(0, 100, 32):
            for h in range(2):
                top = np.abs(x[a:a + 32, h]).max()
                assert np.abs(x - y)[a:a + 32, h].max() <= top * 2.0 ** -4 and np.abs(y[a:a + 32, h]).max() <= 2 * top
        assert (np.abs(x - y) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * 30 * 5 / 224).all()
    assert np.array_equal(after[[1, 3]], pool[[1, 3]])
    # rows of the last block that are not there yet are zeros
    k2, v2, _ = o8.rows(after, table, 128)
    assert (k2[100:] == 0).all() and (v2[100:] == 0).all()
    # a row at a time, the larger ones later: each held to its block's last scale
    one = pool.copy()
    for i in range(100):
        one = o8.write(one, k[i:i + 1] * (1 + i % 32), v[i:i + 1], slot[i:i + 1])
    ok, _, _ = o8.rows(one, table, 100)
    big = k * (1 + pos % 32)[:, None, None]
    # two roundings: half a step each, the second of what the first made of it
    step = 2.0 ** (one[table][:, :, o8.SCALES:o8.SCALES + 2].astype(float) - 127)
    least = np.stack([step[p // 64, :, p % 64 // 32] for p in pos]) * 2.0 ** -9
    assert (np.abs(ok - big) <= 2.0 ** -4 * np.abs(big) + least[..., None]).all()


def test_attention_is_a_softmax():
    rng = np.random.default_rng(2)
    pool = np.zeros((3, 1, o8.PAGE_BYTES), np.uint8)
    pool = o8.write(pool, _rows(rng, 192, 1), _rows(rng, 192, 1), np.arange(192))
    q, kt, vt = rng.standard_normal((1, 2, 2, 128)), rng.standard_normal((1, 2, 1, 128)), rng.standard_normal((1, 2, 1, 128))
    out, lse, most, lse_most = o8.attention(q, kt, vt, pool, [[1, 0]], [70])
    k, v, _ = o8.rows(pool, [1, 0], 70)
    for i in range(2):
        keys, vals = np.concatenate([k[:, 0], kt[0, :i + 1, 0]]), np.concatenate([v[:, 0], vt[0, :i + 1, 0]])
        for h in range(2):
            w = np.exp(keys @ q[0, i, h] / np.sqrt(128))
            assert np.allclose(out[0, i, h], w @ vals / w.sum(), rtol=1e-12) and np.isclose(lse[0, i, h], np.log(w.sum()))
    assert (most < 0.02).all() and (lse_most < 1e-3).all()
    got, off = o8.weights(np.ones((3, 1, 64)), q[0], lse[0], pool, [[1, 0]], [69], [70], [0, 1])
    w = np.exp(k[:, 0] @ q[0, 0].T / np.sqrt(128) - lse[0, 0]).sum(1)
    assert np.allclose(np.concatenate([got[1, 0], got[0, 0, :6]]), np.concatenate([1 + w[:69], w[69:]]))
    assert (got[2] == 1).all() and (got[0, 0, 6:] == 1).all() and off.max() < 1e-4


@pytest.mark.parametrize("n,budget,first,recent", [(70, 40, 0, 0), (70, 40, 4, 10), (200, 129, 3, 64), (33, 32, 0, 40),
                                                   (100, 5, 4, 3), (100, 7, 40, 2), (20, 20, 1, 1), (20, 30, 1, 1), (20, 0, 1, 1)])
def test_eviction_keeps_the_heaviest(n, budget, first, recent):
    rng = np.random.default_rng(n + budget)
    pool = o8.write(np.zeros((4, 1, o8.PAGE_BYTES), np.uint8), _rows(rng, 256, 1), _rows(rng, 256, 1), np.arange(256))
    w = rng.integers(-2, 9, (4, 1, 64)).astype(np.float32)
    table = np.array([[3, 1, 0, 2]])
    k, v, _ = o8.rows(pool, table[0], n)
    flat = w[table[0]].reshape(-1)[:n].clip(min=0)
    after, w2, add = o8.evict(pool, w, table, [n], [budget], first, recent)
    keep = min(n, budget)
    assert add[0] == keep - n
    if keep in (0, n):
        assert np.array_equal(after, pool) and np.array_equal(w2, w)
        return
    stay = set(range(n - min(recent, keep), n))
    for some in (range(min(first, n)), range(n)):
        for t in sorted((t for t in some if t not in stay), key=lambda t: (-flat[t], t)):
            if len(stay) < keep:
                stay.add(t)
    stay = sorted(stay)
    k2, v2, _ = o8.rows(after, table[0], keep)
    # codes of rows from blocks of other scales are rounded once more
    assert (np.abs(k2 - k[stay]) <= 2.0 ** -4 * np.abs(k[stay]) + 1e-4).all()
    assert (np.abs(v2 - v[stay]) <= 2.0 ** -4 * np.abs(v[stay]) + 1e-4).all()
    raw = w[table[0]].reshape(-1)
    assert np.array_equal(w2[table[0]].reshape(-1)[:keep], raw[stay]) and np.array_equal(w2[table[0]].reshape(-1)[keep:], raw[keep:])


def test_norm_rotates_as_rope_does():
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((5, 3, 128)), rng.standard_normal(128)
    pos = np.array([0, 1, 7, 1000, -3])
    y, _ = o8.norm_rotate(x, w, pos)
    n = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-6) * w
    for h in range(3):
        assert np.allclose(y[:, h], oracle.rope(n[:, h], pos, 10000.0))
    assert np.allclose((y ** 2).sum(-1), (n ** 2).sum(-1))
    assert np.allclose(o8.norm_rotate(x, None, None, rope_base=0.0)[0], x)


def test_writes_pass_over_skipped_entries():
    """A run of a block's entries is one whatever is skipped inside it."""
    rng = np.random.default_rng(5)
    pool = rng.integers(0, 256, (2, 1, o8.PAGE_BYTES)).astype(np.uint8)
    k, v = _rows(rng, 6, 1, 3.0), _rows(rng, 6, 1)
    k[3] *= 100
    for slot, src in (([0, -1, 1, 2], None), ([0, 128, 1, 2], None), ([0, 64, 1, 2], [0, -1, 2, 3]), ([0, 2, 1, 2], [0, 6, 2, 3])):
        src = np.arange(4) if src is None else np.array(src)
        want = o8.write(pool, k, v, [0, 1, 2], [0, 2, 3])
        assert np.array_equal(o8.write(pool, k, v, slot, src), want)
