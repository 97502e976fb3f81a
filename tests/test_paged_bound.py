"""The bound that paged attention is held to: a model of the kernel's 6-bit parts
keeps it, and one with a part, a product or a rotation missing does not."""
import numpy as np
import pytest

import oracle
import paged_bound as pb

D = pb.D


def test_parts_leave_what_they_should():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((400, D)) * 2.0 ** rng.integers(-30, 30, (400, 1)) * rng.choice([1, 1e-2, 1e-4], (400, D))
    part, left, f = pb.parts_of(x)
    top = np.repeat(np.abs(x).reshape(400, 4, 32).max(-1), 32, axis=-1)
    assert (top <= 7.5 * f).all() and (top * (1 + 2.0 ** -19) > 3.75 * f).all()
    for i, most in enumerate((-2, -7, -12)):
        assert (np.abs(left[i]) <= 2.0 ** most * f).all() and (np.abs(left[i]) > 2.0 ** (most - 1) * f).any()
    assert np.allclose(sum(part) + left[2], x, rtol=0, atol=0)
    assert (np.abs(left[2]) <= 2.0 ** -13 * top).all()
    # three of the nine products of a tree key's parts are not added
    rest = sum(np.abs(part[i][:200]) * np.abs(part[j][200:]) for i, j in ((1, 2), (2, 1), (2, 2)))
    assert (rest <= 2.0 ** -11 * top[:200] * top[200:]).all()
    assert {(i, j) for i in range(3) for j in range(3)} - set(pb.ALL) == {(1, 2), (2, 1), (2, 2)}


def _cached(rng, B, R, Hkv, n):
    q, k, v, mask = pb.pairs_of_cached_keys(rng, B, R, Hkv, n)
    width = -(-n // 64)
    table = rng.permutation(B * width).astype(np.int32).reshape(B, width)
    pool = np.zeros((B * width, Hkv, oracle.PAGE_BYTES), np.uint8)
    for b in range(B):
        slot = table[b, np.arange(n) // 64] * 64 + np.arange(n) % 64
        pool = oracle.paged_write(pool, k[b], v[b], slot, rope_base=0.0)
    held = oracle.paged_rows(pool, table[0], n)
    assert np.array_equal(held[0], k[0]) and np.array_equal(held[1], v[0])     # they are 4-bit values
    none = np.zeros((B, R, Hkv, D))
    return dict(q=q, k_tree=none, v_tree=none, pool=pool, table=table, prefix_len=[n] * B, mask=mask, rope_base=0.0)


def _tree(rng, B, R, Hkv, base):
    q, kt, vt, mask, pos = pb.pairs_of_tree_keys(rng, B, R, Hkv, base)
    return dict(q=q, k_tree=kt, v_tree=vt, pool=np.zeros((1, Hkv, oracle.PAGE_BYTES), np.uint8),
                table=np.zeros((B, 1), np.int32), prefix_len=[0] * B, mask=mask, pos_ids=pos, rope_base=base)


def _random(rng, B, R, H, Hkv, n, qscale=1.0, rope_base=10000.0):
    k, v = (pb.bf16(rng.standard_normal((64, Hkv, D))) for _ in "kv")
    pool = oracle.paged_write(np.zeros((1, Hkv, oracle.PAGE_BYTES), np.uint8), k, v, np.arange(64), rope_base=0.0)
    row = lambda h, s=1.0: pb.bf16(rng.standard_normal((B, R, h, D)) * s)  # noqa: E731
    return dict(q=row(H, qscale), k_tree=row(Hkv), v_tree=row(Hkv), pool=pool,
                table=np.zeros((B, -(-max(n, 1) // 64)), np.int32), prefix_len=[n] * B, rope_base=rope_base)


@pytest.mark.parametrize("q_parts", [1, 2])
def test_a_lost_part_of_the_query_breaks_the_bound(q_parts):
    s = _cached(np.random.default_rng(2), 2, 3, 2, 70)
    o, bound, norm, model = pb.attention(**s)
    assert pb.within(model, o, bound, norm) == (True, True)
    assert (bound < 0.12).all() and (np.abs(o) < 0.9).all()
    lost = pb.attention(**s, q_parts=q_parts)[3]
    assert not pb.within(lost, o, bound, norm)[0] and not pb.within(lost, o, bound, norm)[1]
    if q_parts == 2:  # what the third part adds has one sign; what the second adds may cancel in a row
        assert not (np.abs(lost - o) <= 3 * bound).any()


@pytest.mark.parametrize("k_parts", [1, 2])
def test_a_lost_part_of_a_tree_key_breaks_the_bound(k_parts):
    s = _tree(np.random.default_rng(3), 2, 6, 2, 10000.0)
    rows = s["pos_ids"] == 0        # those that the keys were made for
    o, bound, norm, model = pb.attention(**s)
    assert pb.within(model, o, bound, norm) == (True, True)
    assert (bound[rows] < 0.12).all() and (np.abs(o[rows]) < 0.9).all()
    lost = pb.attention(**s, k_parts=k_parts)[3]
    assert not pb.within(lost, o, bound, norm)[0] and not pb.within(lost, o, bound, norm)[1]
    if k_parts == 2:  # what the third part adds has one sign; what the second adds may cancel in a row
        assert not (np.abs(lost - o) <= 3 * bound)[rows].any()
    turn = pb.attention(**s, rotate_tree=False)[3]
    assert not pb.within(turn, o, bound, norm)[1]


@pytest.mark.parametrize("lost", [(2, 0), (1, 1), (0, 2), (1, 0), (0, 1)])
def test_a_lost_product_breaks_the_bound(lost):
    """Each of the products of a tree key's parts counts in rows made for it."""
    if lost in ((2, 0), (1, 0)):
        s = _tree(np.random.default_rng(3), 2, 6, 2, 10000.0)
    else:
        q, kt, vt, mask = pb.pairs_of_signs(np.random.default_rng(4), 2, 6, 2, *((1, 4.1875) if lost == (1, 1) else (2, 6.0)))
        s = dict(q=q, k_tree=kt, v_tree=vt, pool=np.zeros((1, 2, oracle.PAGE_BYTES), np.uint8),
                 table=np.zeros((2, 1), np.int32), prefix_len=[0, 0], mask=mask, rope_base=0.0)
    o, bound, norm, model = pb.attention(**s)
    assert pb.within(model, o, bound, norm) == (True, True)
    bad = pb.attention(**s, products=[x for x in pb.ALL if x != lost])[3]
    assert not pb.within(bad, o, bound, norm)[0] and not pb.within(bad, o, bound, norm)[1]


@pytest.mark.parametrize("B,R,H,Hkv,n", [(1, 1, 17, 1, 500), (1, 48, 1, 1, 640), (1, 65, 4, 4, 100), (2, 5, 8, 2, 193)])
def test_random_rows_notice_what_is_wrong(B, R, H, Hkv, n):
    s = _random(np.random.default_rng(R), B, R, H, Hkv, n)
    o, bound, norm, model = pb.attention(**s)
    assert np.allclose(o, oracle.paged_attention(s["q"], s["k_tree"], s["v_tree"], s["pool"], s["table"], s["prefix_len"])[0],
                       atol=1e-12)
    assert pb.within(model, o, bound, norm) == (True, True)
    for wrong in (np.zeros_like(o), pb.attention(**s, q_parts=1)[3], o * 1.02):
        assert not pb.within(wrong, o, bound, norm)[1]
    if R > 1:
        assert not pb.within(pb.attention(**s, rotate_tree=False)[3], o, bound, norm)[1]
