"""Pins of the paged cache's oracle: the 4-bit rounding against a search over
all values, page bytes back and forth, plans against a free list kept in a
Python list, and attention against the dense oracle on the same keys."""
import numpy as np
import pytest

import oracle

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def test_rounding_is_the_nearest_value_of_the_smallest_scale():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 128)) * 2.0 ** rng.integers(-40, 40, (50, 1))
    code, scale = oracle.fp4_round(x)
    v = oracle.fp4_value(code, scale)
    for r in range(50):
        for g in range(4):
            a = x[r, 32 * g:32 * g + 32]
            s = 2.0 ** (float(scale[r, g]) - 127)
            assert np.abs(a).max() <= 7 * s and np.abs(a).max() > 3.5 * s
            near = np.abs(np.abs(a)[:, None] - VALUES * s).min(1)
            assert np.array_equal(np.abs(np.abs(a) - np.abs(v[r, 32 * g:32 * g + 32])), near)
            assert (np.signbit(v[r, 32 * g:32 * g + 32]) == np.signbit(a)).all()


def test_rounding_ties_limits_and_the_not_finite():
    x = np.zeros((1, 128))
    x[0, :10] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -5.0]
    code, scale = oracle.fp4_round(x)
    assert scale[0, 0] == 127 and list(oracle.fp4_value(code, scale)[0, :10]) == [0, 1, 1, 2, 2, 4, 4, 6, 0, -4]
    assert scale[0, 1] == 2 and (code[0, 32:] == 0).all()      # a group of zeros
    x[0, 0] = np.nextafter(7.0, 8.0)
    assert oracle.fp4_round(x)[1][0, 0] == 128
    x[0, 40], x[0, 70] = 3e38, np.inf
    x[0, 100] = np.nan
    code, scale = oracle.fp4_round(x)
    assert list(scale[0]) == [128, 252, 255, 255]
    v = oracle.fp4_value(code, scale)[0]
    assert v[40] == 6 * 2.0 ** 125 and np.isnan(v[64:]).all()
    assert oracle.fp4_round(np.full((1, 32), 2.0 ** -128))[1][0, 0] == 2  # below half the least value: 0


def test_page_bytes_hold_what_they_are_given():
    rng = np.random.default_rng(2)
    parts = [rng.integers(0, 16, (64, 128)).astype(np.uint8), rng.integers(0, 256, (64, 4)).astype(np.uint8),
             rng.integers(0, 16, (64, 128)).astype(np.uint8), rng.integers(0, 256, (64, 4)).astype(np.uint8)]
    page = oracle.page_of(*parts)
    for a, b in zip(parts, oracle.page_parts(page)):
        assert np.array_equal(a, b)
    assert page[3 * 64 + 10] == parts[0][3, 20] + 16 * parts[0][3, 21]
    assert page[8192 + (2 * 16 + 37 % 16) * 4 + 2] == parts[1][37, 2]      # key token 37, group 2
    assert page[8448 + ((37 % 16) * 4 + 2) * 4 + 2] == parts[3][37, 2]     # value token 37, group 2


@pytest.mark.parametrize("seed", range(6))
def test_plans_keep_a_free_list(seed):
    """Steps of appends, cuts and ends with a small pool: the tables name each
    page once, free and held pages make up the pool, and every token's slot is
    where its table says."""
    rng = np.random.default_rng(seed)
    B, max_pages, n_pages = 7, 5, 17
    length, table = np.zeros(B, np.int32), np.full((B, max_pages), -1, np.int32)
    queue, ends = rng.permutation(n_pages).astype(np.int32), np.array([0, n_pages])
    for step in range(40):
        add = rng.integers(-100, 130, B).astype(np.int32)
        add[rng.random(B) < 0.2] = 0
        n_slots = int(rng.integers(0, 500))
        r = oracle.paged_plan(length, add, table, queue, ends, n_slots)
        free = [int(queue[i % n_pages]) for i in range(ends[0], ends[1])]
        taken = back = 0
        for b in range(B):
            new = max(int(length[b] + add[b]), 0)
            pages = lambda n: -(-int(n) // 64)  # noqa: E731
            if add[b] > 0:
                assert r["len"][b] in (length[b], new)
                served = r["len"][b] == new
                got = r["slot"][min(r["cu"][b], n_slots):min(r["cu"][b] + add[b], n_slots)]
                if served:
                    need = pages(new) - pages(length[b])
                    assert list(r["table"][b, pages(length[b]):pages(new)]) == free[taken:taken + need]
                    taken += need
                    for t in range(add[b]):
                        p = int(length[b]) + t
                        assert got[t] == 64 * r["table"][b, p // 64] + p % 64
                else:
                    assert (got == -1).all()
                    assert pages(new) > max_pages or r["cu"][b] + add[b] > n_slots or \
                        taken + pages(new) - pages(length[b]) > len(free) or r["ends"][0] < ends[1]
            else:
                assert r["len"][b] == new
                back += pages(length[b]) - pages(new)
        assert list(r["ends"]) == [ends[0] + taken, ends[1] + back]
        length, table, queue, ends = r["len"], r["table"], r["queue"], r["ends"]
        held = [int(table[b, p]) for b in range(B) for p in range(-(-int(length[b]) // 64))]
        left = [int(queue[i % n_pages]) for i in range(ends[0], ends[1])]
        assert sorted(held + left) == list(range(n_pages))


def test_plan_takes_the_accepted_path():
    #      0 - 1 - 2        rows in the order parents come before children
    #        \ 3 - 4
    parent = [-1, 0, 1, 0, 3]
    mask = np.zeros((1, 5, 5), np.int32)
    for i, p in enumerate(parent):
        mask[0, i] = mask[0, p] if p >= 0 else 0
        mask[0, i, i] = 1
    table, queue = np.full((1, 2), -1, np.int32), np.arange(3, dtype=np.int32)
    r = oracle.paged_plan([62], [3], np.array([[2, -1]], np.int32), queue, [0, 2], 5, mask, [4])
    assert list(r["src"]) == [0, 3, 4, -1, -1] and list(r["slot"]) == [2 * 64 + 62, 2 * 64 + 63, 0, -1, -1]
    assert list(r["pos"]) == [62, 63, 64, -1, -1] and list(r["table"][0]) == [2, 0]
    assert oracle.paged_plan([0], [3], table, queue, [0, 3], 5, mask, [1])["src"].tolist() == [0, 1, -1, -1, -1]


@pytest.mark.parametrize("rope_base", [0.0, 10000.0])
def test_attention_is_the_dense_one_on_the_cached_values(rope_base):
    rng = np.random.default_rng(3)
    B, R, H, Hkv, D = 2, 5, 4, 2, 128
    lens = [70, 0]
    pool = np.zeros((3, Hkv, oracle.PAGE_BYTES), np.uint8)
    table = np.array([[2, 0], [-1, -1]], np.int32)
    k, v = rng.standard_normal((2, 70, Hkv, D))
    slot = [64 * table[0, p // 64] + p % 64 for p in range(70)]
    pool = oracle.paged_write(pool, k, v, slot, np.arange(70), rope_base=rope_base)
    kc, vc, there = oracle.paged_rows(pool, table[0], 70)
    assert there.all()
    want = oracle.rope(k.transpose(1, 0, 2), np.arange(70), rope_base).transpose(1, 0, 2) if rope_base else k
    assert np.abs(kc - want).max() < 0.17 * np.abs(want).max()      # half a step of two in seven
    dense = [np.zeros((B, 70, Hkv, D)) for _ in "kv"]
    dense[0][0], dense[1][0] = kc, vc
    q, kt, vt = (rng.standard_normal((B, R, h, D)) for h in (H, Hkv, Hkv))
    mask = np.tril(np.ones((B, R, R), np.int32))
    mask[:, 2] = [1, 0, 1, 0, 0]
    pos = np.tile([0, 1, 1, 2, 3], (B, 1))
    got, mean, _ = oracle.paged_attention(q, kt, vt, pool, table, lens, [5, 3], mask, pos, rope_base=rope_base)
    if rope_base:
        ref = oracle.tree_attention(q, kt, vt, *dense, lens, [5, 3], mask, pos, rope_base)
        assert np.allclose(got, ref, atol=1e-12)
    assert (np.abs(got) <= mean + 1e-12).all() and (got[1, 3:] == 0).all()
    # an absent page's keys are absent, a chain is the lower triangle, and a longest length cuts prefixes off
    lost = oracle.paged_attention(q, kt, vt, pool, np.array([[2, 7], [0, 0]]), [70, 0], [5, 3], mask, pos)[0]
    cut = oracle.paged_attention(q, kt, vt, pool, table, [64, 0], [5, 3], mask, pos - 0)[0]
    assert not np.allclose(lost[0], cut[0])  # the positions still count them
    a = oracle.paged_attention(q, kt, vt, pool, table, lens, max_len=64, rope_base=0.0)[0]
    b = oracle.paged_attention(q, kt, vt, pool, table, [64, 0], mask=np.tril(np.ones((B, R, R))),
                               pos_ids=np.tile(np.arange(R), (B, 1)), rope_base=0.0)[0]
    assert np.array_equal(a, b)
