"""The 8-bit paged cache at its edges on the GPU, against the oracle: rows whose scores are
all -infinity, values and norms near the ends of fp32's range, entries that are skipped
inside a block, and calls without rows."""
import numpy as np
import pytest
import torch

from gpu_pipeline import dev, host, say
from oracle import paged8 as o8

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_17139_amd as fc  # noqa: E402
from test_paged import bf16, f64, on_gpu, trees  # noqa: E402
from test_paged8 import BF, D, INF, _norm, attend, make_pool, same_pool  # noqa: E402


# ------------------------------------------------------------- attention --

def _one_sided(rng, n_pages, Hkv, dim, sign):
    """Pages of random rows whose `dim` has one sign everywhere, and is not 0."""
    k, v = (bf16(rng, 64 * n_pages, Hkv, D) for _ in "kv")
    k[..., dim] = sign * (k[..., dim].abs() + 1)
    pool = torch.zeros((n_pages, Hkv, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), dev(np.arange(64 * n_pages, dtype=np.int32)))
    return pool


@pytest.mark.parametrize("R,H,Hkv,lens", [
    (1, 1, 1, [1]), (1, 8, 2, [130, 0]), (4, 8, 2, [70, 200]), (9, 4, 1, [64, 33]), (30, 1, 1, [100]),   # pages a wave
    (1, 4, 1, [3001]), (7, 4, 1, [1300, 5]), (20, 2, 1, [2500]),                                        # in parts
    (65, 4, 2, [100, 0]), (70, 2, 1, [64]), (130, 1, 1, [200]), (65, 2, 1, [2049]),                     # through LDS
], ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("value", [INF, -INF])
def test_rows_whose_scores_are_all_minus_infinity(R, H, Hkv, lens, value):
    """An infinity in a query whose scores all become -infinity shows in its row, and in
    no other; a row that may see nothing is 0 whatever its query holds."""
    rng = np.random.default_rng(R + H + sum(lens))
    B, dim, sign = len(lens), 3, -np.sign(value)
    pool = _one_sided(rng, 5, Hkv, dim, sign)
    q, kt = bf16(rng, B, R, H, D), bf16(rng, B, R, Hkv, D)
    kt[..., dim] = sign * (kt[..., dim].abs() + 1)
    q[:, 0, 0, dim] = value
    q[:, R - 1, H - 1, dim] = value
    q[:, R // 2, H // 2, dim] = value
    table = rng.integers(0, 5, (B, -(-max(lens) // 64))).astype(np.int32)
    say(f"scores of -infinity R={R} H={H} lens={lens} {value}")
    got = attend(rng, B, R, H, Hkv, lens, pool=pool, table=table, q=q, kt=kt, max_len=max(lens))
    assert np.isnan(got[:, 0, 0]).all() and np.isnan(got[:, R - 1, H - 1]).all()
    assert np.isnan(got).any(-1).sum() <= 3 * B
    t = trees(rng, B, R)
    t["mask"][:, R // 2] = 0
    attend(rng, B, R, H, Hkv, lens, t, pool=pool, table=table, q=q, kt=kt, max_len=max(lens))
    # nothing but absent pages, and masks that leave a row nothing
    got = attend(rng, B, R, H, Hkv, lens, t, pool=pool, table=np.full_like(table, -1), q=q, kt=kt, max_len=max(lens))
    assert (got[:, R // 2] == 0).all()
    t["num_nodes"][:] = R // 2
    attend(rng, B, R, H, Hkv, lens, t, pool=pool, table=table, q=q, kt=kt, max_len=max(lens))


@pytest.mark.parametrize("R,H,Hkv,lens", [(1, 8, 2, [130, 0]), (9, 4, 1, [64, 33]), (30, 1, 1, [100]), (1, 4, 1, [3001]),
                                          (20, 2, 1, [2500]), (65, 4, 2, [100, 0]), (65, 2, 1, [2049])],
                         ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("side", [1, 0])
def test_infinities_in_queries_and_keys(R, H, Hkv, lens, side):
    """The same with scores of +infinity alone or of both signs, in queries and in the
    tree's keys: NaN in the rows that have or see them, nothing elsewhere."""
    rng = np.random.default_rng(R + H + sum(lens) + side)
    B, dim = len(lens), 7
    pool = _one_sided(rng, 5, Hkv, dim, 1) if side else make_pool(rng, 5, Hkv)
    q, kt = bf16(rng, B, R, H, D), bf16(rng, B, R, Hkv, D)
    if side:
        kt[..., dim] = kt[..., dim].abs() + 1
    table = rng.integers(0, 5, (B, -(-max(lens) // 64))).astype(np.int32)
    one = q.clone()
    one[:, R // 2, H - 1, dim], one[:, 0, 0, dim] = INF, INF
    say(f"infinities in queries R={R} H={H} lens={lens} side={side}")
    t = trees(rng, B, R)
    got = attend(rng, B, R, H, Hkv, lens, t, pool=pool, table=table, q=one, kt=kt, max_len=max(lens))
    assert np.isnan(got[0, R // 2, H - 1]).all() and np.isnan(got).any(-1).sum() <= 2 * B
    high = kt.clone()                               # q's largest dims meet an infinity of their sign
    q[..., dim] = q[..., dim].abs() + 0.5
    high[:, R // 2, :, dim] = INF
    got = attend(rng, B, R, H, Hkv, lens, t, pool=pool, table=table, q=q, kt=high, max_len=max(lens))
    sees = t["mask"][:, :, R // 2] == 1
    assert (np.isnan(got).all((2, 3)) == sees).all() and not np.isnan(got[~sees]).any()


@pytest.mark.parametrize("R,H,n", [(1, 2, 300), (1, 2, 3001), (20, 1, 3001), (20, 2, 3001), (65, 2, 300), (65, 1, 2500)])
def test_keys_of_score_minus_infinity_beside_others(R, H, n):
    """Pages, tree rows, or both whose scores are -infinity count for nothing beside keys
    of finite scores, wherever they lie: as if they were absent or masked."""
    rng = np.random.default_rng(R + n)
    width = -(-n // 64)
    k, v = bf16(rng, 64 * 6, 1, D), bf16(rng, 64 * 6, 1, D)
    k[..., 3] = 0
    k[:192, :, 3] = -2.0 ** 70          # pages 0 to 2; times 2^70 less than fp32 holds
    pool = torch.zeros((6, 1, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), dev(np.arange(384, dtype=np.int32)))
    q, kt, vt = bf16(rng, 1, R, H, D), bf16(rng, 1, R, 1, D), bf16(rng, 1, R, 1, D)
    q[..., 3] = 2.0 ** 70
    kt[..., 3] = 0
    low = kt.clone()
    low[..., 3] = -INF
    t = dict(trees(rng, 1, R))
    alone = {**t, "mask": np.zeros_like(t["mask"])}
    plen, page = np.array([n], np.int32), rng.integers(3, 6, width)
    for name, finite in (("all but one", np.arange(width) == width // 2), ("the first", np.arange(width) == 0),
                         ("the last", np.arange(width) == width - 1), ("every other", np.arange(width) % 2 == 0),
                         ("the second half", np.arange(width) >= width // 2)):
        say(f"-infinity beside others R={R} n={n}: finite pages are {name}")
        table = np.where(finite, page, page - 3).astype(np.int32)[None]
        there = np.where(finite, page, -1).astype(np.int32)[None]
        for keys, tree in ((low, t), (kt, t), (kt, alone)):
            got, want = [], []
            for tab, tr, to in ((table, tree, got), (there, alone if keys is low else tree, want)):
                lse = torch.empty((1, R, H), device="cuda")
                to += [fc.fc_paged_byte_attention(q.cuda(), keys.cuda(), vt.cuda(), pool, dev(tab), dev(plen), tree=on_gpu(tr),
                                                  lse=lse), lse]
            assert not torch.isnan(want[0]).any() and want[0].any()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the tree's rows alone are finite
    say(f"-infinity beside others R={R} n={n}: finite are the tree's rows")
    table = (page - 3).astype(np.int32)[None]
    got, want = (fc.fc_paged_byte_attention(q.cuda(), kt.cuda(), vt.cuda(), pool, dev(x), dev(plen), tree=on_gpu(t))
                 for x in (table, np.full_like(table, -1)))
    assert torch.equal(got, want) and got.any() and not torch.isnan(got).any()


@pytest.mark.parametrize("q0,q1", [(9.6875, 0.3125), (8.6875, 0.640625)])
def test_sums_of_large_values_over_the_longest_prefix(q0, q1):
    """Values just below 2^78 over as many tokens as a table may hold, with weights that
    are many times a row's first: 1.75 * 2^19 and 1.75 * 2^17 (rounded to bf16) where the
    first page's are 1.  Their sum reaches 2^128 unless the row is scaled down on its way."""
    n, value = 2 ** 31 - 65, 1.5 * 2.0 ** 77
    pages = -(-n // 64)
    k = torch.zeros((128, 1, D))
    k[64:, 0, 0], k[64:, 0, 1] = 16, 1
    pool = torch.zeros((2, 1, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_byte_write(pool, k.to(BF).cuda(), torch.full((128, 1, D), value).to(BF).cuda(),
                           dev(np.arange(128, dtype=np.int32)))
    # each of a workgroup's eight waves begins with a page of the small weights, in each of
    # the 128 parts of 2^18 pages that a prefix of this length is cut into
    table = (torch.arange(pages, dtype=torch.int32, device="cuda") % 2 ** 18 >= 8).int()[None]
    q = torch.zeros((1, 1, 1, D))
    q[..., 0], q[..., 1] = q0, q1
    vt, lse = torch.full((1, 1, 1, D), value).to(BF).cuda(), torch.empty((1, 1, 1), device="cuda")
    say(f"sums of large values, score {16 * q0 + q1}")
    got = fc.fc_paged_byte_attention(q.to(BF).cuda(), torch.zeros_like(vt), vt, pool, table, dev(np.array([n], np.int32)),
                                     max_len=n, lse=lse)
    # a wave adds 2^15 times to a sum, 2^-24 of it off each time, above the line and below
    # it; the result is bf16
    assert ((got.float().double() - value).abs() <= (2.0 ** -8 + 2.0 ** -8) * value).all()
    few = 128 * 8 * 64
    want = np.log((n - few) * np.exp((16 * q0 + q1) / np.sqrt(D)) + few + 1)
    assert abs(float(lse) - want) <= 2.0 ** -9 + 2.0 ** -20


# ------------------------------------------------------------------- norm --

@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
@pytest.mark.parametrize("n", [1, 40])
def test_norms_at_both_ends_of_the_range(n, eps):
    """Heads whose squares, or their sum, are more than fp32 holds or less: the result is
    what the formula gives, whatever the size of the numbers."""
    rng = np.random.default_rng(n)
    powers = np.array([126, 100, 66, 64, 60, 0, -40, -45, -50, -64, -70, -100, -126, -130])
    say(f"norms at both ends n={n} eps={eps}")
    q = torch.from_numpy(rng.uniform(0.5, 1.9, (n, len(powers), D)) * rng.choice([-1, 1], (n, len(powers), D)) *
                         2.0 ** powers[:, None]).to(BF)
    k = q.flip(1).clone()
    k[..., 5::9] = 0                                # a few alone
    k[:, :, 64:] *= 2.0 ** -20
    w = [1 + bf16(rng, D, scale=0.3) for _ in "qk"]
    pos = rng.integers(0, 100_000, n).astype(np.int32)
    _norm(q, k, *w, pos, eps=eps)
    _norm(q, k, *w, None, eps=eps, rope_base=0.0)
    odd = q.clone()                                 # what is not finite leaves no other head
    odd[0, 0, 3], odd[0, 1, 70], odd[0, -1, 9], odd[0, 3] = INF, -INF, float("nan"), 0
    got = f64(fc.fc_norm_rotate(odd.cuda(), None, w[0].cuda(), None, dev(pos), eps=eps)[0])
    rest = f64(fc.fc_norm_rotate(q.cuda(), None, w[0].cuda(), None, dev(pos), eps=eps)[0])
    assert np.array_equal(got[1:], rest[1:]) and np.array_equal(got[0, 4:-1], rest[0, 4:-1])
    assert np.isnan(got[0, 0, [3, 67]]).all() and np.isnan(got[0, 1, [6, 70]]).all() and np.isnan(got[0, -1]).all()
    assert np.isnan(got[0, 3]).all() if eps == 0 else (got[0, 3] == 0).all()


# ---------------------------------------------------------------- weights --

@pytest.mark.parametrize("H,Hkv,lens,adds", [(4, 2, [70, 5, 90, 0], [9, 0, -20, 1]), (1, 1, [0], [1]), (8, 2, [30], [300])])
@pytest.mark.parametrize("rows,entries", [(0, None), (0, 0), (0, 7), (7, 0)])
def test_weights_of_calls_without_rows(H, Hkv, lens, adds, rows, entries):
    """New tokens that no row pays for weigh nothing, though their places held other
    tokens' weights: also where there are no rows at all, or no entries."""
    rng = np.random.default_rng(sum(lens) + rows)
    new, B = [n + a for n, a in zip(lens, adds)], len(lens)
    n_pages = sum(-(-n // 64) for n in new) + 2
    pool, perm, at = make_pool(rng, n_pages, Hkv), rng.permutation(n_pages).astype(np.int32), 0
    table = np.full((B, max(-(-n // 64) for n in new) + 1), -1, np.int32)
    for b, n in enumerate(new):
        m = -(-n // 64)
        table[b, :m] = perm[at:at + m]
        at += m
    cu = np.concatenate([[0], np.cumsum(np.maximum(adds, 0))]).astype(np.int32)
    src = None if entries is None else rng.integers(0, 7, entries).astype(np.int32)
    w = rng.uniform(1, 3, (n_pages, Hkv, 64)).astype(np.float32)
    q, lse = bf16(rng, rows, H, D), rng.uniform(0, 8, (rows, H)).astype(np.float32)
    say(f"weights without rows H={H} lens={lens} adds={adds} rows={rows} entries={entries}")
    got = dev(w)
    fc.fc_paged_byte_weights(got, q.cuda(), dev(lse), pool, dev(table), dev(np.array(lens, np.int32)),
                             dev(np.array(new, np.int32)), dev(cu), src=None if src is None else dev(src))
    want, _ = o8.weights(w, f64(q), lse, host(pool), table, lens, new, cu, src)
    assert (want != w).any() and np.array_equal(host(got), want.astype(np.float32))
    # on another stream, and captured
    again, side = dev(w), torch.cuda.Stream()
    args = (q.cuda(), dev(lse), pool, dev(table), dev(np.array(lens, np.int32)), dev(np.array(new, np.int32)), dev(cu))
    kw = dict(src=None if src is None else dev(src))
    torch.cuda.synchronize()
    fc.fc_paged_byte_weights(again, *args, **kw, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(again, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fc.fc_paged_byte_weights(again, *args, **kw)
    for i in range(3):
        again.copy_(dev(w))
        graph.replay()
        busy = torch.full((1 << 20,), 7, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        assert torch.equal(again, got), i
        del busy


# ------------------------------------------------------------------ write --

@pytest.mark.parametrize("gap", [1, 2, 31, 32, 33, 63, 64, 65, 200, 600, 5000])
@pytest.mark.parametrize("kind", ["slots", "rows", "slots and rows", "a block's first slot", "another block's"])
def test_skipped_entries_inside_a_block(gap, kind):
    """Entries of one block with skipped ones among them - outside the pool, of a row that
    is not there, or both, one or thousands - are one run, wherever it begins and ends."""
    rng = np.random.default_rng(gap)
    Hkv, n_pages = 3, 6
    say(f"skipped entries, {gap} of {kind}")
    for first in (0, 5):                                       # the block's first row is written, or not
        for lead in (0, 1, 29, 30, 31, 32, 39, 70):            # entries of other blocks before it
            rows = first + rng.permutation(32 - first)[:rng.integers(2, 33 - first)]
            if first == 0 and lead % 2:
                rows = rows[::-1]
            at = np.sort(rng.integers(0, len(rows) + 1, 3))    # where skipped ones lie
            slot, live = [64 + x for x in range(32)][:lead] + [128 + x for x in range(lead - 32)], []
            live += [True] * len(slot)
            for i, t in enumerate(rows):
                for _ in range(int((at == i).sum())):
                    slot += [-7] * gap
                    live += [False] * gap
                slot.append(32 + int(t))
                live.append(True)
            slot += [-1] * (gap if lead % 3 else 0) + [192, 193]
            live += [False] * (gap if lead % 3 else 0) + [True, True]
            slot, live = np.array(slot), np.array(live)
            n = len(slot)
            src, bad = rng.integers(0, 100, n), ~live
            if kind == "slots":
                slot[bad] = rng.choice([-1, -2 ** 31, 2 ** 31 - 1, 64 * n_pages], bad.sum())
            else:
                src[bad] = rng.choice([-1, 100, -2 ** 31, 2 ** 31 - 1], bad.sum())
                if kind == "slots and rows":
                    slot[bad] = rng.choice([-1, 33, 64 * n_pages + 5], bad.sum())
                elif kind == "a block's first slot":
                    slot[bad] = 32
                elif kind == "another block's":
                    slot[bad] = rng.choice([5, 64, 300], bad.sum())
                else:
                    slot[bad] = 32 + rng.integers(0, 32, bad.sum())
            k, v = bf16(rng, 100, Hkv, D), bf16(rng, 100, Hkv, D, scale=30.0)
            pool = make_pool(rng, n_pages, Hkv)
            want = o8.write(host(pool), f64(k), f64(v), slot, src)
            # at every distance from a 16-byte boundary, with slots of the block ahead and behind
            at = 4 + lead % 4
            near = dev(np.concatenate([np.full(at, 40), slot, np.full(8, 41)]).astype(np.int32))[at:at + n]
            fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), near, src=dev(src.astype(np.int32)))
            same_pool(pool, want, (first, lead))


def test_skipped_entries_of_whole_calls():
    """A padded batch: every sequence's rows in a place of their own, most of them skipped;
    calls of nothing but skipped entries; rows that follow one another without src."""
    rng = np.random.default_rng(3)
    B, R, Hkv, n_pages = 40, 65, 2, 60
    pool = make_pool(rng, n_pages, Hkv)
    slot = np.full((B, R), -1)
    for b in range(B):
        on = np.sort(rng.permutation(R)[:rng.integers(0, 9)])
        slot[b, on] = 64 * b + 30 + np.arange(len(on)) - (28 if b % 3 == 0 else 0)
    slot = slot.reshape(-1)
    k, v = bf16(rng, B * R, Hkv, D), bf16(rng, B * R, Hkv, D, scale=20.0)
    say("skipped entries of a padded batch")
    want = o8.write(host(pool), f64(k), f64(v), slot)
    fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), dev(slot.astype(np.int32)))
    same_pool(pool, want)
    fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), torch.full((100_000,), -1, dtype=torch.int32, device="cuda"))
    same_pool(pool, want)
    say("skipped entries, a hundred thousand around each of a few")
    for at in range(4):
        slot = np.full(400_000 + at, -1)
        slot[[7, 100_000, 200_001, 200_002, 399_999]] = [64, 70, 65, 130, 128]
        near = dev(np.concatenate([np.full(at, 131), slot, np.full(8, 132)]).astype(np.int32))[at:at + len(slot)]
        src = rng.integers(0, B * R, len(slot))
        want = o8.write(host(pool), f64(k), f64(v), slot, src)
        fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), near, src=dev(src.astype(np.int32)))
        same_pool(pool, want, at)
