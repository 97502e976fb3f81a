"""The paged 4-bit cache on the GPU against the oracle: plans and written bytes
element by element, attention within bounds that follow from what is rounded."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from gpu_pipeline import dev, host, say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_17139_amd as fc  # noqa: E402

D = fc.FC_TREE_ATTN_HEAD_DIM
BF = torch.bfloat16


def f64(t: torch.Tensor) -> np.ndarray:
    return t.float().cpu().numpy().astype(np.float64)


def bf16(rng, *shape, scale=1.0) -> torch.Tensor:
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(BF)


def trees(rng, B, R, deep=9):
    parent = np.full((B, R), -1)
    pos, mask = np.zeros((B, R), np.int32), np.zeros((B, R, R), np.int32)
    for b in range(B):
        for i in range(R):
            if i:
                ok = np.flatnonzero(pos[b, :i] < deep)
                parent[b, i] = rng.choice(ok)
                pos[b, i] = pos[b, parent[b, i]] + 1
                mask[b, i] = mask[b, parent[b, i]]
            mask[b, i, i] = 1
    return dict(num_nodes=np.full(B, R, np.int32), pos_ids=pos, mask=mask, parent=parent.astype(np.int32))


def on_gpu(tree):
    return None if tree is None else {f: dev(v) for f, v in tree.items()}


# ------------------------------------------------------------------- plan --

def _plan(length, add, table, queue, ends, n_slots, mask=None, last=None):
    """One plan on both sides, every result equal; returns the oracle's."""
    want = oracle.paged_plan(length, add, table, queue, ends, n_slots, mask, last)
    t, q = dev(table), dev(queue)
    args = (dev(length), dev(add), t, q, dev(np.asarray(ends, np.int64)), n_slots)
    kw = {} if mask is None else dict(tree=dict(mask=dev(mask)), last_node=dev(last))
    for again in range(2):  # a plan repeated is the same plan
        got = fc.fc_paged_plan(*args, **kw)
        torch.cuda.synchronize()
        for f in fc.PLAN_FIELDS:
            assert np.array_equal(host(got[f]), want[f]), (f, again)
        assert np.array_equal(host(t), want["table"]) and np.array_equal(host(q), want["queue"]), again
    return want


@pytest.mark.parametrize("B,max_pages,n_pages,most", [
    (1, 1, 1, 64), (1, 4, 9, 200), (7, 5, 17, 130), (63, 40, 600, 1500), (300, 6, 700, 90), (700, 3, 1500, 40),
    (5, 400, 1500, 9000),
])
def test_plan_steps_match_oracle(B, max_pages, n_pages, most):
    """Steps of appends, cuts and ends on a pool that is often short: over
    several windows of the slot map, several chunks of sequences, and a ring
    that goes round."""
    rng = np.random.default_rng(B)
    length, table = np.zeros(B, np.int32), np.full((B, max_pages), -1, np.int32)
    queue, ends = rng.permutation(n_pages).astype(np.int32), np.array([0, n_pages], np.int64)
    for step in range(10):
        add = rng.integers(-most // 2, most, B).astype(np.int32)
        add[rng.random(B) < 0.3] = 0
        add[rng.random(B) < 0.1] = -2 ** 31
        total = int(np.maximum(add, 0).sum())
        n_slots = [total, total + 77, total // 2, 0][step % 4]
        say(f"plan B={B} step={step} tokens={total} slots={n_slots}")
        r = _plan(length, add, table, queue, ends, n_slots)
        length, table, queue, ends = r["len"], r["table"], r["queue"], r["ends"]
        if step == 5:  # numbers of a pool long in use
            ends = ends + n_pages * (2 ** 40 // n_pages)


def test_plan_of_nothing():
    none = np.zeros(0, np.int32)
    for n_slots in (0, 5, 3000):
        say(f"plan of no sequences, {n_slots} slots")
        _plan(none, none, np.zeros((0, 4), np.int32), np.arange(3, dtype=np.int32), [1, 3], n_slots)
    _plan(np.array([5, 0], np.int32), np.zeros(2, np.int32), np.array([[0, -1], [-1, -1]], np.int32),
          np.array([1, 2, 0], np.int32), [3, 5], 0)


@pytest.mark.parametrize("B,R", [(1, 1), (3, 65), (70, 33), (9, 256), (130, 17)])
def test_plan_of_accepted_rows_matches_oracle(B, R):
    rng = np.random.default_rng(R)
    t = trees(rng, B, R)
    last = rng.integers(0, R, B).astype(np.int32)
    add = np.array([t["pos_ids"][b, last[b]] + 1 for b in range(B)], np.int32)
    last[rng.random(B) < 0.1] = -1          # no such row: no source
    last[rng.random(B) < 0.05] = R
    add[rng.random(B) < 0.1] += 1           # more tokens than rows
    length = rng.integers(0, 500, B).astype(np.int32)
    held = -(-length // 64)
    perm = rng.permutation(int(held.sum()) + B).astype(np.int32)
    table = np.full((B, 9), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    queue = np.concatenate([perm[at:], np.full(at, -1, np.int32)])
    say(f"plan of accepted rows B={B} R={R}")
    _plan(length, add, table, queue, [0, B], int(add.sum()) + 3, t["mask"], last)


def test_plan_of_many_sequences():
    """More sequences than a workgroup has threads, most of them short, and more
    accepted paths than one: chunks whose sums go on, and slots that run out."""
    rng = np.random.default_rng(3)
    B = 2600
    length = rng.integers(0, 150, B).astype(np.int32)
    held = -(-length // 64)
    perm = rng.permutation(int(held.sum()) + 900).astype(np.int32)
    table, at = np.full((B, 4), -1, np.int32), 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    queue = np.concatenate([perm[at:], np.full(at, -1, np.int32)])
    add = rng.integers(-70, 40, B).astype(np.int32)
    add[rng.random(B) < 0.02] = 200         # more than a table holds, at times
    total = int(np.maximum(add, 0).sum())
    for n_slots in (total, total // 3, 1, total + 5000):
        say(f"plan of {B} sequences, {n_slots} of {total} slots")
        _plan(length, add, table, queue, [0, 900], n_slots)
    t = trees(rng, 1100, 9)
    last = rng.integers(-2, 10, 1100).astype(np.int32)
    add = np.array([t["pos_ids"][b, min(max(last[b], 0), 8)] + 1 for b in range(1100)], np.int32)
    say("plan of 1100 accepted paths, some of no row")
    _plan(length[:1100], add, table[:1100], queue, [0, 900], int(add.sum()), t["mask"], last)


def test_plan_of_bad_tables_and_lengths():
    """Lengths past the table, table entries outside the pool, a ring whose
    ends say more than it can hold: nothing outside the buffers is touched and
    slots that do not exist are -1."""
    table = np.array([[7, -3, 1], [0, 1, 2]], np.int32)
    queue = np.array([0, 1, 2, 3], np.int32)
    say("plan of bad tables")
    r = _plan(np.array([10, -5], np.int32), np.array([20, 3], np.int32), table, queue, [0, 4], 30)
    assert (r["slot"][:20] == -1).all()
    _plan(np.array([10 ** 9, 5], np.int32), np.array([1, 3], np.int32), table, queue, [0, 4], 30)
    got = fc.fc_paged_plan(dev(np.array([0, 0], np.int32)), dev(np.array([192, 192], np.int32)), dev(table), dev(queue),
                           dev(np.array([5, 10 ** 6], np.int64)), 400)
    torch.cuda.synchronize()
    assert host(got["len"]).tolist() == [192, 0]    # four pages at most, whatever the ends say


# ---------------------------------------------------------- write and read --

def _write_case(rng, n_pages, Hkv, n_src, n, rope_base, scale=1.0, use_src=True, k=None, v=None):
    k = bf16(rng, n_src, Hkv, D, scale=scale) if k is None else k
    v = bf16(rng, n_src, Hkv, D, scale=scale) if v is None else v
    slot = rng.permutation(n_pages * 64)[:n].astype(np.int32)
    slot[rng.random(n) < 0.1] = -1
    slot[rng.random(n) < 0.05] += 64 * n_pages
    src = rng.integers(-1, n_src + 1, n).astype(np.int32) if use_src else None
    pos = rng.integers(0, 200_000, n).astype(np.int32)
    before = rng.integers(0, 256, (n_pages, Hkv, fc.FC_PAGE_HEAD_BYTES)).astype(np.uint8)
    pool = dev(before)
    fc.fc_paged_write(pool, k.cuda(), v.cuda(), dev(slot), dev(pos), src=None if src is None else dev(src),
                      rope_base=rope_base)
    torch.cuda.synchronize()
    want = oracle.paged_write(before, f64(k), f64(v), slot, pos, src, rope_base)
    # a slot of -1 that was moved up by the pool's size is the last one, and may be
    # another entry's too: what a slot given twice holds is left open, so it is not compared
    row = np.arange(n) if src is None else src
    taken = slot[(slot >= 0) & (slot < 64 * n_pages) & (row >= 0) & (row < n_src)]
    for sl in [x for x in set(taken.tolist()) if (taken == x).sum() > 1]:
        for h in range(Hkv):
            parts, got = oracle.page_parts(want[sl // 64, h]), oracle.page_parts(host(pool)[sl // 64, h])
            for a, b in zip(parts, got):
                a[sl % 64] = b[sl % 64]
            want[sl // 64, h] = oracle.page_of(*parts)
    assert np.array_equal(host(pool), want)
    rows = np.arange(-1, 64 * n_pages + 1, dtype=np.int32)
    out = [torch.full((len(rows), Hkv, D), 7.0, dtype=BF, device="cuda") for _ in "kv"]
    got = fc.fc_paged_read(pool, dev(rows), out=out)
    torch.cuda.synchronize()
    for g, part in zip(got, (0, 2)):
        ref = np.full((len(rows), Hkv, D), 7.0)
        for i, sl in enumerate(rows):
            if 0 <= sl < 64 * n_pages:
                for h in range(Hkv):
                    p = oracle.page_parts(want[sl // 64, h])
                    ref[i, h] = oracle.fp4_value(p[part][sl % 64], p[part + 1][sl % 64])
        g = f64(g)
        # random bytes hold scales past bfloat16's range too: those the cache itself never writes
        held = np.isnan(ref) | (np.abs(ref) <= 3.38e38)
        assert np.array_equal(g[held], ref[held].astype(np.float32).astype(np.float64), equal_nan=True)


@pytest.mark.parametrize("Hkv,n_pages,n_src,n,rope_base", [
    (1, 1, 1, 1, 10000.0), (1, 2, 40, 100, 10000.0), (2, 1, 9, 64, 0.0), (3, 2, 33, 71, 1e6), (8, 1, 20, 37, 500.0),
    (17, 1, 5, 20, 10000.0), (40, 1, 3, 9, 10000.0),
])
def test_writes_match_oracle(Hkv, n_pages, n_src, n, rope_base):
    rng = np.random.default_rng(Hkv)
    say(f"write Hkv={Hkv} n={n} rope_base={rope_base}")
    _write_case(rng, n_pages, Hkv, n_src, n, rope_base)
    _write_case(rng, n_pages, Hkv, max(n, n_src), n, rope_base, scale=1e-3, use_src=False)


def test_writes_of_long_runs():
    """Enough tokens for several a workgroup: runs of positions, broken ones, far
    ones, and the same bytes as in writes of a few tokens each."""
    rng = np.random.default_rng(4)
    for Hkv, n in ((1, 33_000), (8, 9_001), (48, 1_300)):
        pages = -(-n // 64)
        pos = np.arange(n) % 700 + np.repeat(rng.integers(0, 2 ** 30, -(-n // 700)), 700)[:n]
        pos[rng.random(n) < 0.01] = 5
        pos[100:103] = 2 ** 31 - 1, -2 ** 31, 1 - 2 ** 31  # no run, and one of far positions before 0
        k, v = bf16(rng, n, Hkv, D).cuda(), bf16(rng, n, Hkv, D).cuda()
        slot, pos = dev(rng.permutation(64 * pages)[:n].astype(np.int32)), dev(pos.astype(np.int32))
        pools = [torch.zeros((pages, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda") for _ in range(2)]
        say(f"writes of long runs, {n} tokens of {Hkv} heads")
        fc.fc_paged_write(pools[0], k, v, slot, pos)
        for i in range(0, n, 1000):
            fc.fc_paged_write(pools[1], k[i:i + 1000], v[i:i + 1000], slot[i:i + 1000], pos[i:i + 1000])
        assert torch.equal(pools[0], pools[1])
        at, x = np.r_[100:103, rng.integers(0, n, 40)], host(pools[0])  # the same rows again by the oracle: nothing changes
        again = oracle.paged_write(x, f64(k[at]), f64(v[at]), host(slot)[at], host(pos)[at])
        assert np.array_equal(again, x)


def test_writes_of_every_kind_of_value():
    """Ties, the edges of the scales, zeros of both signs, the smallest and
    largest numbers, infinities and NaN: not rotated, and turned by nothing at
    position 0."""
    rng = np.random.default_rng(5)
    x = torch.zeros((40, 2, D), dtype=torch.float64)
    x[:, :] = torch.from_numpy(rng.choice([0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, -7, 0.5, -3], (40, 2, D)))
    x[1::4] *= 2.0 ** 90
    x[2::4] *= 2.0 ** -120
    x[3::4, :, ::9] *= 1.0625
    x[5, 0, :32], x[6, 1, 32:64], x[7] = 0.0, -0.0, 3e38
    x[8, 0, 40], x[9, 1, 3], x[10, 0, 127], x[11, :, :] = np.inf, -np.inf, np.nan, np.nan
    x[12, 0], x[13] = 2.0 ** -130, 1e-39
    x[14, :, 0::2] = 2.0 ** 127
    x = x.to(BF)
    say("write of every kind of value")
    for rope_base, pos in ((0.0, None), (10000.0, np.zeros(40, np.int32))):
        pool = torch.zeros((1, 2, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
        slot = rng.permutation(64)[:40].astype(np.int32)
        fc.fc_paged_write(pool, x.cuda(), x.flip(0).cuda(), dev(slot), None if pos is None else dev(pos), rope_base=rope_base)
        torch.cuda.synchronize()
        with np.errstate(invalid="ignore"):
            want = oracle.paged_write(np.zeros((1, 2, 8704), np.uint8), f64(x), f64(x.flip(0)), slot, pos, rope_base=rope_base)
        got = host(pool)
        # a rotation by 0 gives 0 * x: only the sign of a zero may differ
        for h in range(2):
            for i, (a, b) in enumerate(zip(oracle.page_parts(got[0, h]), oracle.page_parts(want[0, h]))):
                zero = ((a | b) & 7) == 0 if rope_base and i == 0 else np.zeros(a.shape, bool)
                assert ((a == b) | zero).all(), (rope_base, h, i)


def test_writes_from_a_fused_projection():
    """k and v as slices of [rows][(H + 2 Hkv)][D], three- and four-dimensional,
    give what copies of them give; rows at uneven distances are refused."""
    rng = np.random.default_rng(6)
    B, R, H, Hkv = 3, 7, 4, 2
    qkv = bf16(rng, B * R, H + 2 * Hkv, D).cuda()
    k, v = qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    slot, pos = dev(rng.permutation(128)[:B * R].astype(np.int32)), dev(np.arange(B * R, dtype=np.int32) * 1000)
    pools = [torch.zeros((2, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda") for _ in range(3)]
    say("write from a fused projection")
    fc.fc_paged_write(pools[0], k.contiguous(), v.contiguous(), slot, pos)
    fc.fc_paged_write(pools[1], k, v, slot, pos)
    four = qkv.view(B, R, H + 2 * Hkv, D)
    fc.fc_paged_write(pools[2], four[:, :, H:H + Hkv], four[:, :, H + Hkv:], slot, pos)
    torch.cuda.synchronize()
    assert torch.equal(pools[0], pools[1]) and torch.equal(pools[0], pools[2]) and pools[0].any()
    with pytest.raises(ValueError, match="evenly spaced"):
        fc.fc_paged_write(pools[0], four[:, :5, H:H + Hkv], four[:, :5, H + Hkv:], slot, pos)


# -------------------------------------------------------------- attention --

def make_pool(rng, n_pages, Hkv):
    """Pages of written rows, in full."""
    pool = torch.zeros((n_pages, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    k, v = bf16(rng, 64 * n_pages, Hkv, D), bf16(rng, 64 * n_pages, Hkv, D)
    fc.fc_paged_write(pool, k.cuda(), v.cuda(), dev(np.arange(64 * n_pages, dtype=np.int32)), rope_base=0.0)
    return pool


def bound(o, mean, far, keys):
    """What roundings may move a result by.  A score of a cached key: the three
    parts of a query leave 2^-13 of the largest of its 32 dims; of a tree's key:
    no more than query and key in bf16 would (2^-8 each, so 2^-7 + 2^-16
    together); both: the
    hardware's sine and cosine (2^-18 each of a pair's two products) and fp32.
    Scores that move by delta at most move each weight by e^(2 delta) - 1 of
    itself; weights are rounded to bf16 (2^-8), sums are fp32, and so is the
    result to bf16 (2^-8 of itself)."""
    delta = np.maximum((2.0 ** -13 + 2.0 ** -16) * far[0], (2.0 ** -7 + 2.0 ** -15) * far[1]) + 1e-6
    rel = np.expm1(2 * delta) + 2.0 ** -8 + (keys + 300) * 2.0 ** -23
    return rel[..., None] * mean * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(o) + 1e-30


def attend(rng, B, R, H, Hkv, lens, tree=None, rope_base=10000.0, pool=None, table=None, max_len=None, qscale=1.0,
           n_pages=None, kw=None, width=None, q=None):
    """One call against the oracle, within the bound; returns the result."""
    if pool is None:
        n_pages = n_pages or max(1, sum(-(-max(n, 0) // 64) for n in lens))
        pool = make_pool(rng, n_pages, Hkv)
    if table is None:
        width = width or max(1, max(-(-max(n, 0) // 64) for n in lens))
        table = rng.integers(0, pool.shape[0], (B, width)).astype(np.int32)
    q = bf16(rng, B, R, H, D, scale=qscale) if q is None else q
    kt, vt = bf16(rng, B, R, Hkv, D), bf16(rng, B, R, Hkv, D)
    plen = np.asarray(lens, np.int32)
    got = fc.fc_paged_attention(q.cuda(), kt.cuda(), vt.cuda(), pool, dev(table), dev(plen), tree=on_gpu(tree),
                                max_len=max_len, rope_base=rope_base, **(kw or {}))
    torch.cuda.synchronize()
    got = f64(got)
    t = {} if tree is None else {f: tree[f] for f in ("num_nodes", "mask", "pos_ids")}
    o, mean, far = oracle.paged_attention(f64(q), f64(kt), f64(vt), host(pool), table, plen, max_len=max_len,
                                          rope_base=rope_base, **t)
    most = bound(o, mean, far, max(max(lens), 0) + R)
    err = np.abs(got - o)
    same_nan = np.isnan(got) == np.isnan(o)
    assert same_nan.all()
    bad = ~(np.isnan(o) | (err <= most))
    assert not bad.any(), (float(np.nanmax(err)), np.argwhere(bad)[:5].tolist(), float(np.nanmax(err / most)))
    return got


SIZES = [  # B, R, H, Hkv, lens
    (1, 1, 1, 1, [0]), (2, 1, 4, 4, [1, 64]), (3, 1, 8, 2, [63, 65, 300]), (1, 1, 40, 8, [129]), (1, 1, 17, 1, [500]),
    (1, 2, 4, 1, [40]), (2, 4, 8, 2, [128, 0]), (2, 5, 8, 2, [64, 193]), (1, 16, 2, 2, [70]), (1, 17, 2, 2, [70]),
    (2, 33, 3, 3, [0, 257]), (1, 48, 1, 1, [640]), (1, 65, 4, 4, [100]), (2, 65, 4, 1, [130, 31]), (1, 96, 1, 1, [90]),
    (1, 101, 1, 1, [321]), (1, 128, 1, 1, [64]), (1, 129, 1, 1, [64]), (1, 256, 2, 1, [200]), (1, 250, 1, 1, [0]),
]


@pytest.mark.parametrize("B,R,H,Hkv,lens", SIZES, ids=lambda x: str(x).replace(" ", ""))
def test_attention_matches_oracle(B, R, H, Hkv, lens):
    rng = np.random.default_rng(R * 100 + H)
    say(f"attention B={B} R={R} H={H} Hkv={Hkv} lens={lens}")
    attend(rng, B, R, H, Hkv, lens)                                          # a chain
    t = trees(rng, B, R)
    t["num_nodes"] = rng.integers(max(R - 3, 1), R + 1, B).astype(np.int32)
    got = attend(rng, B, R, H, Hkv, lens, t)
    for b in range(B):
        assert (got[b, t["num_nodes"][b]:] == 0).all()
    attend(rng, B, R, H, Hkv, lens, t, rope_base=0.0, qscale=3.0)


def test_attention_in_parts_matches_oracle():
    """Prefixes long enough to be cut: over tiles of one row, a tree's rows, and
    lengths from nothing to the longest in one call."""
    rng = np.random.default_rng(7)
    for B, R, H, Hkv, lens in ((1, 1, 4, 1, [3001]), (4, 1, 8, 2, [0, 64, 1500, 2999]), (1, 65, 2, 1, [2049]),
                               (3, 7, 4, 1, [5, 700, 1300]), (2, 33, 2, 2, [1000, 130])):
        need = fc.fc_paged_attention_workspace_bytes(B, R, H, Hkv, max(lens))
        say(f"attention in parts B={B} R={R} lens={lens} workspace={need}")
        assert need > 0
        pool = make_pool(rng, 30, Hkv)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        attend(rng, B, R, H, Hkv, lens, trees(rng, B, R), pool=pool, width=-(-max(lens) // 64), kw=dict(workspace=ws),
               max_len=max(lens))


def test_attention_bounds_and_far_positions():
    rng = np.random.default_rng(8)
    pool = make_pool(rng, 8, 2)
    say("a longest length below a prefix, and above all; one page far out")
    attend(rng, 2, 3, 4, 2, [500, 77], pool=pool, max_len=200, width=8)
    attend(rng, 2, 3, 4, 2, [100, 77], pool=pool, max_len=0, width=8)
    attend(rng, 2, 3, 4, 2, [10 ** 6, -4], pool=pool, width=8)
    # position 131,000 and beyond: only a few pages exist, the others are absent
    table = np.full((1, 2050), -1, np.int32)
    table[0, [0, 700, 2046]] = [3, 4, 5]
    attend(rng, 1, 5, 4, 2, [131_000], pool=pool, table=table)
    attend(rng, 1, 5, 4, 2, [131_000], trees(rng, 1, 5), pool=pool, table=table, rope_base=1e6)


def _along(rng, u, sizes, Hkv):
    """A pool of one page per size: keys of that size along u (a row of signs)
    or, every third, against it, and a little noise."""
    n = len(sizes)
    way = np.where(np.arange(64 * n) % 3 == 2, -1.0, 1.0) * np.repeat(sizes, 64)
    k = way[:, None, None] * u + rng.standard_normal((64 * n, Hkv, D)) * 0.02
    pool = torch.zeros((n, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_write(pool, torch.from_numpy(k).to(BF).cuda(), bf16(rng, 64 * n, Hkv, D).cuda(),
                      dev(np.arange(64 * n, dtype=np.int32)), rope_base=0.0)
    return pool


@pytest.mark.parametrize("R,G", [(1, 1), (5, 2), (30, 1), (64, 1), (65, 1), (70, 4)])
def test_attention_of_scores_far_apart(R, G):
    """Scores that grow by far more than a weight's range from page to page, fall
    so, or do both: between nothing and e^90 apart, each row its own way."""
    rng = np.random.default_rng(R)
    u = rng.choice([-1.0, 1.0], D)
    for sizes in (np.linspace(0, 8, 12), np.linspace(8, 0, 12), np.abs(np.linspace(-8, 8, 12)),
                  8 * (np.arange(12) % 5 == 3)):
        pool = _along(rng, u, sizes, 1)
        c = np.where(np.arange(R * G) % 4 == 3, -1.0, 1.0) * rng.uniform(0, 1, R * G)  # score: c * size * 128 / sqrt(128)
        q = torch.from_numpy(c.reshape(1, R, G, 1) * u).to(BF)
        say(f"scores far apart R={R} G={G} sizes {sizes[0]:.0f} to {sizes[-1]:.0f}")
        for lens in ([768], [747]):
            attend(rng, 1, R, G, 1, lens, pool=pool, table=np.arange(12, dtype=np.int32)[None], rope_base=0.0, q=q)


def test_attention_rows_do_not_move_each_other():
    """A row's bits are its own: other rows of its wave whose scores lie far
    apart, or are not finite, change nothing."""
    rng = np.random.default_rng(21)
    u = rng.choice([-1.0, 1.0], D)
    pool = _along(rng, u, np.linspace(0, 8, 12), 1)
    table, plen = dev(np.arange(12, dtype=np.int32)[None]), dev(np.array([760], np.int32))
    for R in (1, 9, 33, 65):
        G = 3 if R == 1 else 1
        q = bf16(rng, 1, R, G, D, scale=0.3)
        kt, vt = bf16(rng, 1, R, 1, D), bf16(rng, 1, R, 1, D)
        other = q.clone()
        change = np.arange(R * G) % 3 != 0
        other.view(R * G, D)[torch.from_numpy(change)] = torch.from_numpy(u).to(BF)
        other.view(R * G, D)[1] = float("nan")
        say(f"rows do not move each other R={R}")
        a, b = (fc.fc_paged_attention(x.cuda(), kt.cuda(), vt.cuda(), pool, table, plen, rope_base=0.0) for x in (q, other))
        a, b = (x.view(R * G, D).view(torch.int16).cpu().numpy() for x in (a, b))
        assert np.array_equal(a[~change], b[~change]) and not np.array_equal(a[change], b[change])


def test_attention_of_masks_that_leave_nothing():
    """Rows whose mask admits no row, other values than 1 in masks (they do not
    admit), lengths of nodes outside [0, R]: zero where nothing is attended."""
    rng = np.random.default_rng(9)
    B, R = 4, 20
    t = trees(rng, B, R)
    t["mask"][:, 3] = 0
    t["mask"][:, 7] *= 2
    t["mask"][1] = -2 ** 31
    t["num_nodes"] = np.array([R, R, -1, 3 * R], np.int32)
    say("masks that leave nothing")
    got = attend(rng, B, R, 4, 2, [0, 0, 0, 0], t)
    assert (got[0, [3, 7]] == 0).all() and (got[1] == 0).all() and (got[2] == 0).all() and (got[3, 4] != 0).any()
    got = attend(rng, B, R, 4, 2, [0, 70, 70, 0], t)
    assert (got[1] != 0).any() and (got[2] == 0).all()


def test_attention_of_absent_pages():
    rng = np.random.default_rng(10)
    pool = make_pool(rng, 6, 2)
    table = np.array([[0, -1, 6, 2], [2 ** 31 - 1, -2 ** 31, 7, 5], [9, 9, 9, 9]], np.int32)
    say("pages outside the pool")
    got = attend(rng, 3, 1, 8, 2, [256, 200, 150], pool=pool, table=table)
    assert (got != 0).all(-1).any()
    t = trees(rng, 3, 70)
    t["mask"][2] = 0
    got = attend(rng, 3, 70, 4, 2, [256, 200, 150], t, pool=pool, table=table)
    assert (got[2] == 0).all()


@pytest.mark.parametrize("R", [1, 5, 40, 65, 100])
def test_attention_does_not_see_what_lies_behind_the_prefix(R):
    """NaN scales and any codes in slots past the length, in the rows behind
    num_nodes, and in other pages: the same bits as with zeros there."""
    rng = np.random.default_rng(11)
    B, H, Hkv, n = 2, 4, 2, [70, 129]
    pool = make_pool(rng, 8, Hkv)
    clean, dirty = host(pool).copy(), host(pool).copy()
    table = np.array([[1, 2, 7], [3, 4, 5]], np.int32)
    for b in range(B):
        for p in range(3):
            for h in range(Hkv):
                parts = [oracle.page_parts(x[table[b, p], h]) for x in (clean, dirty)]
                for t in range(64):
                    if 64 * p + t >= n[b]:
                        for i in range(4):
                            parts[0][i][t] = 0
                            parts[1][i][t] = 255 if i % 2 else rng.integers(0, 16, 128)
                clean[table[b, p], h], dirty[table[b, p], h] = (oracle.page_of(*x) for x in parts)
    q, kt, vt = bf16(rng, B, R, H, D).cuda(), bf16(rng, B, R, Hkv, D).cuda(), bf16(rng, B, R, Hkv, D).cuda()
    t = trees(rng, B, R)
    t["num_nodes"] = np.array([max(R - 2, 1), R], np.int32)
    outs = []
    say(f"behind the prefix R={R}")
    for x in (clean, dirty):
        if R > 2:
            fill = 0.0 if x is clean else float("nan")
            kt[0, R - 2:], vt[0, R - 2:], q[0, R - 2:] = fill, fill, fill
        outs.append(fc.fc_paged_attention(q, kt, vt, dev(x), dev(table), dev(np.array(n, np.int32)), tree=on_gpu(t)))
    torch.cuda.synchronize()
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1])


def test_attention_shows_what_is_not_finite():
    """A NaN or an infinity among the values, keys or queries that a row
    attends to makes the row NaN, and no other row."""
    rng = np.random.default_rng(12)
    B, R, H, Hkv = 5, 20, 2, 2
    pool = make_pool(rng, 10, Hkv)
    table = np.arange(10, dtype=np.int32).reshape(5, 2)
    q, kt, vt = bf16(rng, B, R, H, D), bf16(rng, B, R, Hkv, D), bf16(rng, B, R, Hkv, D)
    x = host(pool).copy()
    parts = oracle.page_parts(x[table[0, 1], 1])
    parts[1][5, 2] = 255                    # tree 0, head 1: a key's scale
    x[table[0, 1], 1] = oracle.page_of(*parts)
    parts = oracle.page_parts(x[table[1, 0], 0])
    parts[3][9, 0] = 255                    # tree 1, head 0: dims 0 .. 31 of a value
    x[table[1, 0], 0] = oracle.page_of(*parts)
    q[2, 4, 1, 100] = float("inf")
    kt[3, 6, 0, 3] = float("nan")
    vt[4, 2, 1, 7] = float("nan")
    t = trees(rng, B, R)
    say("not finite")
    got = f64(fc.fc_paged_attention(q.cuda(), kt.cuda(), vt.cuda(), dev(x), dev(table), dev(np.full(B, 100, np.int32)),
                                    tree=on_gpu(t)))
    nan = np.isnan(got)
    assert nan[0, :, 1].all() and not nan[0, :, 0].any()
    assert nan[1, :, 0, :32].all() and not nan[1, :, 0, 32:].any() and not nan[1, :, 1].any()
    assert nan[2, 4, 1].all() and nan[2].sum() == D
    sees = t["mask"][3, :, 6] == 1
    assert nan[3, sees, 0].all() and not nan[3, ~sees, 0].any() and not nan[3, :, 1].any()
    sees = t["mask"][4, :, 2] == 1
    assert nan[4, sees, 1, 7].all() and not nan[4, ~sees].any() and not nan[4, :, 0].any()


def test_attention_of_a_fused_projection():
    """Queries, keys and values as slices give the bits that copies give."""
    rng = np.random.default_rng(13)
    B, R, H, Hkv = 2, 9, 8, 2
    qkv = bf16(rng, B, R, H + 2 * Hkv, D).cuda()
    q, kt, vt = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
    pool, table, plen = make_pool(rng, 4, Hkv), dev(np.array([[0, 1], [3, 2]], np.int32)), dev(np.array([100, 64], np.int32))
    say("attention of a fused projection")
    a = fc.fc_paged_attention(q, kt, vt, pool, table, plen)
    b = fc.fc_paged_attention(q.contiguous(), kt.contiguous(), vt.contiguous(), pool, table, plen)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_attention_agrees_with_the_dense_kernel():
    """A prefix read out of the pool and given to fc_tree_attention: the same
    attention, but for the roundings of both."""
    rng = np.random.default_rng(14)
    B, R, H, Hkv, n = 2, 33, 8, 4, 200
    pool = make_pool(rng, 8, Hkv)
    table = np.array([[0, 5, 2, 7], [1, 3, 4, 6]], np.int32)
    slot = (table[:, np.arange(n) // 64] * 64 + np.arange(n) % 64).astype(np.int32)
    kc, vc = (x.view(B, n, Hkv, D) for x in fc.fc_paged_read(pool, dev(slot.reshape(-1))))
    q, kt, vt = bf16(rng, B, R, H, D).cuda(), bf16(rng, B, R, Hkv, D).cuda(), bf16(rng, B, R, Hkv, D).cuda()
    t, plen = on_gpu(trees(rng, B, R)), dev(np.full(B, n, np.int32))
    say("against the dense kernel")
    a = f64(fc.fc_paged_attention(q, kt, vt, pool, dev(table), plen, tree=t))
    b = f64(fc.fc_tree_attention(q, kt, vt, kc, vc, plen, t))
    # scores of up to about 5 with 2^-7 between the kernels' roundings: 2 * 5 * 2^-7 of the values, 3 at most a dim
    assert np.abs(a - b).max() < 2 * 5 * 2.0 ** -7 * 3 and np.abs(a - b).mean() < 0.01


def test_offsets_past_32_bits():
    """Pages beyond 4 GiB of one pool are written, read and attended."""
    Hkv, n_pages = 16, 33_000                      # 4.6 GB
    assert fc.fc_paged_pool_bytes(n_pages, Hkv) > 2 ** 32
    rng = np.random.default_rng(15)
    pool = torch.empty((n_pages, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    small = torch.zeros((2, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    k, v = bf16(rng, 100, Hkv, D).cuda(), bf16(rng, 100, Hkv, D).cuda()
    table, pos = np.array([[n_pages - 1, n_pages - 2]], np.int32), np.arange(100, dtype=np.int32)
    slot = table[0, pos // 64] * 64 + pos % 64
    say("past 4 GiB")
    fc.fc_paged_write(pool, k, v, dev(slot), dev(pos))
    fc.fc_paged_write(small, k, v, dev(pos), dev(pos))
    got, want = fc.fc_paged_read(pool, dev(slot)), fc.fc_paged_read(small, dev(pos))
    q, kt, vt = bf16(rng, 1, 3, Hkv, D).cuda(), bf16(rng, 1, 3, Hkv, D).cuda(), bf16(rng, 1, 3, Hkv, D).cuda()
    a = fc.fc_paged_attention(q, kt, vt, pool, dev(table), dev(np.array([100], np.int32)))
    b = fc.fc_paged_attention(q, kt, vt, small, dev(np.array([[0, 1]], np.int32)), dev(np.array([100], np.int32)))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(a, b) and got[0].any()


# ------------------------------------------------- together, streams, graphs --

class _Cache:
    """Steps of a serving loop on both sides: what is accepted is planned,
    written and attended."""

    def __init__(self, rng, B, Hkv, n_pages, max_pages):
        self.B, self.Hkv = B, Hkv
        self.s = fc.paged_state(B, max_pages, n_pages, "cuda")
        self.pool = fc.paged_pool(n_pages, Hkv, "cuda").zero_()
        self.o = {f: host(v).copy() for f, v in self.s.items()}
        self.o_pool = host(self.pool).copy()

    def step(self, add, n_slots, k, v, tree=None, last=None, dev_add=None):
        mask = None if tree is None else tree["mask"]
        kw = {} if tree is None else dict(tree=on_gpu(tree), last_node=dev(last))
        p = fc.fc_paged_plan(self.s["len"], dev(add) if dev_add is None else dev_add, self.s["table"], self.s["queue"],
                             self.s["ends"], n_slots, **kw)
        fc.fc_paged_write(self.pool, k, v, p["slot"], p["pos"], src=p["src"])
        self.s.update(len=p["len"], ends=p["ends"])
        r = oracle.paged_plan(self.o["len"], add, self.o["table"], self.o["queue"], self.o["ends"], n_slots, mask, last)
        self.o_pool = oracle.paged_write(self.o_pool, f64(k).reshape(-1, self.Hkv, D), f64(v).reshape(-1, self.Hkv, D),
                                         r["slot"], r["pos"], r["src"])
        self.o.update({f: r[f] for f in ("len", "ends", "table", "queue")})
        torch.cuda.synchronize()
        for f in self.o:
            assert np.array_equal(host(self.s[f]), self.o[f]), f
        assert np.array_equal(host(self.pool), self.o_pool)


def test_a_serving_loop():
    """Prompts in; then steps of a tree: attention over the cache, acceptance by
    fc_verify_accept, the accepted rows planned and written from its results on
    the device, a sequence that ends and another that takes its pages."""
    rng = np.random.default_rng(16)
    B, R, H, Hkv = 3, 17, 4, 2
    c = _Cache(rng, B, Hkv, 9, 4)
    add = np.array([70, 0, 129], np.int32)
    n = int(add.sum())
    c.step(add, n + 5, bf16(rng, n, Hkv, D).cuda(), bf16(rng, n, Hkv, D).cuda())
    for step in range(4):
        say(f"serving step {step}")
        t = trees(rng, B, R, 5)
        t["node_tok"] = rng.integers(1, 50, (B, R)).astype(np.int32)
        target = rng.integers(-1, 50, (B, R)).astype(np.int32)
        for b in range(B):  # a path that the model agrees with
            for i in range(1, R):
                if rng.random() < 0.7:
                    target[b, t["parent"][b, i]] = t["node_tok"][b, i]
        attend_pool, lens = c.pool, host(c.s["len"])
        q, kt, vt = bf16(rng, B, R, H, D), bf16(rng, B, R, Hkv, D), bf16(rng, B, R, Hkv, D)
        got = f64(fc.fc_paged_attention(q.cuda(), kt.cuda(), vt.cuda(), attend_pool, c.s["table"], c.s["len"],
                                        tree=on_gpu(t), max_len=int(lens.max())))
        o, mean, far = oracle.paged_attention(f64(q), f64(kt), f64(vt), c.o_pool, c.o["table"], lens, t["num_nodes"],
                                              t["mask"], t["pos_ids"])
        assert (np.abs(got - o) <= bound(o, mean, far, int(lens.max()) + R)).all()
        a = fc.fc_verify_accept(on_gpu(t), dev(target), m=5)
        c.step(host(a["accept_len"]), B * 6, kt.cuda(), vt.cuda(), t, host(a["last_node"]), dev_add=a["accept_len"])
        if step == 1:
            gone = np.array([0, 0, -2 ** 31], np.int32)
            c.step(gone, 0, bf16(rng, 1, Hkv, D).cuda(), bf16(rng, 1, Hkv, D).cuda())
            again = np.array([0, 0, 200], np.int32)
            c.step(again, 200, bf16(rng, 200, Hkv, D).cuda(), bf16(rng, 200, Hkv, D).cuda())
    assert (c.o["len"] > 0).all()


def _state(rng, B=2, R=9, H=8, Hkv=2, n=700):
    pool = make_pool(rng, 12, Hkv)
    return dict(q=bf16(rng, B, R, H, D).cuda(), k_tree=bf16(rng, B, R, Hkv, D).cuda(),
                v_tree=bf16(rng, B, R, Hkv, D).cuda(), pool=pool,
                table=dev(rng.integers(0, 12, (B, -(-n // 64))).astype(np.int32)),
                prefix_len=dev(np.array([n, n // 3], np.int32)), tree=on_gpu(trees(rng, B, R)))


def test_attention_workspaces_and_repeats():
    """A workspace of NaN, one too small, one out of line; two calls the same
    bits."""
    rng = np.random.default_rng(17)
    s = _state(rng)
    need = fc.fc_paged_attention_workspace_bytes(2, 9, 8, 2, 11 * 64)
    assert need > 0
    say("workspaces")
    want = fc.fc_paged_attention(**s)
    ws = torch.full((need + 32,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(want, fc.fc_paged_attention(**s, workspace=ws[:need]))
    assert torch.equal(want, fc.fc_paged_attention(**s))
    for bad in (ws[:need - 1], ws[8:8 + need]):
        with pytest.raises(fc.FcError):
            fc.fc_paged_attention(**s, workspace=bad)


def test_calls_on_another_stream():
    """A call on a side stream while the current one still reads blocks that it
    has freed, of the sizes of the call's own tensors: they are not the call's."""
    rng = np.random.default_rng(18)
    s = _state(rng)
    want = fc.fc_paged_attention(**s)
    slot = dev(np.arange(12 * 64, dtype=np.int32))
    k, v = fc.fc_paged_read(s["pool"], slot)
    side, a = torch.cuda.Stream(), torch.rand(6144, 6144, device="cuda")
    sizes = [fc.fc_paged_attention_workspace_bytes(2, 9, 8, 2, 11 * 64), want.numel() * 2, k.numel() * 2]
    say("side stream")
    for i in range(3):
        busy = [torch.full((n // 4 + 1,), i + 1, dtype=torch.int32, device="cuda") for n in sizes]
        seen = [torch.empty_like(x) for x in busy]
        torch.cuda.synchronize()
        a @ a
        for x, y in zip(busy, seen):
            y.copy_(x)  # runs after the product
        del busy, x
        got = fc.fc_paged_attention(**s, stream=side)
        k2, v2 = fc.fc_paged_read(s["pool"], slot, stream=side)
        torch.cuda.synchronize()
        assert all((x == i + 1).all() for x in seen)
        assert torch.equal(got, want) and torch.equal(k, k2) and torch.equal(v, v2)


def test_a_step_in_a_captured_graph():
    """Plan, write and attention captured together: every replay, on new inputs
    and with other work between, gives the eager results."""
    rng = np.random.default_rng(19)
    B, R, H, Hkv, n_pages, width = 2, 9, 8, 2, 30, 12
    s = fc.paged_state(B, width, n_pages, "cuda")
    pool = make_pool(rng, n_pages, Hkv)
    first = fc.fc_paged_plan(s["len"], dev(np.array([600, 130], np.int32)), s["table"], s["queue"], s["ends"], 730)
    new = lambda h: bf16(rng, B, R, h, D).cuda()  # noqa: E731
    q, kt, vt = new(H), new(Hkv), new(Hkv)
    t = on_gpu(trees(rng, B, R))
    add, last = dev(np.array([2, 1], np.int32)), dev(np.array([5, 0], np.int32))
    lens, ends = first["len"].clone(), first["ends"].clone()

    def step():
        p = fc.fc_paged_plan(lens, add, s["table"], s["queue"], ends, 2 * R, tree=t, last_node=last)
        fc.fc_paged_write(pool, kt, vt, p["slot"], p["pos"], src=p["src"])
        return p, fc.fc_paged_attention(q, kt, vt, pool, s["table"], p["len"], tree=t)

    say("a step captured")
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p, out = step()
    for i in range(4):
        for x in (q, kt, vt):
            x.copy_(new(x.shape[2]))
        row = torch.randint(0, R, (B,), device="cuda", dtype=torch.int32)
        last.copy_(row)
        add.copy_(t["pos_ids"].gather(1, row[:, None].long())[:, 0] + 1)
        graph.replay()
        got, plan, held = out.clone(), {f: v.clone() for f, v in p.items()}, pool.clone()
        busy = torch.full((8 << 20,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        q_plan, want = step()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(held, pool), i
        assert all(torch.equal(plan[f], q_plan[f]) for f in plan), i
        lens.copy_(plan["len"])
        ends.copy_(plan["ends"])
        del busy


def test_refusals_on_the_gpu():
    """What the host refuses once tensors are on a device."""
    rng = np.random.default_rng(20)
    s = _state(rng)
    say("refusals")
    with pytest.raises(fc.FcError):
        fc.fc_paged_attention(**s, max_len=11 * 64 + 1)
    with pytest.raises(fc.FcError):
        fc.fc_paged_attention(**s, rope_base=1.0)
    with pytest.raises(fc.FcError):
        fc.fc_paged_attention(**s, rope_base=float("nan"))
    with pytest.raises(ValueError, match="one device"):
        fc.fc_paged_attention(**{**s, "prefix_len": s["prefix_len"].cpu()})
    st = fc.paged_state(2, 3, 9, "cuda")
    add = dev(np.array([1, 2], np.int32))
    out = fc.fc_paged_plan(st["len"], add, st["table"], st["queue"], st["ends"], 5)
    with pytest.raises(fc.FcError):
        fc.fc_paged_plan(out["len"], add, st["table"], st["queue"], st["ends"], 5, out=out)
    ptr = ctypes.c_void_p(s["pool"].data_ptr() + 8)
    assert fc.lib().fc_paged_read(ptr, 12, 2, D, ptr, 1, ptr, ptr, None) == 1
