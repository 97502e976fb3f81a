"""The 8-bit paged cache on the GPU against the oracle: written, moved and read bytes
element by element, computed numbers within bounds that follow from what is rounded."""
import numpy as np
import pytest
import torch

import oracle
from gpu_pipeline import dev, host, say
from oracle import paged8 as o8

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_17139_amd as fc  # noqa: E402
from test_paged import bf16, f64, on_gpu, trees  # noqa: E402

D, BF = 128, torch.bfloat16
NAN, INF = float("nan"), float("inf")


def same_pool(got, want, what=""):
    """Bytes equal but for the sign of codes that are NaN; the bytes behind the scales are nobody's."""
    a, b = (host(x) if torch.is_tensor(x) else x for x in (got, want))
    a, b = a.copy(), b.copy()
    for x in (a, b):
        c = x[..., :o8.SCALES]
        c[(c & 127) == 127] = 127
    assert np.array_equal(a, b), (what, np.argwhere(a != b)[:5].tolist())


def make_pool(rng, n_pages, Hkv, scale=1.0):
    """Pages of random rows, some channels and some tokens larger than others."""
    k, v = (bf16(rng, 64 * n_pages, Hkv, D, scale=scale) for _ in "kv")
    for x in (k, v):
        x[..., 5::37] *= 6
        x[::13] *= 3
    pool = torch.zeros((n_pages, Hkv, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), dev(np.arange(64 * n_pages, dtype=np.int32)))
    return pool


# ------------------------------------------------------------------- norm --

def _norm(q, k, wq, wk, pos, **kw):
    got = fc.fc_norm_rotate(None if q is None else q.cuda(), None if k is None else k.cuda(),
                            None if wq is None else wq.cuda(), None if wk is None else wk.cuda(),
                            None if pos is None else dev(pos), **kw)
    torch.cuda.synchronize()
    for x, w, y in zip((q, k), (wq, wk), got):
        if x is None:
            assert y is None
            continue
        rows = f64(x).reshape(-1, *x.shape[-2:])
        want, most = o8.norm_rotate(rows, None if w is None else f64(w), pos, **kw)
        y = f64(y).reshape(want.shape)
        assert np.array_equal(np.isnan(y), np.isnan(want))
        ok = ~np.isnan(want)
        assert (np.abs(y - want)[ok] <= most[ok]).all(), float(np.nanmax(np.abs(y - want) / most))
    return got


@pytest.mark.parametrize("n,H,Hkv", [(1, 32, 8), (1, 1, 1), (3, 5, 5), (0, 4, 2), (70, 40, 8), (5, 3, 0), (5, 0, 3),
                                     (1030, 3, 1), (4099, 2, 1)])
def test_norm_rotate_matches_oracle(n, H, Hkv):
    rng = np.random.default_rng(n + H)
    say(f"norm n={n} H={H} Hkv={Hkv}")
    q, k = bf16(rng, n, H, D, scale=3.0) if H else None, bf16(rng, n, Hkv, D, scale=0.1) if Hkv else None
    w = [1 + bf16(rng, D, scale=0.3) if x is not None else None for x in (q, k)]
    pos = rng.integers(-5, 200_000, n).astype(np.int32)
    _norm(q, k, *w, pos)
    if H and Hkv:
        _norm(q, k, None, w[1], pos, rope_base=1e6)
        _norm(q, k, w[0], None, None, rope_base=0.0, eps=0.5)
        _norm(q, k, None, None, pos)


def test_norm_rotate_of_numbers_that_are_none():
    rng = np.random.default_rng(4)
    q, k = bf16(rng, 6, 2, D), bf16(rng, 6, 2, D)
    q[0] = 0                       # nothing to norm: eps alone keeps it finite
    q[1, 0, 3], q[2, 1, 70] = NAN, INF
    k[3] *= 2.0 ** -70             # squares below fp32's least
    k[4] = 2.0 ** 60               # and a sum of them near its largest
    say("norm of zeros, infinities, small and large numbers")
    pos = np.array([2 ** 31 - 1, -2 ** 31, 0, 5, 7, 9], np.int32)
    w = [torch.ones(D).to(BF)] * 2
    got = fc.fc_norm_rotate(q.cuda(), k.cuda(), w[0].cuda(), w[1].cuda(), dev(pos))
    a, b = f64(got[0]), f64(got[1])
    assert (a[0] == 0).all() and np.isnan(a[1, 0]).all() and np.isnan(a[2, 1, 70]) and not np.isnan(a[1, 1]).any()
    want, most = o8.norm_rotate(f64(k), f64(w[1]), pos)
    ok = np.arange(6) != 3
    assert (np.abs(b - want)[ok] <= most[ok]).all() and (np.abs(b[3]) < 1e-15).all()


def test_norm_rotate_in_place_and_in_slices():
    """Rows of a fused projection, normed where they are; batches of rows; results beside their rows."""
    rng = np.random.default_rng(5)
    B, R, H, Hkv = 2, 9, 4, 2
    qkv = bf16(rng, B, R, H + 2 * Hkv, D).cuda()
    pos = rng.integers(0, 5000, (B, R)).astype(np.int32)
    w = 1 + bf16(rng, D, scale=0.3)
    say("norm in slices")
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:].clone()
    want = fc.fc_norm_rotate(q.clone(), k.clone(), w.cuda(), w.cuda(), dev(pos))
    got = fc.fc_norm_rotate(q, k, w.cuda(), w.cuda(), dev(pos))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = fc.fc_norm_rotate(q, None, w.cuda(), None, dev(pos), out=(torch.empty_like(want[0]), None))
    assert torch.equal(one[0], want[0]) and one[1] is None
    fc.fc_norm_rotate(q, k, w.cuda(), w.cuda(), dev(pos), out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, :, H + Hkv:], v)
    with pytest.raises(fc.FcError):   # the keys' place is the queries'
        fc.fc_norm_rotate(q[:, :, :Hkv], k, None, None, dev(pos), out=(k, q[:, :, :Hkv]))
    with pytest.raises(fc.FcError):
        fc.fc_norm_rotate(qkv[:, :, 1:1 + H], None, None, None, dev(pos), out=(qkv[:, :, :H], None))


# ----------------------------------------------------------- write and read --

def _write(pool, k, v, slot, src=None):
    want = o8.write(host(pool), f64(k).reshape(-1, *k.shape[-2:]), f64(v).reshape(-1, *v.shape[-2:]), slot, src)
    fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), dev(np.asarray(slot, np.int32)),
                       src=None if src is None else dev(np.asarray(src, np.int32)))
    torch.cuda.synchronize()
    same_pool(pool, want)
    return want


def _read(pool, slot):
    """Rows of slots as the oracle has them: what a page stands for, exactly."""
    k, v = fc.fc_paged_byte_read(pool, dev(np.asarray(slot, np.int32)))
    p = host(pool)
    for i, s in enumerate(slot):
        for h in range(p.shape[1]):
            for got, want in zip((k, v), o8.held(p[s // 64, h])):
                assert np.array_equal(f64(got[i, h]), want[s % 64], equal_nan=True), (i, s, h)


@pytest.mark.parametrize("Hkv,n_pages,lens,adds", [
    (1, 3, [0], [1]), (2, 4, [0, 31], [32, 1]), (3, 5, [5, 64, 33], [1, 1, 1]), (8, 6, [60, 0], [11, 7]),
    (1, 9, [0, 0], [300, 129]), (5, 4, [17], [150]), (2, 12, [1, 2, 3, 4], [64, 63, 62, 33]),
])
def test_writes_match_oracle(Hkv, n_pages, lens, adds):
    """Prompts and single tokens, into new blocks and into begun ones, whose scale
    stays or rises; then read back."""
    rng = np.random.default_rng(Hkv + n_pages)
    say(f"write Hkv={Hkv} lens={lens} adds={adds}")
    pool = dev(rng.integers(0, 256, (n_pages, Hkv, o8.PAGE_BYTES)).astype(np.uint8))
    perm, at, tables = rng.permutation(n_pages), 0, []
    for n, a in zip(lens, adds):
        m = -(-(n + a) // 64)
        tables.append(perm[at:at + m])
        at += m
    slots = lambda a, b: np.concatenate([t[np.arange(x, y) // 64] * 64 + np.arange(x, y) % 64  # noqa: E731
                                         for t, x, y in zip(tables, a, b)]).astype(np.int32)
    before = slots([0] * len(lens), lens)
    if len(before):
        _write(pool, bf16(rng, len(before), Hkv, D), bf16(rng, len(before), Hkv, D, scale=1e-3), before)
    for scale in (1.0, 100.0, 1e-4):
        new = slots(lens, [n + a for n, a in zip(lens, adds)])
        n = len(new)
        src = rng.permutation(n + 3)[:n]
        _write(pool, bf16(rng, n + 3, Hkv, D, scale=scale), bf16(rng, n + 3, Hkv, D, scale=scale), new, src)
        lens = [n + a for n, a in zip(lens, adds)]
        adds = [min(a, 64 * len(t) - n) for a, n, t in zip([1, 2, 40, 5], lens, tables)]
    held = slots([0] * len(lens), lens)
    _read(pool, rng.permutation(held)[:40])
    _read(pool, held[:100])


def test_a_block_row_by_row():
    """32 rows one after another, each larger than the last, smaller, or all alike:
    the block's scale rises with them, and what was there is rounded to it."""
    rng = np.random.default_rng(6)
    say("a block row by row")
    for grow in (1.3, 1 / 1.3, 1.0, 40.0):
        pool = dev(rng.integers(0, 256, (2, 2, o8.PAGE_BYTES)).astype(np.uint8))
        want = host(pool)
        for t in range(40):
            k, v = bf16(rng, 1, 2, D, scale=grow ** min(t, 20)), bf16(rng, 1, 2, D, scale=grow ** -min(t, 20))
            want = o8.write(want, f64(k), f64(v), [64 + t])
            fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), dev(np.array([64 + t], np.int32)))
        same_pool(pool, want, grow)


def test_write_rounds_to_even_and_marks_what_is_not_finite():
    rng = np.random.default_rng(7)
    ties = np.sort(o8.VALUES[:127])
    row = np.concatenate([ties[30:], (ties[30:-1] + ties[31:]) / 2])
    k = np.zeros((40, 1, D))
    k[0, 0, :64], k[1, 0, :64], k[2, 0, :65] = row[:64], row[64:128], row[-65:]
    k[3] = 448.0
    k[:32, 0, 100:] = rng.choice([1, -1], (32, 28)) * 2.0 ** rng.integers(-12, 8, (32, 28))
    v = k[::-1].copy()
    k, v = torch.from_numpy(k).to(BF), torch.from_numpy(v).to(BF)
    k[4, 0, 7], k[5, 0, 8], k[6, 0, 9], v[4, 0, 7], v[33, 0, 8] = NAN, INF, -INF, INF, NAN
    k[32], v[7] = 3.3e38, -3.3e38     # saturates
    k[33], v[32] = 2.0 ** -133, 2.0 ** -130
    k[34:] = 0
    pool = dev(rng.integers(0, 256, (1, 1, o8.PAGE_BYTES)).astype(np.uint8))
    say("ties, infinities, the largest and the least")
    _write(pool, k, v, np.arange(40))
    _read(pool, np.arange(40))
    got = fc.fc_paged_byte_read(pool, dev(np.arange(40, dtype=np.int32)))
    bad = torch.isnan(got[0]).nonzero().tolist()
    assert bad == [[4, 0, 7], [5, 0, 8], [6, 0, 9]] and torch.isnan(got[1]).sum() == 2
    # one block of nothing but what is not finite: its scale is the least
    _write(pool, torch.full((32, 1, D), NAN).to(BF), torch.full((32, 1, D), INF).to(BF), np.arange(32))
    assert host(pool)[0, 0, o8.SCALES] == 10


def test_writes_skip_and_order():
    """Slots and rows outside of what there is, entries in any order within their
    block, the first row last, slices of a projection, and nothing to do."""
    rng = np.random.default_rng(8)
    pool = dev(rng.integers(0, 256, (3, 2, o8.PAGE_BYTES)).astype(np.uint8))
    guarded = torch.cat([pool, pool])
    qkv = bf16(rng, 2, 40, 8, D)
    k, v = qkv[:, :, 4:6], qkv[:, :, 6:]
    a, b = rng.permutation(32), 32 + rng.permutation(30) + 1
    slot = np.concatenate([a, [-1, 192, 2 ** 31 - 1, -2 ** 31], b, [100, 101], [64]])
    src = rng.permutation(80)[:len(slot)]
    src[[3, 40]] = [-1, 80]
    say("skipped entries and any order")
    want = o8.write(host(pool), f64(k).reshape(80, 2, D), f64(v).reshape(80, 2, D), slot, src)
    g = qkv.cuda()
    fc.fc_paged_byte_write(guarded[:3], g[:, :, 4:6], g[:, :, 6:], dev(slot.astype(np.int32)), src=dev(src.astype(np.int32)))
    same_pool(guarded[:3], want)
    assert torch.equal(guarded[3:], pool)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    fc.fc_paged_byte_write(guarded[:3], g[:, :, 4:6], g[:, :, 6:], none)
    fc.fc_paged_byte_write(guarded[:3], g[0, :0, 4:6], g[0, :0, 6:], dev(slot.astype(np.int32)))
    same_pool(guarded[:3], want)
    out = [torch.full((5, 2, D), 7.0, dtype=BF, device="cuda") for _ in "kv"]
    fc.fc_paged_byte_read(pool, dev(np.array([5, -1, 192, 70, -2 ** 31], np.int32)), out=out)
    for x in out:
        assert (x[[1, 2, 4]] == 7).all()
    fc.fc_paged_byte_read(pool, none)


def test_more_rows_than_one_launch_takes():
    """Writes and reads of more entries than a launch's workgroups hold."""
    n, piece = 2 ** 25 + 96, 2 ** 21 + 64
    pages = -(-n // 64)
    torch.manual_seed(1)
    x = torch.randn((4096, 1, D), dtype=BF, device="cuda")
    slot = torch.arange(n, dtype=torch.int32, device="cuda")
    src = torch.randint(0, 4096, (n,), dtype=torch.int32, device="cuda")
    pools = [torch.zeros((pages, 1, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda") for _ in "ab"]
    say("writes and reads of more than a launch")
    fc.fc_paged_byte_write(pools[0], x, x, slot, src)
    for i in range(0, n, piece):
        fc.fc_paged_byte_write(pools[1], x, x, slot[i:i + piece], src[i:i + piece])
    assert torch.equal(pools[0], pools[1]) and pools[0][-1].any()
    few = [slice(0, 100), slice(2 ** 24 - 50, 2 ** 24 + 50), slice(n - 100, n)]
    k, v = fc.fc_paged_byte_read(pools[0], slot)
    for s in few:
        want = fc.fc_paged_byte_read(pools[1], slot[s])
        assert torch.equal(k[s], want[0]) and torch.equal(v[s], want[1]) and k[s].any()


# ------------------------------------------------------------- attention --

def attend(rng, B, R, H, Hkv, lens, tree=None, pool=None, table=None, max_len=None, qscale=1.5, width=None, q=None,
           kt=None, vt=None, kw=None):
    """One call against the oracle, within what its roundings may do; returns the result."""
    if pool is None:
        pool = make_pool(rng, max(1, sum(-(-max(n, 0) // 64) for n in lens)), Hkv)
    if table is None:
        width = width or max(1, max(-(-max(n, 0) // 64) for n in lens))
        table = rng.integers(0, pool.shape[0], (B, width)).astype(np.int32)
    q = bf16(rng, B, R, H, D, scale=qscale) if q is None else q
    kt = bf16(rng, B, R, Hkv, D) if kt is None else kt
    vt = bf16(rng, B, R, Hkv, D) if vt is None else vt
    plen = np.asarray(lens, np.int32)
    lse = torch.full((B, R, H), 7.0, device="cuda")
    args = (q.cuda(), kt.cuda(), vt.cuda(), pool, dev(table), dev(plen))
    got = fc.fc_paged_byte_attention(*args, tree=on_gpu(tree), max_len=max_len, lse=lse, **(kw or {}))
    plain = fc.fc_paged_byte_attention(*args, tree=on_gpu(tree), max_len=max_len)
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int16), plain.view(torch.int16))  # with and without the logarithms
    got, lse = f64(got), f64(lse)
    t = {} if tree is None else {f: tree[f] for f in ("num_nodes", "mask")}
    o, want_lse, most, lse_most = o8.attention(f64(q), f64(kt), f64(vt), host(pool), table, plen, max_len=max_len, **t)
    for x, y, m in ((got, o, most), (lse, want_lse, lse_most)):
        assert np.array_equal(np.isnan(x), np.isnan(y))
        with np.errstate(invalid="ignore"):
            bad = ~(np.isnan(y) | (x == y) | (np.abs(x - y) <= m))
            assert not bad.any(), (np.argwhere(bad)[:5].tolist(), float(np.nanmax(np.abs(x - y) / m)))
    return got


SIZES = [  # B, R, H, Hkv, lens
    (1, 1, 1, 1, [0]), (2, 1, 4, 4, [1, 64]), (3, 1, 8, 2, [63, 65, 300]), (1, 1, 40, 8, [129]), (1, 1, 17, 1, [500]),
    (1, 2, 4, 1, [40]), (2, 4, 8, 2, [128, 0]), (2, 5, 8, 2, [64, 193]), (1, 16, 2, 2, [70]), (1, 17, 2, 2, [70]),
    (1, 32, 1, 1, [95]), (2, 33, 3, 3, [0, 257]), (1, 48, 1, 1, [640]), (1, 65, 4, 4, [100]), (2, 65, 4, 1, [130, 31]),
    (1, 96, 1, 1, [90]), (1, 101, 1, 1, [321]), (1, 128, 1, 1, [64]), (1, 129, 1, 1, [64]), (1, 256, 2, 1, [200]),
    (1, 250, 1, 1, [0]), (1, 7, 36, 4, [200]),
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
    attend(rng, B, R, H, Hkv, lens, t, qscale=6.0)


def test_attention_in_parts_matches_oracle():
    """Prefixes long enough to be cut, into a workspace of NaN."""
    rng = np.random.default_rng(7)
    for B, R, H, Hkv, lens in ((1, 1, 4, 1, [3001]), (4, 1, 8, 2, [0, 64, 1500, 2999]), (1, 65, 2, 1, [2049]),
                               (3, 7, 4, 1, [5, 700, 1300]), (2, 33, 2, 2, [1000, 130]), (1, 20, 1, 1, [2500])):
        need = fc.fc_paged_byte_attention_workspace_bytes(B, R, H, Hkv, max(lens))
        say(f"attention in parts B={B} R={R} lens={lens} workspace={need}")
        assert need > 0
        pool = make_pool(rng, 30, Hkv)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        attend(rng, B, R, H, Hkv, lens, trees(rng, B, R), pool=pool, width=-(-max(lens) // 64), kw=dict(workspace=ws),
               max_len=max(lens))


def test_attention_bounds_and_absent_pages():
    rng = np.random.default_rng(8)
    pool = make_pool(rng, 8, 2)
    say("a longest length below a prefix, and above all; absent pages; one page far out")
    attend(rng, 2, 3, 4, 2, [500, 77], pool=pool, max_len=200, width=8)
    attend(rng, 2, 3, 4, 2, [100, 77], pool=pool, max_len=0, width=8)
    attend(rng, 2, 3, 4, 2, [10 ** 6, -4], pool=pool, width=8)
    for R in (1, 5, 20, 65):
        table = rng.integers(0, 8, (2, 6)).astype(np.int32)
        table[0, [0, 3]], table[1, [1, 4, 5]] = [-1, 8], [2 ** 31 - 1, -2 ** 31, -7]
        attend(rng, 2, R, 4, 2, [330, 290], pool=pool, table=table)
        attend(rng, 2, R, 4, 2, [330, 64], trees(rng, 2, R), pool=pool, table=np.full((2, 6), -1, np.int32))
    table = np.full((1, 2050), -1, np.int32)
    table[0, [0, 700, 2046]] = [3, 4, 5]
    attend(rng, 1, 5, 4, 2, [131_000], pool=pool, table=table)


@pytest.mark.parametrize("R,H", [(1, 4), (3, 4), (9, 2), (65, 2)])
def test_rows_that_see_nothing(R, H):
    """Masks that leave rows empty, trees of no rows, prefixes of no tokens."""
    rng = np.random.default_rng(R)
    t = trees(rng, 3, R)
    t["mask"][1] = 0
    t["mask"][2, ::2] = 0
    t["num_nodes"] = np.array([0, R, R], np.int32)
    say(f"rows that see nothing R={R}")
    got = attend(rng, 3, R, H, 1, [0, 0, 0], t)
    assert (got[0] == 0).all() and (got[1] == 0).all() and (got[2, ::2] == 0).all()
    attend(rng, 3, R, H, 1, [70, 0, 1], t)
    t["num_nodes"] = np.array([-5, R + 9, 1], np.int32)
    attend(rng, 3, R, H, 1, [70, 70, 70], t)


@pytest.mark.parametrize("R,H,Hkv", [(1, 4, 1), (5, 4, 1), (20, 2, 2), (65, 2, 1), (70, 4, 2)])
def test_what_is_not_finite_stays_where_it_is_seen(R, H, Hkv):
    """NaN and infinities in bytes past a prefix, in masked tree rows, in rows past
    the last, and in absent pages do not count; where they are seen they show."""
    rng = np.random.default_rng(R + H)
    n_pages = 6
    pool = make_pool(rng, n_pages, Hkv)
    spoilt = pool.clone()
    lens, table = [130, 33], np.array([[0, 1, 2], [3, 4, 5]], np.int32)
    for b, n in enumerate(lens):
        for t in range(n, 192):
            page = spoilt[table[b, t // 64]]
            page[:, t % 64 * 128:t % 64 * 128 + 128] = 127
            page[:, 8192:16384].view(-1, 4, 128, 16)[:, t % 64 // 16, :, t % 16] = 255
    spoilt[2, :, o8.SCALES + 1], spoilt[2, :, o8.SCALES + 3] = 255, 255     # blocks that nobody has begun
    spoilt[4, :, o8.SCALES:o8.SCALES + 4] = 0
    spoilt[5, :, o8.SCALES:o8.SCALES + 4] = 255
    t = trees(rng, 2, R)
    t["num_nodes"][1] = max(1, R - 1)
    q, kt, vt = bf16(rng, 2, R, H, D), bf16(rng, 2, R, Hkv, D), bf16(rng, 2, R, Hkv, D)
    say(f"not finite R={R}")
    args = lambda p, q, k, v: (q.cuda(), k.cuda(), v.cuda(), p, dev(table), dev(np.array(lens, np.int32)))  # noqa: E731
    want = fc.fc_paged_byte_attention(*args(pool, q, kt, vt), tree=on_gpu(t))
    q2, k2, v2 = q.clone(), kt.clone(), vt.clone()
    if R > 1:
        q2[1, R - 1], k2[1, R - 1], v2[1, R - 1] = NAN, INF, NAN
    got = fc.fc_paged_byte_attention(*args(spoilt, q2, k2, v2), tree=on_gpu(t))
    assert torch.equal(got, want)
    # seen: a tree row's values by its descendants, its key by them, a query's by itself
    if R > 1:
        j = R // 2
        v3, k3, q3 = vt.clone(), kt.clone(), q.clone()
        v3[0, j, 0, 9], v3[0, j, 0, 70] = NAN, INF
        attend(rng, 2, R, H, Hkv, lens, t, pool=spoilt, table=table, q=q, kt=kt, vt=v3)
        k3[0, j, 0, 3] = NAN
        attend(rng, 2, R, H, Hkv, lens, t, pool=spoilt, table=table, q=q, kt=k3, vt=vt)
        q3[0, 0, 0, 5] = NAN
        attend(rng, 2, R, H, Hkv, lens, t, pool=spoilt, table=table, q=q3, kt=kt, vt=vt)
    # a cached value that is none concerns its dim alone, a key every row
    seen = pool.clone()
    seen[1, 0, 8192 + 5 * 16 + 3] = 127
    a = attend(rng, 2, R, H, Hkv, lens, t, pool=seen, table=table, q=q, kt=kt, vt=vt)
    assert np.isnan(a[0, 0, 0, 5]) and not np.isnan(a[0, 0, 0, 6])
    seen[0, 0, 9] = 127
    a = attend(rng, 2, R, H, Hkv, lens, t, pool=seen, table=table, q=q, kt=kt, vt=vt)
    assert np.isnan(a[0, 0, 0]).all() and not np.isnan(a[1]).any()


def _along(rng, u, sizes):
    """A page per size: keys of that size along u or, every third, against it, and a little noise."""
    n = len(sizes)
    way = np.where(np.arange(64 * n) % 3 == 2, -1.0, 1.0) * np.repeat(sizes, 64)
    k = torch.from_numpy(way[:, None, None] * u + rng.standard_normal((64 * n, 1, D)) * 0.02).to(BF)
    pool = torch.zeros((n, 1, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_byte_write(pool, k.cuda(), bf16(rng, 64 * n, 1, D).cuda(), dev(np.arange(64 * n, dtype=np.int32)))
    return pool


@pytest.mark.parametrize("R,G", [(1, 1), (5, 2), (30, 1), (64, 1), (65, 1), (70, 4)])
def test_attention_of_scores_far_apart(R, G):
    """Scores that grow from page to page by far more than a weight's range, fall so,
    or do both, each row its own way."""
    rng = np.random.default_rng(R)
    u = rng.choice([-1.0, 1.0], D)
    for sizes in (np.linspace(0, 8, 12), np.linspace(8, 0, 12), np.abs(np.linspace(-8, 8, 12)),
                  8 * (np.arange(12) % 5 == 3), 2.0 ** np.linspace(-20, 3, 12)):
        pool = _along(rng, u, sizes)
        c = np.where(np.arange(R * G) % 4 == 3, -1.0, 1.0) * rng.uniform(0, 1, R * G)
        q = torch.from_numpy(c.reshape(1, R, G, 1) * u).to(BF)
        say(f"scores far apart R={R} G={G} sizes {sizes[0]:.3g} to {sizes[-1]:.3g}")
        for lens in ([768], [747]):
            attend(rng, 1, R, G, 1, lens, pool=pool, table=np.arange(12, dtype=np.int32)[None], q=q)


def test_attention_rows_do_not_move_each_other():
    rng = np.random.default_rng(21)
    u = rng.choice([-1.0, 1.0], D)
    pool = _along(rng, u, np.linspace(0, 8, 12))
    table, plen = dev(np.arange(12, dtype=np.int32)[None]), dev(np.array([760], np.int32))
    for R in (1, 9, 33, 65):
        G = 3 if R == 1 else 1
        q = bf16(rng, 1, R, G, D, scale=0.3)
        kt, vt = bf16(rng, 1, R, 1, D), bf16(rng, 1, R, 1, D)
        other = q.clone()
        change = np.arange(R * G) % 3 != 0
        other.view(R * G, D)[torch.from_numpy(change)] = torch.from_numpy(u).to(BF)
        other.view(R * G, D)[1] = NAN
        say(f"rows do not move each other R={R}")
        a, b = (fc.fc_paged_byte_attention(x.cuda(), kt.cuda(), vt.cuda(), pool, table, plen) for x in (q, other))
        a, b = (x.view(R * G, D).view(torch.int16).cpu().numpy() for x in (a, b))
        assert np.array_equal(a[~change], b[~change]) and not np.array_equal(a[change], b[change])


def test_blocks_of_far_scales():
    """Blocks whose scales lie far apart, at both ends of what a scale may be."""
    rng = np.random.default_rng(22)
    k, v = np.ones((256, 1, D)), rng.standard_normal((256, 1, D))
    v *= 2.0 ** np.repeat([0, 70, -100, 20, -126, 60, 0, 30], 32)[:, None, None]
    k *= 2.0 ** np.repeat([-120, 0, -60, 3, 1, -20, -100, 2], 32)[:, None, None] * rng.choice([-1, 1], (256, 1, D))
    pool = torch.zeros((4, 1, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_byte_write(pool, torch.from_numpy(k).to(BF).cuda(), torch.from_numpy(v).to(BF).cuda(),
                       dev(np.arange(256, dtype=np.int32)))
    for R in (1, 20, 65):
        say(f"far scales R={R}")
        attend(rng, 1, R, 1, 1, [256], pool=pool, table=np.arange(4, dtype=np.int32)[None], qscale=0.3)


@pytest.mark.parametrize("R,H,Hkv,n", [(1, 8, 2, 100), (1, 8, 2, 3000), (6, 8, 2, 3000), (65, 4, 4, 100), (70, 2, 1, 2000)])
def test_results_in_place_of_queries(R, H, Hkv, n):
    """out may be q, and lie beside what is read; anything between is refused."""
    rng = np.random.default_rng(R)
    B, width = 3, -(-n // 64)
    pool, table = make_pool(rng, 6, Hkv), dev(rng.integers(0, 6, (B, width)).astype(np.int32))
    lens = dev(np.array([n, n // 2, 0], np.int32))
    block = torch.empty((3 * B, R, H, 128), dtype=BF, device="cuda")
    q, kt, vt = block[B:2 * B], bf16(rng, B, R, Hkv, 128).cuda(), bf16(rng, B, R, Hkv, 128).cuda()
    q.copy_(bf16(rng, B, R, H, 128))
    t = on_gpu(trees(rng, B, R))
    say(f"in place R={R} n={n}")
    want = fc.fc_paged_byte_attention(q, kt, vt, pool, table, lens, tree=t)
    for out in (block[:B], block[2 * B:], q):
        assert torch.equal(want, fc.fc_paged_byte_attention(q, kt, vt, pool, table, lens, tree=t, out=out))
    for at in (B - 1, B + 1):
        with pytest.raises(fc.FcError):
            fc.fc_paged_byte_attention(q, kt, vt, pool, table, lens, tree=t, out=block[at:at + B])


def test_attention_of_slices():
    """Queries, keys and values as slices of one projection give the bits of copies."""
    rng = np.random.default_rng(23)
    for R in (1, 5, 33):
        B, H, Hkv = 2, 4, 2
        pool, table = make_pool(rng, 8, Hkv), dev(rng.integers(0, 8, (B, 5)).astype(np.int32))
        qkv = bf16(rng, B, R, H + 2 * Hkv, D).cuda()
        parts = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
        plen = dev(np.array([300, 77], np.int32))
        say(f"slices R={R}")
        a = fc.fc_paged_byte_attention(*parts, pool, table, plen)
        assert torch.equal(a, fc.fc_paged_byte_attention(*[p.clone() for p in parts], pool, table, plen))


def test_offsets_past_32_bits():
    """Pages beyond 4 GiB of one pool are written, read, attended, weighed and cut."""
    Hkv, n_pages = 16, 17_000                      # 4.5 GB
    assert fc.fc_paged_byte_pool_bytes(n_pages, Hkv) > 2 ** 32
    rng = np.random.default_rng(15)
    pool = torch.empty((n_pages, Hkv, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    small = torch.zeros((2, Hkv, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    w = [fc.paged_token_weights(n, Hkv, "cuda") for n in (n_pages, 2)]
    k, v = bf16(rng, 100, Hkv, D).cuda(), bf16(rng, 100, Hkv, D).cuda()
    tables, pos = [np.array([[n_pages - 1, n_pages - 2]], np.int32), np.array([[0, 1]], np.int32)], np.arange(100)
    q, kt, vt = (bf16(rng, 1, 3, Hkv, D).cuda() for _ in "qkv")
    got = []
    say("past 4 GiB")
    for p, table, wt in zip((pool, small), tables, w):
        slot = dev((table[0, pos // 64] * 64 + pos % 64).astype(np.int32))
        n = dev(np.array([100], np.int32))
        fc.fc_paged_byte_write(p, k, v, slot)
        lse = torch.empty((1, 3, Hkv), device="cuda")
        out = fc.fc_paged_byte_attention(q, kt, vt, p, dev(table), n, lse=lse)
        fc.fc_paged_byte_weights(wt, q, lse, p, dev(table), n - 3, n, dev(np.array([0, 3], np.int32)))
        add = fc.fc_paged_byte_evict(p, wt, dev(table), n, n - 31, first=2, recent=5)
        rows = fc.fc_paged_byte_read(p, slot[:69])
        got.append([out, lse, wt[torch.from_numpy(table[0]).long().cuda()], add, *rows])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][4].any()


def test_more_trees_than_one_launch_takes():
    rng = np.random.default_rng(2)
    for B, R, Hkv, piece in ((65536, 1, 64, 30000), (5000, 40, 8, 2300)):
        pool = make_pool(rng, 40, Hkv)
        torch.manual_seed(2)
        x = torch.randn((B, R, Hkv, D), dtype=BF, device="cuda")
        table = torch.randint(0, 40, (B, 2), dtype=torch.int32, device="cuda")
        plen = torch.randint(0, 129, (B,), dtype=torch.int32, device="cuda")
        say(f"attention of {B} trees of {R} rows")
        got = fc.fc_paged_byte_attention(x, x, x, pool, table, plen)
        for i in range(0, B, piece):
            want = fc.fc_paged_byte_attention(*[x[i:i + piece]] * 3, pool, table[i:i + piece], plen[i:i + piece])
            assert torch.equal(got[i:i + piece], want), i


# ---------------------------------------------------------------- weights --

def weigh(rng, H, Hkv, lens, adds, n_src=None, table=None, pool=None, width=None, max_len=None, lse=None, shift=0):
    """One call against the oracle: every weight of the pool, those that are left alone too."""
    B, new = len(lens), [n + a for n, a in zip(lens, adds)]
    n_pages = sum(-(-max(n, 0) // 64) for n in new) + 2
    pool = make_pool(rng, n_pages, Hkv) if pool is None else pool
    width = width or max(1, max(-(-max(n, 0) // 64) for n in new))
    if table is None:
        perm, at = rng.permutation(pool.shape[0]).astype(np.int32), 0
        table = np.full((B, width), -1, np.int32)
        for b, n in enumerate(new):
            m = min(-(-max(n, 0) // 64), width)
            table[b, :m] = perm[at:at + m]
            at += m
    cu = (np.concatenate([[0], np.cumsum(np.maximum(adds, 0))]) + shift).astype(np.int32)
    n = max(int(cu[-1]), 1)
    rows = n_src or n
    src = None if n_src is None else rng.integers(0, rows, n).astype(np.int32)
    q = bf16(rng, rows, H, D, scale=1.5)
    lse = rng.uniform(0, 8, (rows, H)).astype(np.float32) if lse is None else lse(rows)
    w = rng.uniform(0, 3, (pool.shape[0], Hkv, 64)).astype(np.float32)
    got = dev(w)
    args = (q.cuda(), dev(lse), pool, dev(table), dev(np.array(lens, np.int32)), dev(np.array(new, np.int32)), dev(cu))
    for again in range(2):
        got.copy_(dev(w))
        fc.fc_paged_byte_weights(got, *args, src=None if src is None else dev(src), max_len=max_len)
        first = got.clone() if not again else first
    assert torch.equal(got.view(torch.int32), first.view(torch.int32))
    want, most = o8.weights(w, f64(q), lse, host(pool), table, lens, new, cu, src, max_len)
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~(np.isnan(want) | (got == want) | (np.abs(got - want) <= most))
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), float(np.nanmax(np.abs(got - want) / (most + 1e-30))))
    return got


@pytest.mark.parametrize("H,Hkv,lens,adds", [
    (1, 1, [0], [1]), (4, 1, [0, 63], [1, 1]), (8, 2, [64, 0, 300], [1, 11, 5]), (5, 5, [31, 1], [40, 3]),
    (17, 1, [100], [9]), (2, 2, [0], [200]), (6, 2, [70, 500], [130, 70]), (1, 1, [1000], [33]), (3, 1, [10, 20], [0, 0]),
])
def test_weights_match_oracle(H, Hkv, lens, adds):
    rng = np.random.default_rng(H + sum(lens))
    say(f"weights H={H} Hkv={Hkv} lens={lens} adds={adds}")
    weigh(rng, H, Hkv, lens, adds)
    weigh(rng, H, Hkv, lens, adds, n_src=sum(adds) + 5)


def test_weights_that_are_left_alone():
    """Sequences that lose tokens or gain none, rows outside of what there is, rows
    that attended to nothing, absent pages, a longest length, weights that are none."""
    rng = np.random.default_rng(9)
    say("weights left alone")
    weigh(rng, 4, 2, [70, 5, 90, 0], [0, 3, -20, 0])
    weigh(rng, 4, 2, [70, 5], [9, 20], shift=-3)
    weigh(rng, 4, 2, [70, 5], [9, 20], shift=12)
    none = lambda n: np.where(rng.random((n, 4)) < 0.5, -np.inf, rng.uniform(0, 8, (n, 4))).astype(np.float32)  # noqa: E731
    weigh(rng, 4, 2, [70, 5], [9, 20], lse=none)
    nan = lambda n: np.where(rng.random((n, 4)) < 0.1, np.nan, rng.uniform(0, 8, (n, 4))).astype(np.float32)  # noqa: E731
    weigh(rng, 4, 2, [70, 5], [9, 20], lse=nan)
    weigh(rng, 4, 2, [70, 200], [9, 20], max_len=128)
    table = np.array([[0, -1, 2], [3, 99, 4]], np.int32)
    weigh(rng, 4, 2, [130, 70], [9, 90], table=table, pool=make_pool(rng, 6, 2))


def test_weights_of_keys_that_are_none():
    """NaN bytes behind the last token and blocks nobody began count for nothing; a key
    that is a NaN pays into its own weight alone."""
    rng = np.random.default_rng(10)
    pool = make_pool(rng, 3, 1)
    table = np.array([[1, 2]], np.int32)
    pool[2, 0, 10 * 128:64 * 128] = 127
    pool[2, 0, o8.SCALES + 1] = 255
    pool[1, 0, 7 * 128 + 5] = 127
    say("keys that are none")
    for add in (2, 50):
        got = weigh(rng, 3, 1, [74 - add], [add], table=table, pool=pool)
        assert np.isnan(got[1, 0, 7]) and np.isnan(got).sum() == 1


# ------------------------------------------------------------------ evict --

def cut(rng, Hkv, lens, budgets, first=0, recent=0, weights=None, table=None, max_len=None, ws=None):
    n_pages = sum(-(-max(n, 0) // 64) for n in lens) + 2
    pool = make_pool(rng, n_pages, Hkv)
    B, width = len(lens), max(1, max(-(-max(n, 0) // 64) for n in lens))
    if table is None:
        perm, at = rng.permutation(n_pages).astype(np.int32), 0
        table = np.full((B, width), -1, np.int32)
        for b, n in enumerate(lens):
            m = -(-max(n, 0) // 64)
            table[b, :m] = perm[at:at + m]
            at += m
    w = rng.uniform(0, 1, (n_pages, Hkv, 64)).astype(np.float32) ** 4 if weights is None else weights((n_pages, Hkv, 64))
    want_pool, want_w, want_add = o8.evict(host(pool), w, table, lens, budgets, first, recent, max_len)
    got = dev(w)
    kw = {} if ws is None else dict(workspace=ws)
    add = fc.fc_paged_byte_evict(pool, got, dev(table), dev(np.array(lens, np.int32)), dev(np.array(budgets, np.int32)),
                             first=first, recent=recent, max_len=max_len, **kw)
    torch.cuda.synchronize()
    assert np.array_equal(host(add), want_add)
    assert np.array_equal(host(got).view(np.int32), want_w.view(np.int32))
    same_pool(pool, want_pool)


@pytest.mark.parametrize("Hkv,lens,budgets,first,recent", [
    (1, [2], [1], 0, 0), (1, [64], [63], 0, 0), (2, [65, 64], [64, 10], 1, 2), (3, [200, 10, 0], [100, 50, 5], 4, 16),
    (1, [640], [129], 0, 64), (2, [300, 301], [33, 0], 3, 3), (1, [1000], [999], 10, 10), (1, [500], [40], 100, 20),
    (1, [500], [40], 30, 50), (2, [130, 129, 128], [128, 128, 128], 0, 0), (1, [2300], [1100], 4, 200),
    (8, [90], [31], 4, 8), (1, [70], [-5], 0, 0), (1, [200], [150], 500, 0), (1, [200], [150], 0, 500),
], ids=lambda x: str(x).replace(" ", ""))
def test_evictions_match_oracle(Hkv, lens, budgets, first, recent):
    rng = np.random.default_rng(sum(lens) + first)
    say(f"evict Hkv={Hkv} lens={lens} budgets={budgets} first={first} recent={recent}")
    cut(rng, Hkv, lens, budgets, first, recent)


def test_evictions_by_equal_and_odd_weights():
    """Weights that are equal, negative, NaN, infinite, the least there are, or differ in
    their last bit."""
    rng = np.random.default_rng(11)
    pick = lambda *v: lambda s: rng.choice(np.array(v, np.float32), s)  # noqa: E731
    last = lambda s: (np.float32(1.0).view(np.int32) + rng.integers(0, 3, s)).astype(np.int32).view(np.float32)  # noqa: E731
    for name, w in (("equal", pick(1.0)), ("zeros", pick(0.0, -0.0)), ("two kinds", pick(1.0, 2.0)),
                    ("odd", pick(NAN, INF, -INF, -1.0, 0.0, 1e-45, 3.4e38, 1.0)), ("last bits", last)):
        say(f"evict by {name} weights")
        cut(rng, 2, [700, 65], [300, 64], 2, 9, weights=w)


def test_evictions_of_absent_pages_and_bounds():
    rng = np.random.default_rng(12)
    say("evict with absent pages, a longest length, a workspace of ones")
    table = np.array([[0, -1, 2, 1, 99], [5, 6, 3, 4, -2]], np.int32)
    cut(rng, 2, [300, 260], [130, 200], 2, 9, table=table)
    cut(rng, 2, [300, 100], [90, 60], 2, 9, max_len=192)
    need = fc.fc_paged_byte_evict_workspace_bytes(2, 2, 5 * 64)
    ws = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
    cut(rng, 2, [300, 100], [90, 60], 2, 9, ws=ws[:need])
    with pytest.raises(fc.FcError):
        cut(rng, 2, [300, 100], [90, 60], 2, 9, ws=ws[:need - 1])
    with pytest.raises(fc.FcError):
        cut(rng, 2, [300, 100], [90, 60], 2, 9, ws=ws[8:8 + need])


def test_a_long_eviction():
    """Many pages of one head, with a budget near the length, near half, and small: each
    page waits for those ahead of it."""
    torch.manual_seed(3)
    n, pages = 40_000, 625
    slot = torch.arange(n, dtype=torch.int32, device="cuda")
    x = torch.randn((n, 2, D), device="cuda").to(BF)
    table = torch.randperm(pages, device="cuda").int()[None].contiguous()
    place = (table[0, (slot // 64).long()] * 64 + slot % 64).int()
    pool = fc.paged_byte_pool(pages, 2, "cuda")
    fc.fc_paged_byte_write(pool, x, x, place)
    w = torch.rand((pages, 2, 64), device="cuda")
    for keep in (39_999, 39_000, 20_011, 700):
        say(f"a long eviction to {keep}")
        p, wt = pool.clone(), w.clone()
        add = fc.fc_paged_byte_evict(p, wt, table, torch.tensor([n], dtype=torch.int32, device="cuda"),
                                 torch.tensor([keep], dtype=torch.int32, device="cuda"))
        assert int(add) == keep - n
        k, v = fc.fc_paged_byte_read(p, place[:keep])
        was_k, was_v = fc.fc_paged_byte_read(pool, place)
        flat = w[table[0].long()].transpose(1, 2).reshape(n, 2)
        moved = wt[table[0].long()].transpose(1, 2).reshape(n, 2)
        for h in range(2):
            stay = torch.sort(flat[:, h], dim=0, descending=True, stable=True).indices[:keep].sort().values
            assert torch.equal(moved[:keep, h], flat[stay, h]) and torch.equal(moved[keep:, h], flat[keep:, h])
            for got, was in ((k, was_k), (v, was_v)):
                a, b = got[:, h].float(), was[stay, h].float()
                # rounded once more where the block's scale is another: half a step
                assert ((a - b).abs() <= 2.0 ** -4 * b.abs() + 2.0 ** -8).all() and (a == b).float().mean() > 0.9


# ------------------------------------------------- together, streams, graphs --

def test_a_serving_loop_that_forgets():
    """Prompts in, then steps of trees: norms and rotation, attention, acceptance,
    plans, writes, token weights, and evictions whose pages the plan gives back; on
    both sides, every byte of the cache equal and every number within its bound."""
    rng = np.random.default_rng(16)
    B, R, H, Hkv, n_pages, width = 3, 9, 4, 2, 11, 5
    s = fc.paged_state(B, width, n_pages, "cuda")
    pool, w = fc.paged_byte_pool(n_pages, Hkv, "cuda").zero_(), fc.paged_token_weights(n_pages, Hkv, "cuda")
    seen = np.zeros(B, np.int64)                     # positions, which go on when tokens leave
    weight = (1 + bf16(rng, D, scale=0.2)).cuda()

    def plan(add, n_slots, **kw):
        p = fc.fc_paged_plan(s["len"], add, s["table"], s["queue"], s["ends"], n_slots, **kw)
        old = s["len"]
        s.update(len=p["len"], ends=p["ends"])
        return old, p

    def enter(k, v, q, lse, old, p):
        """The step's rows go in and pay for what they saw; both sides."""
        o_pool = o8.write(host(pool), f64(k).reshape(-1, Hkv, D), f64(v).reshape(-1, Hkv, D), host(p["slot"]), host(p["src"]))
        fc.fc_paged_byte_write(pool, k, v, p["slot"], src=p["src"])
        same_pool(pool, o_pool)
        o_w, most = o8.weights(host(w), f64(q).reshape(-1, H, D), f64(lse).reshape(-1, H), o_pool, host(s["table"]),
                               host(old), host(p["len"]), host(p["cu"]), host(p["src"]))
        fc.fc_paged_byte_weights(w, q, lse, pool, s["table"], old, p["len"], p["cu"], src=p["src"])
        assert (np.abs(f64(w) - o_w) <= most).all()

    add = np.array([70, 1, 129], np.int32)
    n = int(add.sum())
    old, p = plan(dev(add), n + 3)
    q, k, v = (bf16(rng, n, h, D).cuda() for h in (H, Hkv, Hkv))
    q, k = fc.fc_norm_rotate(q, k, weight, weight, dev(np.concatenate([np.arange(a) for a in add]).astype(np.int32)))
    enter(k, v, q, torch.full((n, H), 4.0, device="cuda"), old, p)
    seen += add
    for step in range(6):
        say(f"serving step {step}")
        t = trees(rng, B, R, 5)
        t["node_tok"] = rng.integers(1, 50, (B, R)).astype(np.int32)
        target = rng.integers(-1, 50, (B, R)).astype(np.int32)
        for b in range(B):
            for i in range(1, R):
                if rng.random() < 0.7:
                    target[b, t["parent"][b, i]] = t["node_tok"][b, i]
        q, k, v = (bf16(rng, B, R, h, D).cuda() for h in (H, Hkv, Hkv))
        q, k = fc.fc_norm_rotate(q, k, weight, weight, dev((seen[:, None] + t["pos_ids"]).astype(np.int32)))
        lse = torch.empty((B, R, H), device="cuda")
        got = fc.fc_paged_byte_attention(q, k, v, pool, s["table"], s["len"], tree=on_gpu(t), lse=lse)
        o, o_lse, most, lse_most = o8.attention(f64(q), f64(k), f64(v), host(pool), host(s["table"]), host(s["len"]),
                                                t["num_nodes"], t["mask"])
        assert (np.abs(f64(got) - o) <= most).all() and (np.abs(f64(lse) - o_lse) <= lse_most).all()
        a = fc.fc_verify_accept(on_gpu(t), dev(target), m=5)
        old, p = plan(a["accept_len"], B * 6, tree=on_gpu(t), last_node=a["last_node"])
        seen += host(p["len"]) - host(old)
        enter(k, v, q, lse, old, p)
        if step % 2:
            budget = np.array([40, 30, 100 - 10 * step], np.int32)
            o_pool, o_w, o_add = o8.evict(host(pool), host(w), host(s["table"]), host(s["len"]), budget, 2, 8)
            cut_by = fc.fc_paged_byte_evict(pool, w, s["table"], s["len"], dev(budget), first=2, recent=8)
            same_pool(pool, o_pool)
            assert np.array_equal(host(cut_by), o_add) and np.array_equal(host(w), o_w)
            free = int(s["ends"][1] - s["ends"][0])
            plan(cut_by, 0)
            assert (host(s["len"]) <= np.maximum(budget, 0)).all() and int(s["ends"][1] - s["ends"][0]) >= free
    assert (seen > host(s["len"])).any()


def _state(rng, B=2, R=9, H=8, Hkv=2, n=700):
    pool = make_pool(rng, 12, Hkv)
    return dict(q=bf16(rng, B, R, H, D).cuda(), k_tree=bf16(rng, B, R, Hkv, D).cuda(),
                v_tree=bf16(rng, B, R, Hkv, D).cuda(), pool=pool,
                table=dev(rng.integers(0, 12, (B, -(-n // 64))).astype(np.int32)),
                prefix_len=dev(np.array([n, n // 3], np.int32)), tree=on_gpu(trees(rng, B, R)))


def test_attention_workspaces_and_repeats():
    rng = np.random.default_rng(17)
    s = _state(rng)
    need = fc.fc_paged_byte_attention_workspace_bytes(2, 9, 8, 2, 11 * 64)
    assert need > 0
    say("workspaces")
    want = fc.fc_paged_byte_attention(**s)
    ws = torch.full((need + 32,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(want, fc.fc_paged_byte_attention(**s, workspace=ws[:need]))
    assert torch.equal(want, fc.fc_paged_byte_attention(**s))
    for bad in (ws[:need - 1], ws[8:8 + need]):
        with pytest.raises(fc.FcError):
            fc.fc_paged_byte_attention(**s, workspace=bad)


def test_calls_on_another_stream():
    """Calls on a side stream while the current one still reads blocks that it has freed,
    of the sizes of the calls' own tensors."""
    rng = np.random.default_rng(18)
    s = _state(rng)
    want = fc.fc_paged_byte_attention(**s)
    slot = dev(np.arange(12 * 64, dtype=np.int32))
    k, v = fc.fc_paged_byte_read(s["pool"], slot)
    table, n = dev(np.arange(12, dtype=np.int32)[None]), dev(np.array([768], np.int32))
    w = torch.rand((12, 2, 64), device="cuda")
    p1, w1 = s["pool"].clone(), w.clone()
    fc.fc_paged_byte_evict(p1, w1, table, n, n - 300, recent=7)
    side, a = torch.cuda.Stream(), torch.rand(6144, 6144, device="cuda")
    sizes = [fc.fc_paged_byte_attention_workspace_bytes(2, 9, 8, 2, 11 * 64), want.numel() * 2, k.numel() * 2,
             fc.fc_paged_byte_evict_workspace_bytes(1, 2, 768)]
    say("side stream")
    for i in range(3):
        p2, w2, budget = s["pool"].clone(), w.clone(), n - 300
        busy = [torch.full((m // 4 + 1,), i + 1, dtype=torch.int32, device="cuda") for m in sizes]
        seen = [torch.empty_like(x) for x in busy]
        torch.cuda.synchronize()
        a @ a
        for x, y in zip(busy, seen):
            y.copy_(x)
        del busy, x
        got = fc.fc_paged_byte_attention(**s, stream=side)
        k2, v2 = fc.fc_paged_byte_read(s["pool"], slot, stream=side)
        fc.fc_paged_byte_evict(p2, w2, table, n, budget, recent=7, stream=side)
        torch.cuda.synchronize()
        assert all((x == i + 1).all() for x in seen)
        assert torch.equal(got, want) and torch.equal(k, k2) and torch.equal(v, v2)
        assert torch.equal(p1, p2) and torch.equal(w1, w2)


def test_a_step_in_a_captured_graph():
    """A whole step - norm, attention, plan, write, weights, eviction - captured: every
    replay, on new inputs and with other work between, gives the eager results."""
    rng = np.random.default_rng(19)
    B, R, H, Hkv, n_pages, width = 2, 9, 8, 2, 30, 12
    s = fc.paged_state(B, width, n_pages, "cuda")
    pool = make_pool(rng, n_pages, Hkv)
    w = torch.rand((n_pages, Hkv, 64), device="cuda")
    first = fc.fc_paged_plan(s["len"], dev(np.array([600, 130], np.int32)), s["table"], s["queue"], s["ends"], 730)
    new = lambda h: bf16(rng, B, R, h, D).cuda()  # noqa: E731
    q, k, v = new(H), new(Hkv), new(Hkv)
    t = on_gpu(trees(rng, B, R))
    add, last = dev(np.array([2, 1], np.int32)), dev(np.array([5, 0], np.int32))
    lens, ends, pos = first["len"].clone(), first["ends"].clone(), dev(rng.integers(0, 900, (B, R)).astype(np.int32))
    budget = dev(np.array([590, 125], np.int32))

    def step():
        a, b = fc.fc_norm_rotate(q, k, pos=pos)
        lse = torch.empty((B, R, H), device="cuda")
        out = fc.fc_paged_byte_attention(a, b, v, pool, s["table"], lens, tree=t, lse=lse)
        p = fc.fc_paged_plan(lens, add, s["table"], s["queue"], ends, 2 * R, tree=t, last_node=last)
        fc.fc_paged_byte_write(pool, b, v, p["slot"], src=p["src"])
        fc.fc_paged_byte_weights(w, a, lse, pool, s["table"], lens, p["len"], p["cu"], src=p["src"])
        return p, out, lse, fc.fc_paged_byte_evict(pool, w, s["table"], p["len"], budget, first=2, recent=30)

    say("a step captured")
    keep = pool.clone(), w.clone()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p, out, lse, less = step()
    for i in range(4):
        for x in (q, k, v):
            x.copy_(new(x.shape[2]))
        row = torch.randint(0, R, (B,), device="cuda", dtype=torch.int32)
        last.copy_(row)
        add.copy_(t["pos_ids"].gather(1, row[:, None].long())[:, 0] + 1)
        pool.copy_(keep[0])
        w.copy_(keep[1])
        graph.replay()
        got = [x.clone() for x in (out, lse, less, pool, w, *p.values())]
        busy = torch.full((8 << 20,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        pool.copy_(keep[0])
        w.copy_(keep[1])
        p2, *more = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, [*more, pool, w, *p2.values()])), i
        del busy


def test_graphs_that_share_a_workspace():
    """Two captured calls of each kind with one workspace, replayed in turn."""
    rng = np.random.default_rng(20)
    a, b = _state(rng), _state(rng)
    ws = torch.empty(max(fc.fc_paged_byte_attention_workspace_bytes(2, 9, 8, 2, 11 * 64),
                         fc.fc_paged_byte_evict_workspace_bytes(1, 2, 768)), dtype=torch.uint8, device="cuda")
    table, n = dev(np.arange(12, dtype=np.int32)[None]), dev(np.array([768], np.int32))
    runs = []
    say("graphs that share a workspace")
    for i, s in enumerate((a, b)):
        base, w0 = s["pool"].clone(), torch.rand((12, 2, 64), device="cuda")
        w, budget = w0.clone(), n - 100 * (i + 1)

        def run(s=s, w=w, budget=budget):
            out = fc.fc_paged_byte_attention(**s, workspace=ws)
            return out, fc.fc_paged_byte_evict(s["pool"], w, table, n, budget, recent=5, workspace=ws)

        want = [x.clone() for x in (*run(), s["pool"], w)]
        s["pool"].copy_(base)
        w.copy_(w0)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = run()
        runs.append((g, res, s, w, base, w0, want, budget))  # what a graph reads lives as long as it does
    for i in (0, 1, 1, 0, 1, 0):
        g, res, s, w, base, w0, want, _ = runs[i]
        s["pool"].copy_(base)
        w.copy_(w0)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((*res, s["pool"], w), want)), i


def test_calls_side_by_side():
    """The same calls on several streams at once, each with its own buffers."""
    rng = np.random.default_rng(24)
    s = _state(rng)
    table, n = dev(np.arange(12, dtype=np.int32)[None]), dev(np.array([768], np.int32))
    w, budget = torch.rand((12, 2, 64), device="cuda"), dev(np.array([333], np.int32))
    want = fc.fc_paged_byte_attention(**s)
    p0, w0 = s["pool"].clone(), w.clone()
    fc.fc_paged_byte_evict(p0, w0, table, n, budget)
    streams = [torch.cuda.Stream() for _ in range(5)]
    copies = [(s["pool"].clone(), w.clone()) for _ in streams]
    torch.cuda.synchronize()
    say("side by side")
    outs = []
    for again in range(4):
        for st, (p, x) in zip(streams, copies):
            with torch.cuda.stream(st):
                p.copy_(s["pool"])
                x.copy_(w)
                outs.append(fc.fc_paged_byte_attention(**s))
                fc.fc_paged_byte_evict(p, x, table, n, budget)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    assert all(torch.equal(p, p0) and torch.equal(x, w0) for p, x in copies)


def test_the_4_bit_cache_takes_rows_rotated_before():
    """fc_norm_rotate without norms, then rope_base 0, is the 4-bit cache's own rotation
    but for one rounding to bf16."""
    rng = np.random.default_rng(25)
    n, Hkv = 64, 2
    k, v = bf16(rng, n, Hkv, D), bf16(rng, n, Hkv, D)
    pos = rng.integers(0, 3000, n).astype(np.int32)
    slot = dev(np.arange(n, dtype=np.int32))
    say("4-bit pages of rotated rows")
    pool = fc.paged_pool(1, Hkv, "cuda")
    rotated = fc.fc_norm_rotate(None, k.cuda(), pos=dev(pos))[1]
    fc.fc_paged_write(pool, rotated, v.cuda(), slot, rope_base=0.0)
    want = oracle.paged_write(np.zeros_like(host(pool)), f64(rotated), f64(v), np.arange(n), rope_base=0.0)
    assert np.array_equal(host(pool), want)
    exact = np.stack([oracle.rope(f64(k)[:, h], pos, 10000.0) for h in range(Hkv)], 1)
    pair = np.abs(f64(k))
    assert (np.abs(f64(rotated) - exact) <= 2.0 ** -8 * np.abs(exact) + 2.0 ** -15 * (pair + np.roll(pair, 64, -1))).all()


def test_refusals_on_the_gpu():
    rng = np.random.default_rng(26)
    s = _state(rng)
    say("refusals")
    with pytest.raises(fc.FcError):
        fc.fc_paged_byte_attention(**s, max_len=11 * 64 + 1)
    with pytest.raises(ValueError, match="one device"):
        fc.fc_paged_byte_attention(**{**s, "prefix_len": s["prefix_len"].cpu()})
    with pytest.raises(ValueError, match="pool"):
        fc.fc_paged_byte_attention(**{**s, "pool": fc.paged_pool(3, 2, "cuda")})
    with pytest.raises(fc.FcError):
        fc.fc_norm_rotate(s["q"], s["k_tree"], pos=torch.zeros(18, dtype=torch.int32, device="cuda"), rope_base=1.0)
    w = fc.paged_token_weights(12, 2, "cuda")
    n = dev(np.array([5, 6], np.int32))
    with pytest.raises(fc.FcError):
        fc.fc_paged_byte_evict(s["pool"], w, s["table"], n, n, first=-1)
    with pytest.raises(fc.FcError):
        fc.fc_paged_byte_evict(s["pool"], w, s["table"], n, n, add=n)
    with pytest.raises(ValueError, match="lse"):
        fc.fc_paged_byte_weights(w, s["q"], torch.zeros((2, 9, 4), device="cuda"), s["pool"], s["table"], n, n,
                             dev(np.zeros(3, np.int32)))


def test_evictions_of_far_scales():
    """Tokens of blocks whose scales lie far apart meet in one: the largest decides, small
    codes become smaller or nothing; blocks of nothing but the least codes, of zeros, and
    of NaN."""
    rng = np.random.default_rng(27)
    n, Hkv = 512, 2
    powers = np.repeat(rng.integers(-110, 100, n // 32), 32)
    kinds = [2.0 ** powers, 2.0 ** np.repeat([0, 3, -9, 1], n // 4), np.zeros(n), np.full(n, np.nan)]
    for i, scale in enumerate(kinds):
        k, v = (torch.from_numpy(rng.standard_normal((n, Hkv, D)) * scale[:, None, None]).to(BF) for _ in "kv")
        if i == 1:  # every block has one large row, which leaves; the others' codes are below 8
            k[::32], v[::32] = k[::32] * 2 ** 17, v[::32] * 2 ** 17
        pool = torch.zeros((n // 64, Hkv, fc.FC_PAGE8_HEAD_BYTES), dtype=torch.uint8, device="cuda")
        fc.fc_paged_byte_write(pool, k.cuda(), v.cuda(), dev(np.arange(n, dtype=np.int32)))
        w = rng.uniform(0.1, 1, (n // 64, Hkv, 64)).astype(np.float32)
        w[:, :, ::32] = 0
        table = np.arange(n // 64, dtype=np.int32)[None]
        say(f"evict of far scales, kind {i}")
        for budget in (496, 300, 33):
            got, gw = pool.clone(), dev(w)
            want, ww, _ = o8.evict(host(pool), w, table, [n], [budget])
            fc.fc_paged_byte_evict(got, gw, dev(table), dev(np.array([n], np.int32)), dev(np.array([budget], np.int32)))
            same_pool(got, want, (i, budget))
            assert np.array_equal(host(gw), ww)


@pytest.mark.parametrize("n,budget,first,recent", [(16_385, 9_000, 0, 0), (40_000, 17_000, 5, 300), (33_000, 32_999, 4, 0),
                                                   (50_000, 700, 900, 600)])
def test_evictions_in_parts(n, budget, first, recent):
    """More tokens than one workgroup weighs: counted in parts, with equal weights across
    their borders, beside a short sequence and one that stays."""
    rng = np.random.default_rng(n)
    lens, budgets = [300, n, 64], [120, budget, 64]
    pages = [-(-x // 64) for x in lens]
    perm = rng.permutation(sum(pages) + 3).astype(np.int32)
    table, at = np.full((3, max(pages)), -1, np.int32), 0
    for b, m in enumerate(pages):
        table[b, :m] = perm[at:at + m]
        at += m
    torch.manual_seed(n)
    pool = fc.paged_byte_pool(len(perm), 1, "cuda")
    x = torch.randn((64 * len(perm), 1, D), device="cuda").to(BF)
    fc.fc_paged_byte_write(pool, x, x.flip(0), torch.arange(64 * len(perm), dtype=torch.int32, device="cuda"))
    for weights in (rng.uniform(0, 1, (len(perm), 1, 64)), rng.integers(0, 3, (len(perm), 1, 64))):
        w = weights.astype(np.float32)
        say(f"evict in parts {n} to {budget}")
        want, ww, add = o8.evict(host(pool), w, table, lens, budgets, first, recent)
        got, gw = pool.clone(), dev(w)
        got_add = fc.fc_paged_byte_evict(got, gw, dev(table), dev(np.array(lens, np.int32)), dev(np.array(budgets, np.int32)),
                                         first=first, recent=recent)
        assert np.array_equal(host(got_add), add) and np.array_equal(host(gw), ww)
        same_pool(got, want)


def test_more_sequences_and_pages_than_one_launch_takes():
    """Pairs past 2^20 and tables of 2^17 pages: weights and evictions are those of calls
    with fewer sequences, and of narrower tables."""
    rng = np.random.default_rng(28)
    B, Hkv = 33_000, 32
    pool = make_pool(rng, B // 500, Hkv)
    pool = pool.repeat(500, 1, 1)[:B].contiguous()
    table = torch.randperm(B, device="cuda").int()[:, None].contiguous()
    n, cu = torch.full((B,), 40, dtype=torch.int32, device="cuda"), torch.arange(B + 1, dtype=torch.int32, device="cuda")
    q, lse = bf16(rng, B, Hkv, D).cuda(), torch.rand((B, Hkv), device="cuda") * 4
    budget = torch.randint(0, 41, (B,), dtype=torch.int32, device="cuda")
    w = torch.rand((B, Hkv, 64), device="cuda")
    a, b = (pool.clone(), w.clone()), (pool, w)
    say("more pairs than a launch takes")
    fc.fc_paged_byte_weights(a[1], q, lse, a[0], table, n - 1, n, cu)
    add = fc.fc_paged_byte_evict(*a, table, n, budget)
    for i in range(0, B, 11_000):
        s = slice(i, i + 11_000)
        fc.fc_paged_byte_weights(b[1], q, lse, b[0], table[s], n[s] - 1, n[s], cu[i:i + 11_001].contiguous())
    for i in range(0, B, 11_000):
        s = slice(i, i + 11_000)
        assert torch.equal(add[s], fc.fc_paged_byte_evict(*b, table[s], n[s], budget[s]))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    del a, b, pool, w
    wide = torch.full((1, 2 ** 17 + 3), -1, dtype=torch.int32, device="cuda")
    wide[0, :5] = torch.arange(5, device="cuda")
    pool, w = make_pool(rng, 5, 1), torch.rand((5, 1, 64), device="cuda")
    n = torch.tensor([300], dtype=torch.int32, device="cuda")
    got = []
    say("wide tables")
    # The table's width may change the order in which weights are added, so these are
    # held against the oracle, whose bounds cover every order, and not against each other.
    for rows in (2, 200):
        for width in (wide.shape[1], 5):
            weigh(np.random.default_rng(rows), 3, 1, [300 - rows], [rows], width=width)
    for t in (wide, wide[:, :5].contiguous()):
        for rows in (2, 200):
            p, x = pool.clone(), w.clone()
            q = bf16(np.random.default_rng(rows), rows, 3, D).cuda()
            out = fc.fc_paged_byte_attention(q[None, :2], pool.new_zeros((1, 2, 1, 256)).view(BF), q[None, :2, :1].contiguous(), p, t, n)
            fc.fc_paged_byte_evict(p, x, t, n, n - 77, recent=9)
            got.append((p, x, out))
    for x, y in zip(got[:2], got[2:]):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
        assert (x[2].float() - y[2].float()).abs().max() < 0.03      # other parts: a weight's rounding


@pytest.mark.parametrize("B,R,H,Hkv", [(140, 9, 16, 4), (270, 9, 8, 2), (300, 1, 8, 2), (130, 2, 16, 8)])
@pytest.mark.parametrize("how", ["mixed", "same", "none", "one"])
def test_attention_of_more_workgroups_than_run_at_once(B, R, H, Hkv, how):
    """Trees taken longest first, with ties, with empty prefixes, and with more of them
    than are put in order: each is still answered once."""
    rng = np.random.default_rng(B + R)
    lens = {"mixed": rng.integers(0, 260, B), "same": np.full(B, 130), "none": np.zeros(B, int),
            "one": np.where(np.arange(B) == B // 2, 300, 0)}[how].tolist()
    say(f"attention of many {B},{R},{H},{Hkv} {how}")
    pool = make_pool(rng, 50, Hkv)
    attend(rng, B, R, H, Hkv, lens, pool=pool, width=5, tree=trees(rng, B, R) if how == "mixed" else None)


@pytest.mark.parametrize("H,Hkv,lens,adds", [
    (3, 1, [200], [700]),            # 2,100 rows, three heads: rounds end inside a token
    (5, 1, [0, 640], [300, 1]),      # one sequence of many rows, one of a token
    (7, 1, [63], [129]), (40, 2, [5], [110]), (12, 4, [1000, 3], [40, 300]),
])
def test_weights_of_long_prompts_and_odd_heads(H, Hkv, lens, adds):
    rng = np.random.default_rng(H + sum(adds))
    say(f"weights of prompts H={H} Hkv={Hkv} lens={lens} adds={adds}")
    weigh(rng, H, Hkv, lens, adds)
    weigh(rng, H, Hkv, lens, adds, n_src=sum(adds) + 5)


def test_weights_of_prompts_with_rows_and_pages_missing():
    """Enough rows that half pages are held: rows outside of what there is, rows that
    attended to nothing, logarithms that are none, absent pages, a longest length,
    blocks nobody began, a key that is a NaN."""
    rng = np.random.default_rng(12)
    say("weights of prompts, parts missing")
    for shift in (-3, 40):
        weigh(rng, 4, 2, [70, 5], [190, 260], shift=shift)
    for value in (-np.inf, np.inf, np.nan):
        odd = lambda n: np.where(rng.random((n, 4)) < 0.2, value, rng.uniform(0, 8, (n, 4))).astype(np.float32)  # noqa: E731,B023
        weigh(rng, 4, 2, [70, 5], [190, 260], lse=odd)
    weigh(rng, 4, 2, [70, 200], [190, 100], max_len=160)
    table = np.array([[0, -1, 2, 7, 6], [3, 99, 4, 5, -1]], np.int32)
    weigh(rng, 4, 2, [30, 70], [280, 200], table=table, pool=make_pool(rng, 8, 2))
    weigh(rng, 4, 2, [70, 5, 300, 0], [400, 0, -20, 300])
    pool = make_pool(rng, 6, 1)
    table = np.array([[1, 2, 4, 3, 5]], np.int32)
    pool[5, 0, 10 * 128:64 * 128] = 127
    pool[5, 0, o8.SCALES + 1] = 255
    pool[1, 0, 7 * 128 + 5] = 127
    got = weigh(rng, 3, 1, [6], [260], table=table, pool=pool)
    assert np.isnan(got[1, 0, 7]) and np.isnan(got).sum() == 1


def test_tables_of_millions_of_pages():
    """More parts of a sequence's place than one launch takes in a dimension: the same
    weights and cuts as by a narrow table."""
    rng = np.random.default_rng(31)
    say("weights of wide tables")
    weigh(rng, 3, 1, [290], [10], width=2 ** 19 + 100)
    pool, w = make_pool(rng, 700, 1), torch.rand((700, 1, 64), device="cuda")
    n = torch.tensor([700 * 64 - 5], dtype=torch.int32, device="cuda")
    wide = torch.full((1, 2 ** 23 + 300), -1, dtype=torch.int32, device="cuda")
    wide[0, :700] = torch.randperm(700, device="cuda")
    got = []
    say("an eviction by a wide table")
    for t in (wide, wide[:, :700].contiguous()):
        p, x = pool.clone(), w.clone()
        got.append((p, x, fc.fc_paged_byte_evict(p, x, t, n, n // 2, first=4, recent=9)))
        torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)
