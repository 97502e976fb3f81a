"""The paged cache's calls at the ends of what their documentation allows."""
import numpy as np
import pytest
import torch

import oracle
from gpu_pipeline import dev, host, say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_17139_amd as fc  # noqa: E402
from test_paged import _plan, bf16, f64, make_pool, on_gpu, trees  # noqa: E402
from test_paged_scores import check  # noqa: E402


@pytest.mark.parametrize("R,H", [(1, 4), (5, 2), (20, 1), (40, 1), (65, 2), (130, 1)])
def test_positions_past_32_bits(R, H):
    """prefix_len + pos_ids is a sum of two 32-bit numbers: rows just below 2^31,
    past it, and before 0."""
    rng = np.random.default_rng(R)
    pool, table = make_pool(rng, 3, 1), np.array([[2, 0, 1]] * 2, np.int32)
    t = trees(rng, 2, R)
    t["pos_ids"] = (2 ** 31 - 1 - rng.integers(0, 300, (2, R))).astype(np.int32)
    t["pos_ids"][1, ::3] = -2 ** 31 + rng.integers(0, 300, len(t["pos_ids"][1, ::3]))
    row = lambda h, s=1.0: bf16(rng, 2, R, h, 128, scale=s)  # noqa: E731
    say(f"positions past 32 bits R={R}")
    check(row(H, 3.0), row(1), row(1), pool, table, [150, 60], t)


def test_more_rows_than_one_launch_takes():
    """Writes and reads of more tokens than a launch's workgroups hold, rows given
    in order and by number, are what shorter calls make of them."""
    n, piece = 2 ** 24 + 70, 2 ** 20 + 33
    pages = -(-n // 64)
    torch.manual_seed(1)
    x = torch.randn((n, 1, 128), dtype=torch.bfloat16, device="cuda")
    slot = torch.arange(n, dtype=torch.int32, device="cuda")
    pos = slot.flip(0).contiguous()
    pools = [torch.zeros((pages, 1, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda") for _ in "ab"]
    say("writes and reads of more than a launch")
    fc.fc_paged_write(pools[0], x, x, slot, pos)
    for i in range(0, n, piece):
        fc.fc_paged_write(pools[1], x[i:i + piece], x[i:i + piece], slot[i:i + piece], pos[i:i + piece])
    assert torch.equal(pools[0], pools[1]) and pools[0][-1].any()
    few = 1000                                    # rows that exist: the others are skipped
    pools[1][few // 64:].fill_(0)
    fc.fc_paged_write(pools[1], x[:few], x[:few], slot, pos)
    assert torch.equal(pools[1][:few // 64], pools[0][:few // 64]) and not pools[1][few // 64 + 1:].any()
    del pools[1], x
    got = fc.fc_paged_read(pools[0], slot)
    for i in range(0, n, piece):
        want = fc.fc_paged_read(pools[0], slot[i:i + piece])
        assert torch.equal(got[0][i:i + piece], want[0]) and torch.equal(got[1][i:i + piece], want[1])


def test_more_workgroups_than_a_dimension_takes():
    """A slot map of 2^25 workgroups, all but a few entries empty."""
    rng = np.random.default_rng(1)
    n, Hkv = 2 ** 25 + 70, 32                     # one or two tokens of a workgroup
    slot = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    src, pos = torch.full_like(slot, -1), torch.zeros_like(slot)
    at = torch.tensor([0, 5, 2 ** 20, 2 ** 21 - 1, 2 ** 21, 2 ** 24 + 1, n - 1], device="cuda")
    few = torch.arange(len(at), dtype=torch.int32, device="cuda")
    slot[at], src[at], pos[at] = few * 9, few.flip(0), few * 1000
    k, v = bf16(rng, len(at), Hkv, 128).cuda(), bf16(rng, len(at), Hkv, 128).cuda()
    pools = [torch.zeros((1, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda") for _ in "ab"]
    say("more workgroups than a dimension takes")
    fc.fc_paged_write(pools[0], k, v, slot, pos, src=src)
    fc.fc_paged_write(pools[1], k, v, slot[at], pos[at], src=src[at])
    assert torch.equal(pools[0], pools[1]) and pools[0].any()


@pytest.mark.parametrize("B,R,Hkv,piece", [(65536, 1, 256, 30000), (6000, 97, 8, 2500)])
def test_more_trees_than_one_launch_takes(B, R, Hkv, piece):
    """2^24 workgroups of single tokens, and joins of more rows than a launch
    takes: the bits of calls with fewer trees."""
    rng = np.random.default_rng(2)
    pool = make_pool(rng, 40, Hkv)
    torch.manual_seed(2)
    x = torch.randn((B, R, Hkv, 128), dtype=torch.bfloat16, device="cuda")
    table = torch.randint(0, 40, (B, 2), dtype=torch.int32, device="cuda")
    plen = torch.randint(0, 129, (B,), dtype=torch.int32, device="cuda")
    say(f"attention of {B} trees of {R} rows")
    got = fc.fc_paged_attention(x, x, x, pool, table, plen)
    for i in range(0, B, piece):
        want = fc.fc_paged_attention(*[x[i:i + piece]] * 3, pool, table[i:i + piece], plen[i:i + piece])
        assert torch.equal(got[i:i + piece], want), i
    assert (fc.fc_paged_attention_workspace_bytes(B, R, Hkv, Hkv, 128) > 0) == (R > 96)


@pytest.mark.parametrize("R,H,Hkv,n", [(1, 8, 2, 100), (1, 8, 2, 3000), (65, 4, 4, 100), (70, 2, 1, 2000), (130, 2, 2, 90)])
def test_results_in_place_of_queries(R, H, Hkv, n):
    """out may be q, and lie beside what is read; anything between is refused."""
    rng = np.random.default_rng(R)
    B, width = 3, -(-n // 64)
    pool, table = make_pool(rng, 6, Hkv), dev(rng.integers(0, 6, (B, width)).astype(np.int32))
    lens = dev(np.array([n, n // 2, 0], np.int32))
    block = torch.empty((3 * B, R, H, 128), dtype=torch.bfloat16, device="cuda")
    q, kt, vt = block[B:2 * B], bf16(rng, B, R, Hkv, 128).cuda(), bf16(rng, B, R, Hkv, 128).cuda()
    q.copy_(bf16(rng, B, R, H, 128))
    t = on_gpu(trees(rng, B, R))
    say(f"in place R={R} n={n}")
    want = fc.fc_paged_attention(q, kt, vt, pool, table, lens, tree=t)
    for out in (block[:B], block[2 * B:], q):
        assert torch.equal(want, fc.fc_paged_attention(q, kt, vt, pool, table, lens, tree=t, out=out))
    for at in (B - 1, B + 1):
        with pytest.raises(fc.FcError):
            fc.fc_paged_attention(q, kt, vt, pool, table, lens, tree=t, out=block[at:at + B])


@pytest.mark.parametrize("Hkv,n_pages", [(1, 1), (2, 3), (8, 2), (33, 1)])
def test_writes_at_the_ends_of_the_pool(Hkv, n_pages):
    """Each slot once: the pool's first and last, and those just outside of it,
    whose rows go nowhere."""
    rng = np.random.default_rng(Hkv)
    last = 64 * n_pages - 1
    slot = np.concatenate([[0, last, last + 1, -1, 2 ** 31 - 1, -2 ** 31], 1 + rng.permutation(last - 1)[:40]])
    slot = rng.permutation(slot).astype(np.int32)
    n = len(slot)
    assert len(set(slot.tolist())) == n
    k, v = bf16(rng, n, Hkv, 128), bf16(rng, n, Hkv, 128)
    pos = rng.integers(0, 5000, n).astype(np.int32)
    before = rng.integers(0, 256, (n_pages, Hkv, fc.FC_PAGE_HEAD_BYTES)).astype(np.uint8)
    guarded = dev(np.concatenate([before, before]))      # what lies behind the pool stays as it is
    say(f"writes at the ends of {n_pages} pages of {Hkv} heads")
    fc.fc_paged_write(guarded[:n_pages], k.cuda(), v.cuda(), dev(slot), dev(pos))
    assert np.array_equal(host(guarded[:n_pages]), oracle.paged_write(before, f64(k), f64(v), slot, pos))
    assert np.array_equal(host(guarded[n_pages:]), before)


@pytest.mark.parametrize("B,R", [(300, 65), (1500, 33), (250, 256)])
def test_accepted_paths_across_workgroups_of_the_plan(B, R):
    """A workgroup plans 4,096 slots: paths that begin before one and end in it."""
    rng = np.random.default_rng(B)
    mask, depth = np.zeros((B, R, R), np.int32), np.zeros((B, R), np.int64)
    for b in range(B):
        for i in range(R):
            if i:
                p = i - 1 if rng.random() < 0.9 else int(rng.integers(0, i))
                mask[b, i], depth[b, i] = mask[b, p], depth[b, p] + 1
            mask[b, i, i] = 1
    last = rng.integers(R // 2, R, B).astype(np.int32)
    add = (depth[np.arange(B), last] + 1).astype(np.int32)
    add[::7] += 2                                        # more tokens than rows
    start = np.cumsum(add) - add
    crossing = start // 4096 != (start + add - 1) // 4096
    assert crossing.any()
    length = rng.integers(0, 100, B).astype(np.int32)
    held = -(-length // 64)
    perm = rng.permutation(int(held.sum()) + 4 * B).astype(np.int32)
    table, at = np.full((B, 6), -1, np.int32), 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    queue = np.concatenate([perm[at:], np.full(at, -1, np.int32)])
    say(f"accepted paths across workgroups B={B} R={R} tokens={add.sum()}")
    r = _plan(length, add, table, queue, [0, 4 * B], int(add.sum()) + 9, mask, last)
    for b in np.flatnonzero(crossing):
        assert (r["slot"][start[b]:start[b] + add[b]] >= 0).all()


@pytest.mark.parametrize("R", [1, 20, 65])
def test_large_values_behind_low_first_scores(R):
    """Weights go by what a row saw first: here all but the first pages have scores
    17.5 bits above those, so that half a million weights of 2^17.5 meet values just
    below the largest that the sums are good for."""
    B, Hkv, width = 64, 8, 8192
    k, v = torch.zeros((128, Hkv, 128)), torch.zeros((128, Hkv, 128))
    k[64:], v[64:] = 1.0, 1.5 * 2.0 ** 75
    pool = torch.zeros((2, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_write(pool, k.bfloat16().cuda(), v.bfloat16().cuda(), dev(np.arange(128, dtype=np.int32)), rope_base=0.0)
    table = np.ones((B, width), np.int32)
    table[:, :4] = 0
    q = torch.full((B, R, Hkv, 128), 1.0703125, dtype=torch.bfloat16, device="cuda")    # 17.47 / (128 log2(e) / sqrt(128))
    none = torch.zeros_like(q)
    t = dict(num_nodes=np.full(B, R, np.int32), mask=np.zeros((B, R, R), np.int32), pos_ids=np.zeros((B, R), np.int32))
    say(f"large values R={R}")
    got = f64(fc.fc_paged_attention(q, none, none, pool, dev(table), dev(np.full(B, 64 * width, np.int32)),
                                    tree=on_gpu(t), rope_base=0.0))
    # the first pages weigh 2^-28; equal weights cancel but for their sums' rounding, and 1.5 is a bf16
    assert np.abs(got / (1.5 * 2.0 ** 75) - 1).max() <= 2.0 ** -8


@pytest.mark.parametrize("R", [1, 9, 40])
@pytest.mark.parametrize("small,large", [(-105, 100), (-116, 110), (100, -110)])
def test_sizes_far_apart(R, small, large):
    """Queries below the least scale of their parts against keys near the largest,
    and the other way round: scores of the usual size."""
    rng = np.random.default_rng(R)
    k, v = bf16(rng, 128, 2, 128, scale=2.0 ** large), bf16(rng, 128, 2, 128)
    pool = torch.zeros((2, 2, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    fc.fc_paged_write(pool, k.cuda(), v.cuda(), dev(np.arange(128, dtype=np.int32)), rope_base=0.0)
    say(f"sizes far apart R={R} {small} {large}")
    check(bf16(rng, 1, R, 4, 128, scale=2.0 ** (small + 3)), bf16(rng, 1, R, 2, 128, scale=2.0 ** large),
          bf16(rng, 1, R, 2, 128), pool, np.array([[1, 0]], np.int32), [100], norm=False)


def _some_calls(rng, n):
    """Attention inputs of n calls with prefixes in parts, and what each gives alone."""
    pool = make_pool(rng, 12, 2)
    calls = []
    for i in range(n):
        R = (1, 9, 65)[i % 3]
        row = lambda h: bf16(rng, 2, R, h, 128).cuda()  # noqa: E731
        calls.append(dict(q=row(8), k_tree=row(2), v_tree=row(2), pool=pool,
                          table=dev(rng.integers(0, 12, (2, 30)).astype(np.int32)),
                          prefix_len=dev(np.array([1900 - i, 700], np.int32)), tree=on_gpu(trees(rng, 2, R))))
    want = [fc.fc_paged_attention(**c) for c in calls]
    torch.cuda.synchronize()
    return calls, want


def test_calls_at_once_on_several_streams():
    """Calls side by side on their own streams, each with its own scratch memory."""
    calls, want = _some_calls(np.random.default_rng(30), 6)
    streams = [torch.cuda.Stream() for _ in calls]
    say("calls on several streams")
    for _ in range(3):
        got = [[fc.fc_paged_attention(**c, stream=s) for _ in range(4)] for c, s in zip(calls, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(w, x) for w, g in zip(want, got) for x in g)


def test_graphs_that_share_a_workspace():
    """Two captured graphs with one workspace, replayed in turn with eager work and
    other bytes in the workspace between."""
    calls, want = _some_calls(np.random.default_rng(31), 3)
    need = max(fc.fc_paged_attention_workspace_bytes(2, c["q"].shape[1], 8, 2, 30 * 64) for c in calls)
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")
    say("graphs that share a workspace")
    graphs, outs = [], []
    for c in calls:
        out = torch.empty_like(c["q"])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fc.fc_paged_attention(**c, out=out, workspace=ws)
        graphs.append(g)
        outs.append(out)
    for turn in range(4):
        for i in ((0, 1, 2), (2, 0, 1), (1, 1, 0), (0, 2, 2))[turn]:
            outs[i].fill_(7.0)
            graphs[i].replay()
            assert torch.equal(outs[i], want[i]), (turn, i)
            ws.fill_(255)
            assert torch.equal(fc.fc_paged_attention(**calls[i]), want[i])
