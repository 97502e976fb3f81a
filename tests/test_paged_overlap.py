"""The paged cache's calls refuse outputs that share bytes with what they read:
their workgroups read while others write.  On the host, before any launch."""
import itertools

import pytest

from test_paged_binding import L  # noqa: F401  (a fixture)

B, R, SLOTS, WIDTH, PAGES, HKV, H, N = 4, 3, 10, 2, 5, 2, 4, 7
PAGE = 8704


def _places(sizes, **change):
    """Addresses a megabyte apart, but for those given."""
    return {**{f: (i + 1) << 20 for i, f in enumerate(sizes)}, **change}


def _meet(sizes, written):
    """Every output over the last bytes, and with its last bytes over the first,
    of everything else."""
    for w, other in itertools.product(written, sizes):
        if w != other:
            base = _places(sizes)[other]
            yield w, other, base + (sizes[other] - 1) // 16 * 16
            yield w, other, base - (sizes[w] - 1) // 16 * 16


PLAN = dict(len=4 * B, add=4 * B, mask=4 * B * R * R, last=4 * B, ends=16, table=4 * B * WIDTH, queue=4 * PAGES,
            len_out=4 * B, cu=4 * B + 4, slot=4 * SLOTS, pos=4 * SLOTS, src=4 * SLOTS, ends_out=16)


@pytest.mark.parametrize("w,other,at", _meet(PLAN, list(PLAN)[5:]))
def test_plan(L, w, other, at):  # noqa: F811
    p = _places(PLAN, **{w: at})
    assert L.fc_paged_plan(p["len"], p["add"], p["mask"], p["last"], B, R, SLOTS, p["table"], WIDTH, p["queue"], PAGES,
                           p["ends"], p["len_out"], p["cu"], p["slot"], p["pos"], p["src"], p["ends_out"], None) == 1


WRITE = dict(k=N * HKV * 256, v=N * HKV * 256, slot=4 * N, pos=4 * N, src=4 * N, pool=PAGES * HKV * PAGE)


@pytest.mark.parametrize("w,other,at", _meet(WRITE, ["pool"]))
def test_write(L, w, other, at):  # noqa: F811
    p = _places(WRITE, **{w: at})
    assert L.fc_paged_write(p["pool"], PAGES, HKV, 128, p["k"], HKV * 128, p["v"], HKV * 128, N, p["slot"], p["pos"],
                            p["src"], N, 1e4, None) == 1


READ = dict(k=N * HKV * 256, v=N * HKV * 256, slot=4 * N, pool=PAGES * HKV * PAGE)


@pytest.mark.parametrize("w,other,at", _meet(READ, ["k", "v"]))
def test_read(L, w, other, at):  # noqa: F811
    p = _places(READ, **{w: at})
    assert L.fc_paged_read(p["pool"], PAGES, HKV, 128, p["slot"], N, p["k"], p["v"], None) == 1


QS = (H + 2 * HKV) * 128        # slices of a fused projection: spans that reach past their last row's neighbours
LONG = 3000
ATTENTION = dict(q=2 * ((B * R - 1) * QS + H * 128), k=2 * ((B * R - 1) * QS + HKV * 128), v=B * R * HKV * 256,
                 pool=PAGES * HKV * PAGE, table=4 * B * 50, plen=4 * B, nodes=4 * B, mask=4 * B * R * R, pos=4 * B * R,
                 out=B * R * H * 256, ws=0)


@pytest.mark.parametrize("w,other", [(w, o) for w in ("out", "ws") for o in ATTENTION if w != o])
@pytest.mark.parametrize("last", [True, False])
def test_attention(L, w, other, last):  # noqa: F811
    need = L.fc_paged_attention_workspace_bytes(B, R, H, HKV, LONG)
    assert 0 < need < 1 << 22
    sizes = dict(ATTENTION, ws=need)
    p = {f: (i + 1) << 22 for i, f in enumerate(sizes)}
    p[w] = p[other] + (sizes[other] - 1) // 16 * 16 if last else p[other] - (sizes[w] - 1) // 16 * 16
    call = lambda p: L.fc_paged_attention(  # noqa: E731
        p["q"], QS, p["k"], QS, p["v"], HKV * 128, p["pool"], PAGES, p["table"], 50, p["plen"], p["nodes"], p["mask"],
        p["pos"], B, R, H, HKV, 128, LONG, 1e4, p["out"], p["ws"], need, None)
    assert call(p) == 1
    p["out"] = p["q"]           # rows at another distance than the queries'
    assert call(p) == 1
