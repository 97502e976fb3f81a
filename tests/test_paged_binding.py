"""The paged cache refuses bad arguments on the host: the library by status,
the binding by exception, before anything reaches a GPU."""
import ctypes
import os

import pytest
import torch

import paper_2502_17139_amd as fc

BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fc.LIB_PATH):
        from paper_2502_17139_amd import build
        build.build()
    return fc.lib()


ONE, TWO, ODD = ctypes.c_void_p(16), ctypes.c_void_p(32), ctypes.c_void_p(24)
INF = float("inf")


def test_pool_bytes(L):
    assert fc.fc_paged_pool_bytes(10, 8) == 10 * 8 * 8704
    assert fc.fc_paged_pool_bytes(2 ** 25 - 1, 1024) == (2 ** 25 - 1) * 1024 * 8704
    for bad in ((0, 1), (1, 0), (2 ** 25, 1), (1, 1025), (-1, 1)):
        assert fc.fc_paged_pool_bytes(*bad) == 0


def _plan(L, B=2, R=0, n_slots=4, max_pages=3, n_pages=5, **p):
    at = dict(len=ONE, add=ONE, mask=None, last=None, table=ONE, queue=ONE, ends=ONE, len_out=TWO, cu=ONE, slot=ONE,
              pos=ONE, src=ONE, ends_out=TWO)
    at.update(p)
    return L.fc_paged_plan(at["len"], at["add"], at["mask"], at["last"], B, R, n_slots, at["table"], max_pages,
                           at["queue"], n_pages, at["ends"], at["len_out"], at["cu"], at["slot"], at["pos"], at["src"],
                           at["ends_out"], None)


@pytest.mark.parametrize("change", [
    dict(B=-1), dict(B=65537), dict(n_slots=-1), dict(n_slots=1 << 30), dict(max_pages=0), dict(max_pages=1 << 25),
    dict(n_pages=0), dict(n_pages=1 << 25), dict(mask=ONE), dict(last=ONE), dict(mask=ONE, last=ONE, R=0),
    dict(mask=ONE, last=ONE, R=257), dict(len=None), dict(add=None), dict(table=None), dict(queue=None),
    dict(ends=None), dict(len_out=None), dict(cu=None), dict(slot=None), dict(pos=None), dict(src=None),
    dict(ends_out=None), dict(len_out=ONE), dict(ends_out=ONE),
], ids=str)
def test_plan_rejects(L, change):
    assert _plan(L, **change) == 1


def _write(L, n_pages=2, Hkv=2, D=128, ks=256, vs=256, n_src=3, n=3, base=1e4, pool=ONE, k=ONE, v=ONE, slot=ONE,
           pos=ONE):
    return L.fc_paged_write(pool, n_pages, Hkv, D, k, ks, v, vs, n_src, slot, pos, None, n, base, None)


@pytest.mark.parametrize("change,code", [
    (dict(n_pages=0), 1), (dict(n_pages=1 << 25), 1), (dict(Hkv=0), 1), (dict(Hkv=1025, ks=1 << 20, vs=1 << 20), 1),
    (dict(D=64), 4), (dict(ks=255), 1), (dict(vs=248), 1), (dict(ks=260), 1), (dict(n=-1), 1), (dict(n_src=-1), 1),
    (dict(base=1.0), 1), (dict(base=-3.0), 1), (dict(base=INF), 1), (dict(base=float("nan")), 1), (dict(pool=None), 1),
    (dict(pool=ODD), 1), (dict(k=None), 1), (dict(v=ODD), 1), (dict(slot=None), 1), (dict(pos=None), 1),
    (dict(n=0), 0), (dict(n_src=0), 0),
], ids=str)
def test_write_rejects(L, change, code):
    assert _write(L, **change) == code


def test_read_rejects(L):
    read = lambda pool=ONE, n_pages=1, Hkv=1, D=128, slot=ONE, n=1, k=ONE, v=ONE: L.fc_paged_read(  # noqa: E731
        pool, n_pages, Hkv, D, slot, n, k, v, None)
    for bad in (dict(pool=None), dict(pool=ODD), dict(n_pages=0), dict(Hkv=0), dict(n=-1), dict(slot=None), dict(k=None),
                dict(v=ODD)):
        assert read(**bad) == 1
    assert read(D=96) == 4 and read(n=0, slot=None, k=None, v=None) == 0


def _attention(L, B=1, R=2, H=4, Hkv=2, D=128, max_len=128, max_pages=2, n_pages=3, qs=512, ks=256, vs=256, base=1e4,
               ws=None, ws_bytes=0, **p):
    at = dict(q=ONE, k=ONE, v=ONE, pool=ONE, table=ONE, plen=ONE, out=ONE)
    at.update(p)
    return L.fc_paged_attention(at["q"], qs, at["k"], ks, at["v"], vs, at["pool"], n_pages, at["table"], max_pages,
                                at["plen"], None, None, None, B, R, H, Hkv, D, max_len, base, at["out"], ws, ws_bytes,
                                None)


@pytest.mark.parametrize("change,code", [
    (dict(B=-1), 1), (dict(B=65537), 1), (dict(R=0), 1), (dict(R=257), 1), (dict(H=3), 1), (dict(H=0), 1),
    (dict(Hkv=0), 1), (dict(D=64), 4), (dict(max_len=-1), 1), (dict(max_len=129), 1), (dict(max_pages=0), 1),
    (dict(n_pages=0), 1), (dict(n_pages=1 << 25), 1), (dict(qs=504), 1), (dict(qs=516), 1), (dict(ks=248), 1),
    (dict(vs=250), 1), (dict(base=1.0), 1), (dict(base=INF), 1), (dict(base=float("nan")), 1), (dict(q=None), 1),
    (dict(k=None), 1), (dict(v=None), 1), (dict(pool=None), 1), (dict(table=None), 1), (dict(plen=None), 1),
    (dict(out=None), 1), (dict(out=ODD), 1), (dict(q=ODD), 1), (dict(pool=ODD), 1), (dict(B=0), 0),
    (dict(B=65536, R=256, H=8192, Hkv=1024, qs=8192 * 128, ks=1024 * 128, vs=1024 * 128), 4),
], ids=str)
def test_attention_rejects(L, change, code):
    assert _attention(L, **change) == code


def test_attention_workspace(L):
    size = fc.fc_paged_attention_workspace_bytes
    assert size(1, 1, 8, 1, 0) == 0 and size(0, 1, 8, 1, 1000) == 0 and size(1, 257, 8, 1, 1000) == 0
    need = size(1, 1, 8, 1, 100_000)
    assert need > 8 * 128 * 4
    call = lambda **kw: _attention(L, R=1, H=8, Hkv=1, qs=1024, max_len=100_000, max_pages=2000, **kw)  # noqa: E731
    assert call() == 2 and call(ws=ONE, ws_bytes=need - 1) == 2 and call(ws=ODD, ws_bytes=need) == 1
    assert size(64, 65, 32, 32, 1 << 20) < 1 << 36


def _inputs(B=2, R=3, H=4, Hkv=2, n_pages=5, width=2):
    z = lambda *s, dt=BF: torch.zeros(s, dtype=dt)  # noqa: E731
    return dict(q=z(B, R, H, 128), k_tree=z(B, R, Hkv, 128), v_tree=z(B, R, Hkv, 128),
                pool=z(n_pages, Hkv, 8704, dt=torch.uint8), table=z(B, width, dt=I32), prefix_len=z(B, dt=I32))


@pytest.mark.parametrize("name,bad,match", [
    ("q", torch.zeros((2, 3, 4, 64), dtype=BF), "q"), ("q", torch.zeros((2, 3, 4, 128)), "q"),
    ("k_tree", torch.zeros((2, 3, 4, 128), dtype=BF), "k_tree"), ("v_tree", torch.zeros((2, 2, 2, 128), dtype=BF), "v_tree"),
    ("pool", torch.zeros((5, 2, 8700), dtype=torch.uint8), "pool"), ("pool", torch.zeros((5, 2, 8704)), "pool"),
    ("table", torch.zeros((3, 2), dtype=I32), "table"), ("table", torch.zeros((2, 2), dtype=torch.int64), "table"),
    ("prefix_len", torch.zeros(2, dtype=torch.int64), "prefix_len"),
    ("q", torch.zeros((2, 3, 128, 4), dtype=BF).transpose(2, 3), "contiguous heads"),
    ("q", torch.zeros((2, 5, 4, 128), dtype=BF)[:, :3], "evenly spaced"),
    ("tree", dict(num_nodes=torch.zeros(2, dtype=I32), mask=torch.zeros((2, 3, 4), dtype=I32),
                  pos_ids=torch.zeros((2, 3), dtype=I32)), "mask"),
    ("out", torch.zeros((2, 3, 4, 128)), "out"), ("workspace", torch.zeros(9), "workspace"),
], ids=lambda x: x if isinstance(x, str) else "")
def test_attention_binding_refuses(name, bad, match):
    with pytest.raises(ValueError, match=match):
        fc.fc_paged_attention(**{**_inputs(), name: bad})


def test_bindings_refuse_host_tensors():
    s = _inputs()
    with pytest.raises(ValueError, match="device tensor"):
        fc.fc_paged_attention(**s)
    with pytest.raises(ValueError, match="device tensor"):
        fc.fc_paged_read(s["pool"], torch.zeros(3, dtype=I32))
    st = fc.paged_state(2, 3, 9, "cpu")
    assert st["table"].eq(-1).all() and st["ends"].tolist() == [0, 9]
    with pytest.raises(ValueError, match="device tensor"):
        fc.fc_paged_plan(st["len"], st["len"], st["table"], st["queue"], st["ends"], 3)


def test_plan_and_write_bindings_refuse():
    st = fc.paged_state(2, 3, 9, "cpu")
    args = (st["len"], st["len"].clone(), st["table"], st["queue"], st["ends"], 3)
    with pytest.raises(ValueError, match="go together"):
        fc.fc_paged_plan(*args, tree=dict(mask=torch.zeros((2, 3, 3), dtype=I32)))
    with pytest.raises(ValueError, match="mask"):
        fc.fc_paged_plan(*args, tree=dict(mask=torch.zeros((2, 3, 4), dtype=I32)), last_node=st["len"])
    with pytest.raises(ValueError, match="add"):
        fc.fc_paged_plan(args[0], torch.zeros(3, dtype=I32), *args[2:])
    with pytest.raises(ValueError, match="ends"):
        fc.fc_paged_plan(*args[:4], torch.zeros(2, dtype=I32), 3)
    out = dict(len=st["len"], cu=torch.zeros(3, dtype=I32), slot=torch.zeros(2, dtype=I32))
    with pytest.raises(ValueError, match="slot"):
        fc.fc_paged_plan(*args, out=out)
    s = _inputs()
    k, slot = torch.zeros((6, 2, 128), dtype=BF), torch.zeros(4, dtype=I32)
    with pytest.raises(ValueError, match="pos"):
        fc.fc_paged_write(s["pool"], k, k, slot)
    with pytest.raises(ValueError, match="src"):
        fc.fc_paged_write(s["pool"], k, k, slot, slot, src=slot[:3])
    with pytest.raises(ValueError, match="differ"):
        fc.fc_paged_write(s["pool"], k, k[:5], slot, slot)
    with pytest.raises(ValueError, match="k must"):
        fc.fc_paged_write(s["pool"], torch.zeros((6, 3, 128), dtype=BF), k, slot, slot)
    with pytest.raises(ValueError, match="v must"):
        fc.fc_paged_read(s["pool"], slot, out=(torch.zeros((4, 2, 128), dtype=BF), torch.zeros((3, 2, 128), dtype=BF)))


def test_bindings_refuse_numbers_out_of_range():
    """Numbers that the C call would take 32 bits of."""
    s = _inputs()
    for max_len in (2 ** 31, 2 ** 32 + 64, -2 ** 31):
        with pytest.raises(ValueError, match="max_len"):
            fc.fc_paged_attention(**s, max_len=max_len)
    st = fc.paged_state(2, 3, 9, "cpu")
    for n_slots in (-1, 2 ** 30, 2 ** 32):
        with pytest.raises(ValueError, match="n_slots"):
            fc.fc_paged_plan(st["len"], st["len"], st["table"], st["queue"], st["ends"], n_slots)


def test_bindings_refuse_sizes_out_of_range():
    """Tensors of more entries than 32 bits number (2^32 + 5 would pass as 5), and
    pools without a key head."""
    s, st, one = _inputs(), fc.paged_state(2, 3, 9, "cpu"), torch.zeros(1, dtype=I32)
    long = one.expand(2 ** 32 + 5)
    k = torch.zeros((6, 2, 128), dtype=BF)
    wide, many = one.expand(2, 2 ** 32 + 5), k[:1].expand(2 ** 32 + 6, 2, 128)
    plan = (st["len"], st["len"], st["table"], st["queue"], st["ends"])
    for call in (lambda: fc.fc_paged_write(s["pool"], k, k, long, long),
                 lambda: fc.fc_paged_write(s["pool"], many, many, one, one),
                 lambda: fc.fc_paged_read(s["pool"], long),
                 lambda: fc.fc_paged_read(s["pool"][:1].expand(2 ** 32 + 1, 2, 8704), one),
                 lambda: fc.fc_paged_attention(**{**s, "table": wide}, max_len=64),
                 lambda: fc.fc_paged_plan(*plan[:2], wide, *plan[3:], 3),
                 lambda: fc.fc_paged_plan(*plan[:3], long, plan[4], 3)):
        with pytest.raises(ValueError, match="32-bit"):
            call()
    none = torch.zeros((5, 0, 8704), dtype=torch.uint8)
    with pytest.raises((ValueError, fc.FcError)):
        fc.fc_paged_write(none, k[:, :0], k[:, :0], one, one)


def test_short_prefixes_are_cut_for_one_round_of_workgroups(L):
    """512 workgroups run at once.  Prefixes of fewer than 64 pages are cut into no
    more parts than that leaves room for, so a nearly full card pays for no join:
    63 sequences of 8 key heads are as whole as 64."""
    size = fc.fc_paged_attention_workspace_bytes
    parts = lambda B, R, H, Hkv, n: size(B, R, H, Hkv, n) // (520 * B * R * H) or 1  # noqa: E731
    for n in (700, 2048, 4032):
        for B in range(1, 70):
            assert parts(B, 1, 32, 8, n) == 1 or B * 8 * parts(B, 1, 32, 8, n) <= 512, (B, n)
            assert parts(B, 65, 32, 32, n) == 1 or B * 32 * parts(B, 65, 32, 32, n) <= 512, (B, n)
    assert size(63, 1, 32, 8, 2048) == size(64, 1, 32, 8, 2048) == size(15, 65, 32, 32, 2048) == 0
    assert parts(1, 1, 32, 8, 3000) == 3 and parts(16, 1, 32, 8, 4032) == 4
    assert parts(63, 1, 32, 8, 8192) == 2 and parts(64, 1, 32, 8, 8192) == 1
