"""The 8-bit paged cache and the norm with rotation refuse bad arguments on the host: the
library by status, the binding by exception, before anything reaches a GPU."""
import ctypes
import itertools

import pytest
import torch

import paper_2502_17139_amd as fc
from test_paged_binding import L  # noqa: F401  (a fixture)

BF, I32, F32 = torch.bfloat16, torch.int32, torch.float32
PAGE = 16512
ONE, TWO, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p(2 << 20), ctypes.c_void_p((1 << 20) + 8)
INF, NAN = float("inf"), float("nan")


def test_pool_bytes(L):  # noqa: F811
    assert fc.fc_paged_byte_pool_bytes(10, 8) == 10 * 8 * PAGE
    assert fc.fc_paged_byte_pool_bytes(2 ** 25 - 1, 1024) == (2 ** 25 - 1) * 1024 * PAGE
    for bad in ((0, 1), (1, 0), (2 ** 25, 1), (1, 1025), (-1, 1)):
        assert fc.fc_paged_byte_pool_bytes(*bad) == 0


# ------------------------------------------------------------------- norm --

def _norm(L, n=3, H=4, Hkv=2, D=128, qs=512, ks=256, qos=512, kos=256, eps=1e-6, base=1e4, **p):  # noqa: F811
    at = {f: (i + 1) << 20 for i, f in enumerate(("q", "k", "qw", "kw", "pos", "qo", "ko"))}
    at.update(p)
    return L.fc_norm_rotate(at["q"], qs, at["k"], ks, at["qw"], at["kw"], at["pos"], n, H, Hkv, D, eps, base, at["qo"], qos,
                            at["ko"], kos, None)


@pytest.mark.parametrize("change,code", [
    (dict(n=-1), 1), (dict(H=-1), 1), (dict(H=8193), 1), (dict(Hkv=-1), 1), (dict(Hkv=8193), 1), (dict(D=64), 4),
    (dict(qs=511), 1), (dict(qs=516), 1), (dict(ks=248), 1), (dict(qos=504), 1), (dict(kos=260), 1), (dict(eps=-1e-9), 1),
    (dict(eps=NAN), 1), (dict(eps=INF), 1), (dict(base=1.0), 1), (dict(base=-2.0), 1), (dict(base=INF), 1),
    (dict(base=NAN), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(qo=None), 1), (dict(ko=None), 1), (dict(pos=None), 1),
    (dict(q=(1 << 20) + 8), 1), (dict(k=8), 1), (dict(qw=8), 1), (dict(kw=24), 1), (dict(qo=8), 1), (dict(ko=8), 1),
    (dict(n=0, q=None, k=None), 0), (dict(H=0, Hkv=0, q=None, k=None), 0),
], ids=str)
def test_norm_rejects(L, change, code):  # noqa: F811
    assert _norm(L, **change) == code


NORM = dict(q=3 * 1024, k=3 * 512, qw=256, kw=256, pos=12, qo=3 * 1024, ko=3 * 512)


def _meet(sizes, written):
    """Every output over the last bytes, and with its last bytes over the first, of
    everything else."""
    for w, other in itertools.product(written, sizes):
        if w != other:
            base = (list(sizes).index(other) + 1) << 20
            yield w, base + (sizes[other] - 1) // 16 * 16
            yield w, base - (sizes[w] - 1) // 16 * 16


@pytest.mark.parametrize("w,at", _meet(NORM, ["qo", "ko"]))
def test_norm_rejects_shared_bytes(L, w, at):  # noqa: F811
    assert _norm(L, **{w: at}) == 1


def test_norm_rejects_what_is_not_quite_in_place(L):  # noqa: F811
    q = 1 << 20
    assert _norm(L, qo=q, qos=520) == 1                      # another distance
    assert _norm(L, qs=1024, qos=1024, qo=q + 512) == 1      # a later head's place
    assert _norm(L, qs=768, qos=768, ks=768, k=q + 1024, qo=q + 256, H=4) == 1   # reaches into the keys beside it
    assert _norm(L, H=2, qs=256, qos=256, qo=2 << 20) == 1   # the keys' place


# ----------------------------------------------------------- write and read --

def _write(L, n_pages=2, Hkv=2, D=128, ks=256, vs=256, n_src=3, n=3, **p):  # noqa: F811
    at = dict(pool=1 << 20, k=2 << 20, v=3 << 20, slot=4 << 20, src=5 << 20)
    at.update(p)
    return L.fc_paged_byte_write(at["pool"], n_pages, Hkv, D, at["k"], ks, at["v"], vs, n_src, at["slot"], at["src"], n, None)


@pytest.mark.parametrize("change,code", [
    (dict(n_pages=0), 1), (dict(n_pages=1 << 25), 1), (dict(Hkv=0), 1), (dict(Hkv=1025, ks=1 << 20, vs=1 << 20), 1),
    (dict(D=64), 4), (dict(ks=255), 1), (dict(vs=248), 1), (dict(ks=260), 1), (dict(n=-1), 1), (dict(n_src=-1), 1),
    (dict(pool=None), 1), (dict(pool=8), 1), (dict(k=None), 1), (dict(v=8), 1), (dict(slot=None), 1), (dict(n=0), 0),
    (dict(n_src=0), 0),
], ids=str)
def test_write_rejects(L, change, code):  # noqa: F811
    assert _write(L, **change) == code


WRITE = dict(pool=4 * PAGE, k=3 * 512, v=3 * 512, slot=12, src=12)


@pytest.mark.parametrize("w,at", _meet(WRITE, ["pool"]))
def test_write_rejects_shared_bytes(L, w, at):  # noqa: F811
    assert _write(L, **{w: at}) == 1


def _read(L, n_pages=2, Hkv=2, D=128, n=3, **p):  # noqa: F811
    at = dict(pool=1 << 20, slot=2 << 20, k=3 << 20, v=4 << 20)
    at.update(p)
    return L.fc_paged_byte_read(at["pool"], n_pages, Hkv, D, at["slot"], n, at["k"], at["v"], None)


READ = dict(pool=4 * PAGE, slot=12, k=3 * 512, v=3 * 512)


def test_read_rejects(L):  # noqa: F811
    for bad in (dict(pool=None), dict(pool=8), dict(n_pages=0), dict(Hkv=0), dict(n=-1), dict(slot=None), dict(k=None),
                dict(v=8), dict(Hkv=1025)):
        assert _read(L, **bad) == 1
    assert _read(L, D=96) == 4 and _read(L, n=0, slot=None, k=None, v=None) == 0
    for w, at in _meet(READ, ["k", "v"]):
        assert _read(L, **{w: at}) == 1


# -------------------------------------------------------------- attention --

B, R, H, HKV, LONG = 4, 3, 4, 2, 3000
QS = (H + 2 * HKV) * 128


def _attention(L, B=B, R=R, H=H, Hkv=HKV, D=128, max_len=LONG, max_pages=50, n_pages=5, qs=QS, ks=QS, vs=256, ws_bytes=None,  # noqa: F811
               **p):
    at = {f: (i + 1) << 22 for i, f in enumerate(ATTENTION)}
    at.update(p)
    need = L.fc_paged_byte_attention_workspace_bytes(B, R, H, Hkv, max_len) if ws_bytes is None else ws_bytes
    return L.fc_paged_byte_attention(at["q"], qs, at["k"], ks, at["v"], vs, at["pool"], n_pages, at["table"], max_pages,
                                 at["plen"], at["nodes"], at["mask"], B, R, H, Hkv, D, max_len, at["out"], at["lse"],
                                 at["ws"], need, None)


ATTENTION = dict(q=2 * ((B * R - 1) * QS + H * 128), k=2 * ((B * R - 1) * QS + HKV * 128), v=B * R * HKV * 256,
                 pool=5 * HKV * PAGE, table=4 * B * 50, plen=4 * B, nodes=4 * B, mask=4 * B * R * R, out=B * R * H * 256,
                 lse=4 * B * R * H, ws=0)


@pytest.mark.parametrize("change,code", [
    (dict(B=-1), 1), (dict(B=65537), 1), (dict(R=0), 1), (dict(R=257), 1), (dict(H=0), 1), (dict(H=3), 1), (dict(Hkv=0), 1),
    (dict(H=8194, Hkv=2, qs=1 << 21), 1), (dict(max_len=-1), 1), (dict(max_len=50 * 64 + 1), 1), (dict(max_pages=0), 1),
    (dict(n_pages=0), 1), (dict(n_pages=1 << 25), 1), (dict(D=64), 4), (dict(qs=504), 1), (dict(qs=QS + 4), 1),
    (dict(ks=248), 1), (dict(vs=128), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(pool=None), 1),
    (dict(table=None), 1), (dict(plen=None), 1), (dict(out=None), 1), (dict(q=8), 1), (dict(k=8), 1), (dict(v=8), 1),
    (dict(pool=8), 1), (dict(out=8), 1), (dict(lse=2), 1), (dict(ws=None), 2), (dict(ws_bytes=100), 2), (dict(ws=8), 1),
    (dict(B=0, q=None), 0),
], ids=str)
def test_attention_rejects(L, change, code):  # noqa: F811
    assert _attention(L, **change) == code


@pytest.mark.parametrize("w,other", [(w, o) for w in ("out", "lse", "ws") for o in ATTENTION if w != o])
@pytest.mark.parametrize("last", [True, False])
def test_attention_rejects_shared_bytes(L, w, other, last):  # noqa: F811
    need = L.fc_paged_byte_attention_workspace_bytes(B, R, H, HKV, LONG)
    assert 0 < need < 1 << 22
    sizes = dict(ATTENTION, ws=need)
    base = (list(sizes).index(other) + 1) << 22
    at = base + (sizes[other] - 1) // 16 * 16 if last else base - (sizes[w] - 1) // 16 * 16
    assert _attention(L, **{w: at}) == 1
    assert _attention(L, out=1 << 22) == 1        # the queries' place, at another distance


def test_attention_workspace(L):  # noqa: F811
    size = fc.fc_paged_byte_attention_workspace_bytes
    assert size(1, 1, 8, 1, 0) == 0 and size(0, 1, 8, 1, 1000) == 0 and size(1, 257, 8, 1, 1000) == 0
    assert size(1, 1, 8, 1, 100_000) > 8 * 128 * 4
    assert size(64, 65, 32, 32, 1 << 20) < 1 << 36


# ------------------------------------------------------- weights and evict --

WEIGHTS = dict(w=4 * 5 * HKV * 64, q=2 * (6 * QS + H * 128), lse=4 * 7 * H, pool=5 * HKV * PAGE, table=4 * B * 3, len=4 * B,
               new=4 * B, cu=4 * B + 4, src=4 * 9)


def _weights(L, n_rows=7, n_pages=5, max_pages=3, n=9, B=B, H=H, Hkv=HKV, D=128, max_len=192, qs=QS, **p):  # noqa: F811
    at = {f: (i + 1) << 20 for i, f in enumerate(WEIGHTS)}
    at.update(p)
    return L.fc_paged_byte_weights(at["w"], at["q"], qs, at["lse"], n_rows, at["pool"], n_pages, at["table"], max_pages,
                               at["len"], at["new"], at["cu"], at["src"], n, B, H, Hkv, D, max_len, None)


@pytest.mark.parametrize("change,code", [
    (dict(B=-1), 1), (dict(B=65537), 1), (dict(n_rows=-1), 1), (dict(n=-1), 1), (dict(H=3), 1), (dict(H=1), 1),
    (dict(H=8194, qs=1 << 21), 1), (dict(Hkv=0), 1), (dict(Hkv=1025, H=1025, qs=1 << 20), 1), (dict(n_pages=0), 1),
    (dict(max_pages=0), 1), (dict(max_len=193), 1), (dict(max_len=-1), 1), (dict(D=32), 4), (dict(qs=504), 1),
    (dict(qs=QS + 2), 1), (dict(w=None), 1), (dict(q=None), 1), (dict(lse=None), 1), (dict(pool=None), 1),
    (dict(table=None), 1), (dict(len=None), 1), (dict(new=None), 1), (dict(cu=None), 1), (dict(q=8), 1), (dict(pool=8), 1),
    (dict(w=2), 1), (dict(lse=2), 1), (dict(B=0), 0), (dict(n_rows=0), 0), (dict(n=0), 0), (dict(max_len=0), 0),
], ids=str)
def test_weights_rejects(L, change, code):  # noqa: F811
    assert _weights(L, **change) == code


@pytest.mark.parametrize("w,at", _meet(WEIGHTS, ["w"]))
def test_weights_rejects_shared_bytes(L, w, at):  # noqa: F811
    assert _weights(L, **{w: at}) == 1


EVICT = dict(pool=5 * HKV * PAGE, w=4 * 5 * HKV * 64, table=4 * B * 3, len=4 * B, budget=4 * B, add=4 * B, ws=0)


def _evict(L, n_pages=5, Hkv=HKV, D=128, max_pages=3, B=B, max_len=192, first=1, recent=2, ws_bytes=None, **p):  # noqa: F811
    at = {f: (i + 1) << 20 for i, f in enumerate(EVICT)}
    at.update(p)
    need = L.fc_paged_byte_evict_workspace_bytes(B, Hkv, max_len) if ws_bytes is None else ws_bytes
    return L.fc_paged_byte_evict(at["pool"], at["w"], n_pages, Hkv, D, at["table"], max_pages, at["len"], at["budget"], B,
                             max_len, first, recent, at["add"], at["ws"], need, None)


@pytest.mark.parametrize("change,code", [
    (dict(B=-1), 1), (dict(B=65537), 1), (dict(n_pages=0), 1), (dict(Hkv=0), 1), (dict(Hkv=1025), 1), (dict(max_pages=0), 1),
    (dict(max_len=193), 1), (dict(max_len=-1), 1), (dict(first=-1), 1), (dict(recent=-1), 1), (dict(D=256), 4),
    (dict(pool=None), 1), (dict(w=None), 1), (dict(table=None), 1), (dict(len=None), 1), (dict(budget=None), 1),
    (dict(add=None), 1), (dict(pool=8), 1), (dict(w=2), 1), (dict(ws=None), 2), (dict(ws_bytes=200), 2), (dict(ws=8), 1),
    (dict(B=0), 0),
], ids=str)
def test_evict_rejects(L, change, code):  # noqa: F811
    assert _evict(L, **change) == code


def test_evict_rejects_shared_bytes(L):  # noqa: F811
    need = L.fc_paged_byte_evict_workspace_bytes(B, HKV, 192)
    assert 0 < need < 1 << 20
    for w, at in _meet(dict(EVICT, ws=need), ["pool", "w", "add", "ws"]):
        assert _evict(L, **{w: at}) == 1


# -------------------------------------------------------------- the binding --

z = lambda *s, dt=BF: torch.zeros(s, dtype=dt)  # noqa: E731


def _inputs():
    return dict(q=z(2, 3, 4, 128), k_tree=z(2, 3, 2, 128), v_tree=z(2, 3, 2, 128), pool=z(5, 2, PAGE, dt=torch.uint8),
                table=z(2, 2, dt=I32), prefix_len=z(2, dt=I32))


@pytest.mark.parametrize("name,bad,match", [
    ("q", z(2, 3, 4, 64), "q"), ("q", torch.zeros((2, 3, 4, 128)), "q"), ("k_tree", z(2, 3, 4, 128), "k_tree"),
    ("v_tree", z(2, 2, 2, 128), "v_tree"), ("pool", z(5, 2, 8704, dt=torch.uint8), "pool"), ("pool", z(5, 2, PAGE), "pool"),
    ("table", z(3, 2, dt=I32), "table"), ("prefix_len", z(2, dt=torch.int64), "prefix_len"),
    ("q", z(2, 3, 128, 4).transpose(2, 3), "contiguous heads"), ("q", z(2, 5, 4, 128)[:, :3], "evenly spaced"),
    ("tree", dict(num_nodes=z(2, dt=I32), mask=z(2, 3, 4, dt=I32)), "mask"), ("out", torch.zeros((2, 3, 4, 128)), "out"),
    ("lse", z(2, 3, 4), "lse"), ("lse", torch.zeros((2, 3, 2)), "lse"), ("workspace", torch.zeros(9), "workspace"),
], ids=lambda x: x if isinstance(x, str) else "")
def test_attention_binding_refuses(name, bad, match):
    with pytest.raises(ValueError, match=match):
        fc.fc_paged_byte_attention(**{**_inputs(), name: bad})


def _weights_args(**change):
    a = dict(weights=z(5, 2, 64, dt=F32), q=z(2, 3, 4, 128), lse=z(2, 3, 4, dt=F32), pool=z(5, 2, PAGE, dt=torch.uint8),
             table=z(2, 2, dt=I32), length=z(2, dt=I32), new_length=z(2, dt=I32), cu=z(3, dt=I32))
    return {**a, **change}


def _evict_args(**change):
    a = dict(pool=z(5, 2, PAGE, dt=torch.uint8), weights=z(5, 2, 64, dt=F32), table=z(2, 2, dt=I32), length=z(2, dt=I32),
             budget=z(2, dt=I32))
    return {**a, **change}


def test_bindings_refuse():
    q, k, pos = z(6, 4, 128), z(6, 2, 128), z(6, dt=I32)
    pool, slot = z(5, 2, PAGE, dt=torch.uint8), z(4, dt=I32)
    for match, call in (
        ("required", lambda: fc.fc_norm_rotate(None, None)),
        ("pos", lambda: fc.fc_norm_rotate(q, k)),
        ("pos", lambda: fc.fc_norm_rotate(q, k, pos=pos[:5])),
        ("pos", lambda: fc.fc_norm_rotate(q, k, pos=pos.long())),
        ("rows", lambda: fc.fc_norm_rotate(q, k[:5], pos=pos)),
        ("q_weight", lambda: fc.fc_norm_rotate(q, k, z(64), None, pos)),
        ("k_weight", lambda: fc.fc_norm_rotate(q, k, None, torch.zeros(128), pos)),
        ("with its weight", lambda: fc.fc_norm_rotate(q, None, None, z(128), pos)),
        ("result", lambda: fc.fc_norm_rotate(q, k, pos=pos, out=(z(6, 3, 128), k))),
        ("result", lambda: fc.fc_norm_rotate(q, k, pos=pos, out=(q, None))),
        ("pair", lambda: fc.fc_norm_rotate(q, k, pos=pos, out=(q,))),
        ("pool", lambda: fc.fc_paged_byte_write(z(5, 2, 8704, dt=torch.uint8), k, k, slot)),
        ("src", lambda: fc.fc_paged_byte_write(pool, k, k, slot, src=slot[:3])),
        ("differ", lambda: fc.fc_paged_byte_write(pool, k, k[:5], slot)),
        ("k must", lambda: fc.fc_paged_byte_write(pool, q, k, slot)),
        ("v must", lambda: fc.fc_paged_byte_read(pool, slot, out=(z(4, 2, 128), z(3, 2, 128)))),
        ("weights", lambda: fc.fc_paged_byte_weights(**_weights_args(weights=z(5, 2, 64)))),
        ("weights", lambda: fc.fc_paged_byte_weights(**_weights_args(weights=z(4, 2, 64, dt=F32)))),
        ("lse", lambda: fc.fc_paged_byte_weights(**_weights_args(lse=z(6, 4, dt=F32)))),
        ("cu", lambda: fc.fc_paged_byte_weights(**_weights_args(cu=z(2, dt=I32)))),
        ("length", lambda: fc.fc_paged_byte_weights(**_weights_args(length=z(3, dt=I32)))),
        ("src", lambda: fc.fc_paged_byte_weights(**_weights_args(src=z(3, dt=torch.int64)))),
        ("weights", lambda: fc.fc_paged_byte_evict(**_evict_args(weights=z(5, 2, 32, dt=F32)))),
        ("budget", lambda: fc.fc_paged_byte_evict(**_evict_args(budget=z(3, dt=I32)))),
        ("add", lambda: fc.fc_paged_byte_evict(**_evict_args(add=z(3, dt=I32)))),
        ("workspace", lambda: fc.fc_paged_byte_evict(**_evict_args(workspace=z(3, dt=I32)))),
    ):
        with pytest.raises(ValueError, match=match):
            call()


def test_bindings_refuse_host_tensors():
    k, slot, pool = z(6, 2, 128), z(4, dt=I32), z(5, 2, PAGE, dt=torch.uint8)
    for call in (lambda: fc.fc_paged_byte_attention(**_inputs()), lambda: fc.fc_norm_rotate(k, k, pos=z(6, dt=I32)),
                 lambda: fc.fc_paged_byte_write(pool, k, k, slot), lambda: fc.fc_paged_byte_read(pool, slot),
                 lambda: fc.fc_paged_byte_weights(**_weights_args()), lambda: fc.fc_paged_byte_evict(**_evict_args())):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    assert fc.paged_byte_pool(3, 2, "cpu").shape == (3, 2, PAGE)
    assert fc.paged_token_weights(3, 2, "cpu").eq(0).all()


def test_bindings_refuse_sizes_out_of_range():
    """Numbers that the C call would take 32 bits of."""
    s, one = _inputs(), z(1, dt=I32)
    long, many = one.expand(2 ** 32 + 5), z(1, 2, 128).expand(2 ** 32 + 6, 2, 128)
    wide, k = one.expand(2, 2 ** 32 + 5), z(6, 2, 128)
    for call in (lambda: fc.fc_paged_byte_attention(**s, max_len=2 ** 32 + 64), lambda: fc.fc_paged_byte_read(s["pool"], long),
                 lambda: fc.fc_paged_byte_attention(**{**s, "table": wide}, max_len=64),
                 lambda: fc.fc_paged_byte_write(s["pool"], k, k, long), lambda: fc.fc_paged_byte_write(s["pool"], many, many, one),
                 lambda: fc.fc_paged_byte_read(s["pool"][:1].expand(2 ** 32 + 1, 2, PAGE), one),
                 lambda: fc.fc_norm_rotate(many, None, pos=long), lambda: fc.fc_paged_byte_weights(**_weights_args(), max_len=2 ** 31),
                 lambda: fc.fc_paged_byte_weights(**_weights_args(src=long)),
                 lambda: fc.fc_paged_byte_evict(**_evict_args(), recent=2 ** 32), lambda: fc.fc_paged_byte_evict(**_evict_args(), first=2 ** 31),
                 lambda: fc.fc_paged_byte_evict(**_evict_args(), max_len=2 ** 40)):
        with pytest.raises(ValueError, match="32-bit"):
            call()
