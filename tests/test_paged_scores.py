"""Paged attention on the GPU, within a bound of each key's own roundings: random
rows of every form of the kernels, and rows whose results hang on the last bits
of a query or a key."""
import numpy as np
import pytest
import torch

import paged_bound as pb
from gpu_pipeline import dev, host, say

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_17139_amd as fc  # noqa: E402
from test_paged import BF, D, SIZES, bf16, f64, make_pool, on_gpu, trees  # noqa: E402


def check(q, k_tree, v_tree, pool, table, prefix_len, tree=None, rope_base=10000.0, norm=True):
    """One call on device or host inputs against float64; returns the results."""
    q, k_tree, v_tree = (torch.as_tensor(x).to(BF) for x in (q, k_tree, v_tree))
    prefix_len = np.asarray(prefix_len, np.int32)
    got = f64(fc.fc_paged_attention(q.cuda(), k_tree.cuda(), v_tree.cuda(), pool, dev(table), dev(prefix_len),
                                    tree=on_gpu(tree), rope_base=rope_base))
    t = {} if tree is None else {f: tree[f] for f in ("num_nodes", "mask", "pos_ids")}
    o, bound, most, _ = pb.attention(f64(q), f64(k_tree), f64(v_tree), host(pool), table, prefix_len,
                                     rope_base=rope_base, **t)
    err = np.abs(got - o)
    size = [float(np.sqrt((x ** 2).sum())) for x in (err, most)]
    say(f"  worst {float((err / np.maximum(bound, 1e-30)).max()):.3f} of a bound, norm {size[0]:.3g} of {size[1]:.3g}")
    assert np.isfinite(got).all() and (err <= bound).all()
    assert not norm or size[0] <= size[1]
    return got


@pytest.mark.parametrize("B,R,H,Hkv,lens", SIZES, ids=lambda x: str(x).replace(" ", ""))
def test_random_rows_within_each_keys_roundings(B, R, H, Hkv, lens):
    rng = np.random.default_rng(R * 100 + H + 1)
    say(f"attention B={B} R={R} H={H} Hkv={Hkv} lens={lens}")
    pool = make_pool(rng, 6, Hkv)
    table = rng.integers(0, 6, (B, max(1, -(-max(lens) // 64)))).astype(np.int32)
    row = lambda h, s=1.0: bf16(rng, B, R, h, D, scale=s)  # noqa: E731
    check(row(H), row(Hkv), row(Hkv), pool, table, lens)
    t = trees(rng, B, R)
    check(row(H, 4.0), row(Hkv), row(Hkv), pool, table, lens, t)
    check(row(H, 16.0), row(Hkv), row(Hkv), pool, table, lens, t, rope_base=0.0)


def _tree_of(R, mask, pos=None):
    B = len(mask)
    return dict(num_nodes=np.full(B, R, np.int32), mask=mask,
                pos_ids=np.zeros((B, R), np.int32) if pos is None else pos)


@pytest.mark.parametrize("n", [2, 64, 200, 900])
@pytest.mark.parametrize("R", [1, 7, 20, 40, 65, 100])
def test_the_last_part_of_a_query_decides(R, n):
    """Pairs of cached keys at any place of their pages, in prefixes of one page,
    several, and several parts."""
    rng = np.random.default_rng(1000 * R + n)
    B, Hkv, width = 3, 3, -(-n // 64)
    q, k, v, mask = pb.pairs_of_cached_keys(rng, B, R, Hkv, n)
    table = rng.permutation(B * width).astype(np.int32).reshape(B, width)
    pool = torch.zeros((B * width, Hkv, fc.FC_PAGE_HEAD_BYTES), dtype=torch.uint8, device="cuda")
    slot = table[:, np.arange(n) // 64] * 64 + np.arange(n) % 64
    fc.fc_paged_write(pool, *(torch.from_numpy(x.reshape(B * n, Hkv, D)).to(BF).cuda() for x in (k, v)),
                      dev(slot.reshape(-1).astype(np.int32)), rope_base=0.0)
    say(f"last part of a query R={R} n={n}")
    none = np.zeros((B, R, Hkv, D))
    got = check(q, none, none, pool, table, [n] * B, _tree_of(R, mask), rope_base=0.0, norm=False)
    assert (np.abs(got) < 0.95).all()


@pytest.mark.parametrize("R", [2, 7, 16, 20, 40, 65, 100, 200])
def test_the_last_parts_of_tree_keys_and_queries_decide(R):
    rng = np.random.default_rng(R)
    B, Hkv = 3, 3
    pool, table = make_pool(rng, 1, Hkv), np.zeros((B, 1), np.int32)
    say(f"last parts of tree keys R={R}")
    q, kt, vt, mask, pos = pb.pairs_of_tree_keys(rng, B, R, Hkv, 10000.0)
    check(q, kt, vt, pool, table, [0] * B, _tree_of(R, mask, pos), norm=False)
    for parts, size in ((2, 6.0), (1, 4.1875)):
        q, kt, vt, mask = pb.pairs_of_signs(rng, B, R, Hkv, parts, size)
        check(q, kt, vt, pool, table, [0] * B, _tree_of(R, mask), rope_base=0.0, norm=False)
