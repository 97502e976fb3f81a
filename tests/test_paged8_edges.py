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
