"""Attention over the paged cache in float64, with what the kernel's roundings may
move each result by - key by key - and a model of its 6-bit parts, for tests of
whether that bound would notice a part that is missing."""
import numpy as np

import oracle

D, GROUP, PARTS = 128, 32, 3
LOG2E = np.log2(np.e)
ALL = ((2, 0), (1, 1), (0, 2), (1, 0), (0, 1), (0, 0))  # (key's part, query's part) of a tree key's score


def group_exponents(x):
    """Per group of 32 dims the smallest e with all magnitudes at most 7.5 * 2^e
    (a hair above: float32 may round a magnitude up), -110 at least."""
    top = np.abs(x).reshape(*x.shape[:-1], D // GROUP, GROUP).max(-1) * (1 + 2.0 ** -20)
    with np.errstate(divide="ignore"):
        e = np.ceil(np.log2(top / 7.5))
    return np.maximum(e, -110)


def six_bits(x, scale):
    """The nearest of the 6-bit values (sign, two exponent bits, three of
    mantissa: steps of 1/8 below 2, 1/4 below 4, 1/2 up to 7.5) times scale."""
    a = np.abs(x) / scale
    step = np.where(a < 2, 0.125, np.where(a < 4, 0.25, 0.5))
    return np.sign(x) * np.minimum(np.round(a / step) * step, 7.5) * scale


def parts_of(x):
    """The three 6-bit parts of rows [..., 128], what each leaves over, and the
    scale 2^e of each dim."""
    f = 2.0 ** np.repeat(group_exponents(x), GROUP, axis=-1)
    part, left = [], []
    for s in range(PARTS):
        part.append(six_bits(x, f * 2.0 ** -(0, 4, 9)[s]))
        x = x - part[-1]
        left.append(x)
    return part, left, f


def turned(x, pos, base):
    """Rows rotated, and of each dim the sum of its pair's magnitudes: what an
    error of the sine and cosine is multiplied by."""
    if not base:
        return x, np.zeros_like(x)
    pair = np.abs(x[..., :D // 2]) + np.abs(x[..., D // 2:])
    return oracle.rope(x, pos, base), np.concatenate([pair, pair], -1)


def attention(q, k_tree, v_tree, pool, table, prefix_len, num_nodes=None, mask=None, pos_ids=None, max_len=None,
              rope_base=10000.0, q_parts=PARTS, k_parts=PARTS, products=ALL, rotate_tree=True):
    """(exact, bound, norm, model) of fc_paged_attention in float64.

    A score (a power of two's exponent: q is scaled by log2(e) / sqrt(128)) is off by
    - what the parts leave: 2^-12 * 2^e a dim (half a step, 2^-4, of the third
      part's lowest binade at a remainder of at most 4 steps of 2^(e - 9): 2^-3 *
      2^(e - 9)), times the other factor; for a tree's key both factors', and the
      three products that are left out, of magnitudes at most |what the part
      before left| + |what the part itself left|;
    - the rotation: 2^-18 for the hardware's sine and cosine, each times a pair's
      magnitudes;
    - fp32: at most 384 products are added, 2^-24 each of the sum of magnitudes,
      and some roundings of factors and of the maximum before and after: 420.
    A weight moves by t = 2^d (1 + 2^-8) - 1 of itself at most (it is rounded to
    bf16), so the result sum p (1 + t) v / sum p (1 + t) by
    sum p t |v - o| / (1 - sum p t); sums are fp32, the result is bf16.

    norm: the same with independent errors of the weights, the root of the sum of
    their squares in place of their sum.  Over random keys roundings are no
    better arranged than that (uniform ones are smaller by another sqrt(3)), so
    the norm of all errors of such a call stays below the norm of these.

    model: the result with the first q_parts and k_parts parts and the products
    given, everything else exact."""
    q, k_tree, v_tree = (np.asarray(x, np.float64) for x in (q, k_tree, v_tree))
    B, R, H, _ = q.shape
    Hkv = k_tree.shape[2]
    out, bound, norm, model = (np.zeros((B, R, H, D)) for _ in range(4))
    for b in range(B):
        P = min(max(int(prefix_len[b]), 0), 64 * np.shape(table)[1] if max_len is None else max_len)
        n = R if num_nodes is None else min(max(int(num_nodes[b]), 0), R)
        pos = P + (np.arange(R) if pos_ids is None else np.asarray(pos_ids[b]).astype(np.int64))
        kc, vc, there = oracle.paged_rows(pool, table[b], P)
        kc, vc = kc[there], vc[there]
        see = np.tril(np.ones((R, R), bool)) if mask is None else np.asarray(mask[b]) == 1
        see = see & (np.arange(R) < n)
        for h in range(H):
            g = h // (H // Hkv)
            qh, q_pair = turned(q[b, :, h] * (LOG2E / np.sqrt(D)), pos, rope_base)
            kt, k_pair = turned(k_tree[b, :, g], pos, rope_base)
            qp, ql, qf = parts_of(qh)
            kp, kl, kf = parts_of(kt)
            if not rotate_tree:
                kp, _, _ = parts_of(k_tree[b, :, g])
            mk, mt, mq = np.abs(kc[:, g]), np.abs(kt), np.abs(qh)
            f32 = 420 * 2.0 ** -24
            s_c, s_t = qh @ kc[:, g].T, qh @ kt.T
            d_c = (2.0 ** -12 * qf + 2.0 ** -18 * q_pair + f32 * mq) @ mk.T
            d_t = (2.0 ** -12 * qf + 2.0 ** -18 * q_pair + f32 * mq) @ mt.T + mq @ (2.0 ** -12 * kf + 2.0 ** -18 * k_pair).T
            d_t += 2.0 ** -24 * qf @ kf.T
            q1, q2, k1, k2 = (np.abs(x) + np.abs(y) for x, y in ((ql[0], ql[1]), (ql[1], ql[2]), (kl[0], kl[1]), (kl[1], kl[2])))
            d_t += q1 @ k2.T + q2 @ k1.T + q2 @ k2.T
            m_c = sum(qp[:q_parts]) @ kc[:, g].T
            m_t = sum(qp[j] @ kp[i].T for i, j in products if i < k_parts and j < q_parts)
            vals = np.concatenate([vc[:, g], v_tree[b, :, g]])
            for i in range(n):
                on = np.concatenate([np.ones(len(kc), bool), see[i]])
                if not on.any():
                    continue
                v = vals[on]
                for s, to in (((s_c, s_t), out), ((m_c, m_t), model)):
                    x = np.concatenate([s[0][i], s[1][i]])[on]
                    p = 2.0 ** (x - x.max())
                    p /= p.sum()
                    to[b, i, h] = p @ v
                    if to is out:
                        exact, top = p, np.abs(x).max()
                d = np.concatenate([d_c[i], d_t[i]])[on] + 2.0 ** -22 * top + 2.0 ** -20
                with np.errstate(over="ignore"):
                    t = 2.0 ** d * (1 + 2.0 ** -8) - 1
                o, pt = out[b, i, h], exact * t
                away, rest = np.abs(v - o), max(1 - pt.sum(), 0.0)
                last = (len(v) + 300) * 2.0 ** -23 * (exact @ np.abs(v)) + 2.0 ** -8 * np.abs(o) + 1e-30
                with np.errstate(divide="ignore", invalid="ignore"):
                    bound[b, i, h] = np.where(pt.sum() < 1, pt @ away / rest, np.inf) * (1 + 2.0 ** -8) + last
                    norm[b, i, h] = np.where(pt.sum() < 1, np.sqrt(pt ** 2 @ away ** 2) / rest, np.inf) * (1 + 2.0 ** -8) + last
    return out, bound, norm, model


def within(got, o, bound, norm):
    """Whether every result lies within its bound and all together within theirs."""
    err = np.abs(got - o)
    return bool((err <= bound).all()), bool(np.sqrt((err ** 2).sum()) <= np.sqrt((norm ** 2).sum()))


def signs_of(x, parts=2):
    """The signs of what the first parts leave of rows [..., 128]."""
    return np.where(parts_of(x)[1][parts - 1] >= 0, 1.0, -1.0)


def balanced(x, parts=2):
    """Of candidates [n][128] the row whose sum of signs_of(x) * x comes nearest to
    zero: its score against that row of signs is small, though every dim's next
    part adds to it."""
    return int(np.abs((signs_of(x, parts) * x).sum(-1)).argmin())


def queries(rng, parts=2):
    """Such a query (bf16, and large), and its signs."""
    many = bf16(rng.standard_normal((4000, D)) * 8)
    i = balanced(many * (LOG2E / np.sqrt(D)), parts)
    return many[i], signs_of(many[i] * (LOG2E / np.sqrt(D)), parts)


def pairs_of_cached_keys(rng, B, R, Hkv, n):
    """Trees whose rows all hold one query a head, and prefixes of n tokens of
    which two lie along and against what its first two parts leave over, with
    values 1 and -1: the result is tanh of their score, in which every dim's
    third part counts the same way.  All other keys lie against the query.  The
    mask admits no tree row.  Nothing is rotated."""
    q = np.zeros((B, R, Hkv, D))
    k, v = np.zeros((B, n, Hkv, D)), rng.choice([-3.0, 2.0], (B, n, Hkv, D))
    for b in range(B):
        at = rng.permutation(n)[:2]
        for h in range(Hkv):
            row, sign = queries(rng)
            q[b, :, h] = row
            k[b, :, h] = -6 * np.sign(row)
            k[b, at[0], h], k[b, at[1], h] = 6 * sign, -6 * sign
            v[b, at[0], h], v[b, at[1], h] = 1.0, -1.0
    return q, k, v, np.zeros((B, R, R), np.int32)


def pairs_of_tree_keys(rng, B, R, Hkv, base):
    """The same of two tree rows that every row may see: at a position of their
    own, their rotated keys have all three parts, and the other rows, at
    position 0, are queries of one magnitude with the signs of what two parts of
    the key leave over."""
    q, kt, vt = (np.zeros((B, R, Hkv, D)) for _ in range(3))
    mask, pos = np.zeros((B, R, R), np.int32), np.zeros((B, R), np.int32)
    for b in range(B):
        at = rng.permutation(R)[:2]
        pos[b, at] = int(rng.integers(100, 4000))
        mask[b][:, at] = 1
        for h in range(Hkv):
            many = bf16(rng.standard_normal((4000, D)))
            many_turned = oracle.rope(many, np.full(4000, pos[b, at[0]]), base)
            i = balanced(many_turned)
            q[b, :, h] = bf16(signs_of(many_turned[i]) * 4 / (LOG2E / np.sqrt(D)))
            kt[b, :, h] = bf16(rng.standard_normal((R, D)))
            kt[b, at[0], h], kt[b, at[1], h] = many[i], -many[i]
            vt[b, :, h] = rng.choice([-3.0, 2.0], (R, D))
            vt[b, at[0], h], vt[b, at[1], h] = 1.0, -1.0
    return q, kt, vt, mask, pos


def pairs_of_signs(rng, B, R, Hkv, parts, size):
    """The same with keys of one magnitude and the signs of what the query's
    first parts leave over: of 6 and after two parts, the query's third part
    times a key's first decides; of 4.1875, of which a key's first part leaves
    0.1875, and after one part, the product of the second parts."""
    q, kt, vt = (np.zeros((B, R, Hkv, D)) for _ in range(3))
    mask = np.zeros((B, R, R), np.int32)
    for b in range(B):
        at = rng.permutation(R)[:2]
        mask[b][:, at] = 1
        for h in range(Hkv):
            q[b, :, h], sign = queries(rng, parts)
            kt[b, :, h] = bf16(rng.standard_normal((R, D)))
            kt[b, at[0], h], kt[b, at[1], h] = size * sign, -size * sign
            vt[b, :, h] = rng.choice([-3.0, 2.0], (R, D))
            vt[b, at[0], h], vt[b, at[1], h] = 1.0, -1.0
    return q, kt, vt, mask


def bf16(x):
    """Float64 values rounded to bf16."""
    u = np.asarray(x, np.float32).view(np.uint32)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)
    return u.view(np.float32).astype(np.float64)
