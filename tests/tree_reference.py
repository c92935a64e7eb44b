"""Plain forms, in 64 bits and request by request, of the calls on drafted trees and tails: what the kernels are compared with."""
import numpy as np

PAGE = 16
EPS_BF16 = 2.0 ** -8                    # half a step of a bf16 rounding, relative


def attend(q, keys, values, see):
    """One request: q [n][Hq][D], keys and values [S][Hkv][D], see [n][S] truth values -> out and the bound on a kernel's error, [n][Hq][D].

    The bound counts what the kernels round: probabilities to bf16 for the product with V (half a step each, so half a step of the
    weighted mean of |v| in all), the result to bf16, and the scores, sums of D products of bf16 values in fp32 (each addition half a step of
    2^-23 of what it holds, by no more than the sum of the products' sizes), which shift every probability by as much and the row sum, too.
    Exponentials, row sums and the merge of splits are a few 2^-22: 2^-16 is more than all of them."""
    n, n_q, d = q.shape
    rep = n_q // keys.shape[1]
    out, tol = np.zeros((n, n_q, d)), np.zeros((n, n_q, d))
    for h in range(n_q):
        k, v = keys[:, h // rep], values[:, h // rep]
        s = q[:, h] @ k.T / np.sqrt(d)
        size = (np.abs(q[:, h]) @ np.abs(k).T / np.sqrt(d))
        for i in range(n):
            at = np.nonzero(see[i])[0]
            if len(at) == 0:
                continue
            w = np.exp(s[i, at] - s[i, at].max())
            w /= w.sum()
            out[i, h] = w @ v[at]
            off = d * 2.0 ** -23 * size[i, at].max()
            tol[i, h] = 1.05 * ((EPS_BF16 + 2 * off + 2.0 ** -16) * (w @ np.abs(v[at])) + EPS_BF16 * np.abs(out[i, h]))
    return out, tol


def ancestors(parent, n):
    """[n][n] truth values; a parent that is no lower index counts as none, parent None is a chain."""
    see = np.zeros((n, n), bool)
    for i in range(n):
        p = i - 1 if parent is None else int(parent[i])
        if 0 <= p < i:
            see[i] = see[p]
        see[i, i] = True
    return see


def bits(see, width):
    words = np.zeros(width, np.uint64)
    for i, row in enumerate(see):
        words[i] = sum(1 << int(j) for j in np.nonzero(row)[0])
    return words.view(np.int64)


def tables(tail_len, n_new, parent, pos_base, table, n_blocks, free, n_free, n_max, masks):
    """As enl_tail_tables; returns everything it writes, and how many requests failed."""
    table, n_blocks, free = table.copy(), n_blocks.copy(), free.copy()
    batch = len(tail_len)
    slot, pos, mask = np.full((batch, n_max), -1, np.int32), np.zeros((batch, n_max), np.int32), np.zeros((batch, n_max), np.int64)
    failed, given, want_sum, avail, taken = 0, [], 0, n_free, 0
    for b in range(batch):
        n = 0 if tail_len[b] < 0 else min(max(int(n_new[b]), 0), n_max)
        if tail_len[b] < 0:
            given += table[b, :n_blocks[b]].tolist()
            n_blocks[b] = 0
            continue
        want = -(-(int(tail_len[b]) + n) // PAGE)
        take = max(0, want - int(n_blocks[b]))
        ok = want <= table.shape[1]
        if ok:
            want_sum += take
            if take and want_sum > avail:
                ok = False
            elif take:
                for k in range(take):
                    taken += 1
                    table[b, n_blocks[b] + k] = free[avail - taken]
                n_blocks[b] += take
        failed += not ok
        see = ancestors(None if parent is None else parent[b], n)
        for i in range(n):
            r = int(tail_len[b]) + i
            if ok:
                slot[b, i] = table[b, r // PAGE] * PAGE + r % PAGE
            pos[b, i] = (0 if pos_base is None else pos_base[b]) + tail_len[b] + see[i].sum() - 1
        if masks:
            mask[b] = bits(see, n_max)
    top = avail - taken
    for k, page in enumerate(given):
        free[top + k] = page
    return dict(table=table, n_blocks=n_blocks, free=free, n_free=top + len(given), slot=slot, position=pos, mask=mask, failed=failed)


def accept(n_new, parent, token, target, first, n_max):
    batch = len(n_new)
    out, count, nxt = np.full((batch, n_max), -1, np.int32), np.zeros(batch, np.int32), np.full(batch, -1, np.int32)
    for b in range(batch):
        n = min(max(int(n_new[b]), 0), n_max)
        up = [i - 1 if parent is None else int(parent[b, i]) for i in range(n)]
        up = [p if 0 <= p < i else -1 for i, p in enumerate(up)]
        at, want = -1, None if first is None else int(first[b])
        if first is not None:
            nxt[b] = first[b]
        while True:
            if at < 0 and want is None:
                found = [0] if n else []
            else:
                found = [i for i in range(n) if up[i] == at and token[b, i] == want]
            if not found:
                break
            at = found[0]
            out[b, count[b]] = at
            count[b] += 1
            want = int(target[b, at])
            nxt[b] = want
    return out, count, nxt
