"""Steps whose sequences share prefixes, for the tests: random layouts and their pages."""
import numpy as np

from serving import D, aifs


def make_shared(rng, groups, hq, hkv, page, before=0, behind=0, alone=(0, 0), spans=(), poison=True):
    """groups: (prefix, [(new rows, tokens with them), ...]) each; `alone`: how many of the first and the last sequences are of no
    group (their groups have prefix 0 here).  Where `poison`, every slot that no row may look at holds NaN and infinity, and the table
    entries of a prefix's whole pages are out of range but for the group's first sequence.  `table` is what the entry gets, `full` has every
    sequence's own pages."""
    seqs = [s for _, members in groups for s in members]
    T = before + sum(n for n, _ in seqs) + behind
    start = before + np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
    pos = np.full(T, 3, dtype=np.int32)
    pages_of = lambda n: -(-max(n, 0) // page)
    longest = max([1] + [pages_of(n) for _, n in seqs] + [pages_of(p) for p, _ in groups])
    full = np.full((len(seqs), longest + 1), -7, dtype=np.int32)
    n_pages = 3 + sum(pages_of(p) for p, _ in groups) + sum(pages_of(n) for _, n in seqs)
    order = list(rng.permutation(n_pages))
    kp = np.full((n_pages, hkv, page, D), np.nan if poison else 0, dtype=np.float16)
    vp = np.full_like(kp, np.nan if poison else 0)
    if poison:
        vp[:, :, ::2] = np.inf
    table, group_start, prefix, s = full.copy(), [0], [], 0
    for p, members in groups:
        whole, rest = p // page, p % page
        shared = [order.pop() for _ in range(whole)]
        data = [rng.standard_normal((p, hkv, D)).astype(np.float16), (rng.standard_normal((p, hkv, D)) * 2).astype(np.float16)]
        for i, pg in enumerate(shared):
            for a, x in zip((kp, vp), data):
                a[pg] = x[i * page:(i + 1) * page].transpose(1, 0, 2)
        for m, (n, length) in enumerate(members):
            full[s, :whole] = shared
            own = [order.pop() for _ in range(max(pages_of(length), pages_of(p)) - whole)]
            full[s, whole:whole + len(own)] = own
            table[s] = full[s]
            if poison and m > 0:
                table[s, :whole] = -9 - s
            for a, x, gain in ((kp, data[0], 1), (vp, data[1], 2)):
                if rest:
                    a[full[s, whole], :, :rest] = x[whole * page:].transpose(1, 0, 2)
                if length > p:
                    slot = np.arange(p, length)
                    a[full[s, slot // page], :, slot % page] = (rng.standard_normal((len(slot), hkv, D)) * gain).astype(np.float16)
            pos[start[s]:start[s + 1]] = length - n + aifs(n, spans)
            s += 1
        group_start.append(s)
        prefix.append(p)
    first, last = alone[0], len(groups) - alone[1]
    q = rng.standard_normal((T, hq * D)).astype(np.float16)
    return {"T": T, "start": start, "pos": pos, "table": table, "full": full, "kp": kp, "vp": vp, "q": q, "hq": hq, "hkv": hkv,
            "group_start": np.array(group_start[first:last + 1], dtype=np.int32), "prefix": np.array(prefix[first:last], dtype=np.int32)}
