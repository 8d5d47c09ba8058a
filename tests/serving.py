"""Steps of several sequences over a paged cache, for the tests: random layouts, their pages and the tolerances."""
import numpy as np

from oracle import mquant_oracle as orc

D = 128


def aifs(n, spans):
    """AIFS order of n rows, the spans as far as they lie inside."""
    return orc.aifs_build_perm(n, [(a, min(b, n - a)) for a, b in spans if a < n])[0]


def make_step(rng, seqs, hq, hkv, page, before=0, behind=0, spans=(), poison=True):
    """seqs: (new rows, cached tokens with them) per sequence.  Returns a dict of arrays: row_start, pos, q, pages with
    the cached tokens in them and, where `poison`, NaN and infinity in every slot that no row may look at, and table entries out of
    range behind the last page of a sequence.  `before` and `behind` are rows of no sequence."""
    T = before + sum(n for n, _ in seqs) + behind
    start = before + np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
    pos = np.full(T, 3, dtype=np.int32)
    need = [-(-max(length, 0) // page) for _, length in seqs]
    table = np.full((len(seqs), max([1, *need]) + 1), -7, dtype=np.int32)
    n_pages = sum(need) + 3
    order = rng.permutation(n_pages)
    shape = (n_pages, hkv, page, D)
    kp = np.full(shape, np.nan if poison else 0, dtype=np.float16)
    vp = np.full(shape, np.nan if poison else 0, dtype=np.float16)
    if poison:
        vp[:, :, ::2] = np.inf
    at = 0
    for s, (n, length) in enumerate(seqs):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
        slot = np.arange(max(length, 0))
        pages = table[s, slot // page]
        kp[pages, :, slot % page] = rng.standard_normal((len(slot), hkv, D)).astype(np.float16)
        vp[pages, :, slot % page] = (rng.standard_normal((len(slot), hkv, D)) * 2).astype(np.float16)
        pos[start[s]:start[s + 1]] = length - n + aifs(n, spans)
    q = rng.standard_normal((T, hq * D)).astype(np.float16)
    return {"T": T, "start": start, "pos": pos, "table": table, "kp": kp, "vp": vp, "q": q, "hq": hq, "hkv": hkv}


def attention_bound(st, ref, rows=None):
    """Error bound of the attention per element.  Probabilities are rounded to fp16 (half a step: 2^-11 relative, and
    2^-25 where they are subnormal, of a sum that is at least 1), the output once more (2^-11, 2^-25).  A logit is an fp32 sum of 128
    exact products: off by at most 128 * 2^-24 * sum |q k| / sqrt(128), which changes a probability by that much
    relative, numerator and denominator each.  The fp32 sums over the slots add a quarter of the first term at most: accumulators
    take 16 or 32 slots an instruction, 16384 slots are 1024 additions of 2^-24 each, 2^-14."""
    a = lambda x: np.abs(np.nan_to_num(x.astype(np.float64), nan=0.0, posinf=0.0, neginf=0.0))
    clean = {**st, "kp": np.nan_to_num(st["kp"], nan=0.0, posinf=0.0), "vp": a(st["vp"])}
    mass = orc.paged_attention_f64(st["q"], clean["kp"], clean["vp"], st["table"], st["start"], st["pos"], st["hq"], rows=rows)
    top_v = clean["vp"].max()
    group = st["hq"] // st["hkv"]
    k_abs = a(st["kp"]).max(axis=(0, 2))                                        # [hkv, D]
    q_abs = np.abs(st["q"].astype(np.float64)).reshape(st["T"], st["hq"], D)
    logit = (q_abs * np.repeat(k_abs, group, axis=0)).sum(axis=2) * 128 * 2.0 ** -24 / np.sqrt(128.0)
    slots = np.maximum(st["pos"].astype(np.float64) + 1, 0)[:, None]
    rel = np.repeat(1.25 * 2.0 ** -11 + 2 * np.minimum(logit, 2.0 ** -10), D, axis=1)
    return rel * mass + 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 * (1 + slots * top_v)
