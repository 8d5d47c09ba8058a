"""A serving loop's step around the linears as timed cases: from the lengths of the requests to their next tokens.

A case is a dict of plain values.  ``listed()`` holds the named ones, ``draw(rng)`` gives another of the
same ranges, ``prepare(case, seed)`` makes what a program holds before the call, ``run(state)`` is one
pass: in elementary torch operations (``own`` false) or through the package's entry points (``own``
true).  ``work(case)`` counts the bytes and operations that a pass cannot do without and ``exact(case,
seed)`` gives the results from the definitions in 64 bits.  Kinds of work:

  plan    a step's rows, positions, pages and slots from the lengths of its sequences, pages of ended ones given back
  rotary  norm and rotary embedding of queries and keys: both channel orders, part of a head, positions on three
          axes, frequencies stretched for long contexts; in place of the rows or with the write to cache pages
  shared  attention of new rows over cached pages where groups of sequences begin with the same tokens
  sample  the next token of every row of logits by temperature, top-k, top-p, min-p and a given random number

Head layouts are those of the package's workloads (7B-class: 28 query heads on 4; 72B-class: 64 on 8), in draws also
generic ones.  Keys and values of a cache are fp16 [pages, kv heads, page size, 128]; slot j of a sequence is row j % size of
page table[j // size], and a token's slot is its original position, whatever row order its chunk has.
"""
import math

import numpy as np
import torch

own = False

D = 128
EPS = 1e-6


def listed():
    return [
        # One generating sequence: the smallest bookkeeping there is, latency counts.
        {"name": "plan_b1", "kind": "plan", "n_seq": 1, "rows": 1, "kv": 1281, "page": 16, "end": 0},
        # A wide batch of generating sequences of which every ninth has ended.
        {"name": "plan_b256_decode", "kind": "plan", "n_seq": 256, "rows": 1, "kv": 16384, "page": 16, "end": 9},
        # A step that takes in many prompts of unequal lengths beside generating sequences.
        {"name": "plan_b700_t134302", "kind": "plan", "n_seq": 700, "rows": 900, "kv": 4096, "page": 64, "end": 0},
        # Eight generating sequences of a model with channel halves and positions on three axes, keys normalised.
        {"name": "rotary_append_7b_b8", "kind": "rotary", "append": True, "hq": 28, "hkv": 4, "n_seq": 8, "rows": 1, "kv": 1500,
         "page": 16, "halves": True, "rot": 128, "axes": 3, "scaling": "none", "spans": 0, "norm": True},
        # A long prompt with images entering its cache, channel halves, three axes.
        {"name": "rotary_append_7b_t5000", "kind": "rotary", "append": True, "hq": 28, "hkv": 4, "n_seq": 1, "rows": 5000, "kv": 5000,
         "page": 64, "halves": True, "rot": 128, "axes": 3, "scaling": "none", "spans": 2, "norm": False},
        # A long context on the large shapes, frequencies stretched by the turns they make, half of each head rotated.
        {"name": "rotary_72b_t16384_part", "kind": "rotary", "append": False, "hq": 64, "hkv": 8, "n_seq": 1, "rows": 16384,
         "kv": 16384, "page": 16, "halves": False, "rot": 64, "axes": 1, "scaling": "turns", "spans": 4, "norm": True},
        # Four questions on the same image just behind it: few rows, latency counts.
        {"name": "shared_7b_b4_p1280", "kind": "shared", "hq": 28, "hkv": 4, "groups": 1, "n_seq": 4, "rows": 1, "prefix": 1280,
         "suf_min": 9, "suf_max": 60, "page": 16},
        # A batch of requests that all begin with a long system prompt and generate.
        {"name": "shared_72b_b32_p16384", "kind": "shared", "hq": 64, "hkv": 8, "groups": 1, "n_seq": 32, "rows": 1, "prefix": 16384,
         "suf_min": 20, "suf_max": 2000, "page": 64},
        # Questions of many tokens on three documents, ragged, four to a document.
        {"name": "shared_7b_g3_r150_p6001", "kind": "shared", "hq": 28, "hkv": 4, "groups": 3, "n_seq": 12, "rows": 150,
         "prefix": 6001, "suf_min": 150, "suf_max": 700, "page": 16},
        # One generating sequence of a small vocabulary.
        {"name": "sample_b1_v32000", "kind": "sample", "rows": 1, "V": 32000, "dtype": "fp16", "mode": "all"},
        # A batch of requests, each with settings of its own, over a large vocabulary.
        {"name": "sample_b64_v150001_mixed", "kind": "sample", "rows": 64, "V": 150001, "dtype": "fp16", "mode": "mixed"},
        # The widest batch, logits in 32 bits, drawn from all tokens.
        {"name": "sample_b256_v128000_f32", "kind": "sample", "rows": 256, "V": 128000, "dtype": "fp32", "mode": "plain"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("plan", "rotary", "rotary", "shared", "shared", "shared", "sample", "sample", "sample"))
    hq, hkv = rng.choice(((28, 4), (28, 4), (64, 8), (64, 8), (16, 16), (12, 2), (5, 1)))
    page = rng.choice((16, 32, 64, 128))
    if kind == "plan":
        n_seq = _log_int(rng, 1, 700)
        rows = _log_int(rng, 1, max(1, min(1000, 300000 // n_seq)))
        return {"kind": kind, "n_seq": n_seq, "rows": rows, "kv": _log_int(rng, rows, 16384), "page": page,
                "end": rng.choice((0, 2, 7))}
    if kind == "rotary":
        append = rng.random() < 0.6
        rows = _log_int(rng, 1, 5000 if append else 16000)
        n_seq = _log_int(rng, 1, max(1, min(64, 4096 // rows)))
        axes = rng.choice((1, 3))
        rot = rng.choice((128, 128, 64, 96, 32))
        return {"kind": kind, "append": append, "hq": hq, "hkv": hkv, "n_seq": n_seq, "rows": rows,
                "kv": rows + _log_int(rng, 1, 100000) - 1 if not append else rows + rng.randint(0, 2000), "page": page,
                "halves": rng.random() < 0.6, "rot": rot, "axes": axes,
                "scaling": rng.choice(("none", "linear", "base", "turns")), "spans": rng.randint(0, 3), "norm": rng.random() < 0.5}
    if kind == "shared":
        rows = rng.choice((1, 1, rng.randint(2, 9), _log_int(rng, 10, 300)))
        groups = rng.choice((1, 1, 2, 4))
        suf = max(rows, _log_int(rng, 1, 1500))
        slots = min(30000, 240000 // hkv)                       # of all prefixes and all sequences behind them, half each
        n_seq = groups * _log_int(rng, 1, max(1, min(32, 600 // rows, slots // 2 // suf) // groups))
        most = min(slots // 2 // groups, 90 * 10 ** 9 // (4 * D * hq * rows * n_seq))
        prefix = _log_int(rng, min(64, most), most)
        return {"kind": kind, "hq": hq, "hkv": hkv, "groups": groups, "n_seq": n_seq, "rows": rows, "prefix": prefix,
                "suf_min": rng.randint(rows, suf), "suf_max": suf, "page": page}
    V = _log_int(rng, 1000, 150000)
    return {"kind": kind, "rows": _log_int(rng, 1, min(256, 256 * 64000 // V)), "V": V, "dtype": rng.choice(("fp16", "fp16", "fp32")),
            "mode": rng.choice(("all", "mixed", "mixed", "top_p", "plain", "greedy"))}


# ------------------------------------------------------------------------------------ inputs

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly over their logarithm, the largest first, the rest mixed."""
    return [int(round(hi * (lo / hi) ** ((i * 0.6180339887498949) % 1.0))) for i in range(n)]


def _perm(n, spans):
    """AIFS order of n tokens: the visual ones (three quarters, in `spans` segments) ahead of the text."""
    vis = np.zeros(n, dtype=bool)
    if spans:
        length, gap = (3 * n) // (4 * spans), n // (4 * (spans + 1))
        at = gap
        for _ in range(spans):
            vis[at:at + length] = True
            at += length + gap
    return np.concatenate([np.flatnonzero(vis), np.flatnonzero(~vis)]).astype(np.int32)


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _randn(gen, *shape, gain=1.0):
    out = torch.empty(shape, dtype=torch.float16, device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - a)
        flat[a:a + n] = (torch.randn(n, dtype=torch.float32, device="cuda", generator=gen) * gain).half()
    return out


def _plan_rows(case):
    """Tokens cached and new rows of every sequence: prompts and generating sequences in turn, ended ones -1."""
    n, r = case["n_seq"], case["rows"]
    length = np.asarray(_spread(max(1, case["kv"] // 20), case["kv"], n), dtype=np.int32)
    rows = np.ones(n, dtype=np.int32)
    if r > 1:
        prompt = np.arange(n) % 8 != 5
        rows[prompt] = np.asarray(_spread(max(1, r // 60), r, n), dtype=np.int32)[prompt]
        length[prompt & (np.arange(n) % 3 == 0)] = 0
    if case["end"]:
        rows[np.arange(n) % case["end"] == 1] = -1
    return length, rows


def _pages_of(n, P):
    return -(-n // P)


def _axes_positions(pos, n_axes):
    """Positions on three axes as image prompts have them: of 64 tokens in a row the first 48 are an 8-wide grid."""
    if n_axes == 1:
        return pos[None, :].astype(np.int32)
    block, at = pos // 64, pos % 64
    image = at < 48
    start = block * 32
    text = start + at - 32
    return np.stack([np.where(image, start, text), np.where(image, start + at // 8, text),
                     np.where(image, start + at % 8, text)]).astype(np.int32)


def _rotary(case):
    """What a rotation is made of: base, sections of pairs per axis, stretching."""
    half = case["rot"] // 2
    a = half // 4
    sections = (half,) if case["axes"] == 1 else (a, (half - a) // 2, half - a - (half - a) // 2)
    return {"base": 1e6 if case["axes"] == 3 else 1e4, "sections": sections, "factor": 1.0 if case["scaling"] == "none" else 4.0,
            "trained": 4096.0, "low": 1.0, "high": 32.0, "scale": 1.0 if case["scaling"] != "turns" else 0.1 * math.log(4.0) + 1.0}


def _chunk_rows(case):
    """Rows of every sequence: as many as asked or, from 16 on, fewer and fewer."""
    return [case["rows"] if case["rows"] < 16 else max(1, case["rows"] - 11 * i) for i in range(case["n_seq"])]


def _settings(case):
    """Temperature, top-k, top-p and min-p of every row."""
    kinds = {"all": [(0.8, 50, 0.9, 0.02)], "top_p": [(1.0, 0, 0.95, 0.0), (0.7, 0, 0.8, 0.0)], "plain": [(1.0, 0, 1.0, 0.0)],
             "greedy": [(0.0, 0, 1.0, 0.0)],
             "mixed": [(0.7, 0, 0.9, 0.0), (1.0, 50, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.2, 200, 0.95, 0.0), (1.0, 0, 1.0, 0.05),
                       (1.0, 0, 1.0, 0.0), (0.8, 40, 0.95, 0.05)]}[case["mode"]]
    rows = [kinds[i % len(kinds)] for i in range(case["rows"])]
    return tuple(np.asarray(col) for col in zip(*rows))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    st = {"case": case, "kind": case["kind"]}
    if case["kind"] == "sample":
        B, V = case["rows"], case["V"]
        # logits of a model: probabilities fall as a power of the rank, scattered over the vocabulary
        logits = torch.empty((B, V), dtype=torch.float32, device="cuda")
        for a in range(0, B, 32):
            b = min(B, a + 32)
            logits[a:b] = (3.0 - 1.1 * torch.log(1e-9 + torch.rand((b - a, V), device="cuda", generator=gen))
                           + 0.5 * torch.randn((b - a, V), device="cuda", generator=gen))
        t, k, p, m = _settings(case)
        st.update(logits=logits.half() if case["dtype"] == "fp16" else logits, temperature=_cuda(t.astype(np.float32)),
                  top_k=_cuda(k.astype(np.int32)), top_p=_cuda(p.astype(np.float32)), min_p=_cuda(m.astype(np.float32)),
                  u=torch.rand(B, dtype=torch.float32, device="cuda", generator=gen),
                  token=torch.empty(B, dtype=torch.int32, device="cuda"), logprob=torch.empty(B, dtype=torch.float32, device="cuda"))
        if own:
            from paper_2502_00425_amd import binding as mq
            st["ws"] = torch.empty(mq.sample_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
        return st
    P = case["page"]
    if case["kind"] == "plan":
        length, rows = _plan_rows(case)
        T = int(rows[rows > 0].sum())
        have = [_pages_of(int(n), P) for n in length]
        need = [_pages_of(int(n + max(r, 0)), P) - h for n, r, h in zip(length, rows, have)]
        shared = np.minimum(np.asarray(have), np.arange(len(have)) % 3).astype(np.int32)
        n_pages = sum(have) + sum(need) + 5
        ids = torch.randperm(n_pages, device="cuda", generator=gen, dtype=torch.int32)
        table = torch.full((case["n_seq"], max(h + n for h, n in zip(have, need)) + 1), -1, dtype=torch.int32, device="cuda")
        at = np.cumsum([0] + have)
        where = torch.arange(table.shape[1], device="cuda")[None, :]
        held = where < _cuda(np.asarray(have))[:, None]
        table[held] = ids[(where + _cuda(at[:-1])[:, None])[held]]
        ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        head, count = int(torch.randint(0, n_pages, (1,), device="cuda", generator=gen)), n_pages - int(at[-1])
        ring[(head + torch.arange(count, device="cuda")) % n_pages] = ids[int(at[-1]):]
        order = np.concatenate([_perm(int(r), 1 if r > 16 else 0) for r in rows if r > 0]) if T else np.zeros(0, np.int32)
        st.update(T=T, page=P, table=table, ring=ring, ring_state=_cuda(np.asarray([head, count], np.int32)), length=_cuda(length),
                  rows=_cuda(rows), shared=_cuda(shared), order=_cuda(order.astype(np.int32)), **_plan_outputs(case["n_seq"], T))
        return st
    hq, hkv = case["hq"], case["hkv"]
    if case["kind"] == "rotary":
        rows = _chunk_rows(case)
        lens = [max(r, n) for r, n in zip(rows, _spread(max(1, case["kv"] // 3), case["kv"], len(rows)))]
    else:
        rows = _chunk_rows(case)
        lens = [case["prefix"] + max(r, n) for r, n in zip(rows, _spread(case["suf_min"], case["suf_max"], len(rows)))]
    start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    pos = np.concatenate([n - r + _perm(r, case.get("spans", 0)) for r, n in zip(rows, lens)]).astype(np.int32)
    T = int(start[-1])
    st.update(T=T, hq=hq, hkv=hkv, page=P, rows=rows, lens=lens, start=_cuda(start), pos=_cuda(pos))
    if case["kind"] == "shared" or case["append"]:
        need = [_pages_of(n, P) for n in lens]
        n_seq, groups = len(lens), case.get("groups", 0)
        table = np.full((n_seq, max(need)), -1, dtype=np.int32)
        ids = torch.randperm(sum(need) + 3, device="cuda", generator=gen, dtype=torch.int32)
        host = ids.cpu().numpy()
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = host[at:at + n]
            at += n
        if groups:
            per = n_seq // groups
            group_start = np.arange(groups + 1, dtype=np.int32) * per
            prefix = np.asarray([max(1, case["prefix"] - 5 * g) for g in range(groups)], dtype=np.int32)
            for s in range(n_seq):                              # whole pages of the prefix are the first sequence's
                g = s // per
                table[s, :prefix[g] // P] = table[g * per, :prefix[g] // P]
            st.update(group_start=_cuda(group_start), prefix=_cuda(prefix), group_host=group_start, prefix_host=prefix)
        st.update(table=_cuda(table), k_pages=_randn(gen, sum(need) + 3, hkv, P, D), v_pages=_randn(gen, sum(need) + 3, hkv, P, D))
        if groups:
            for s in range(n_seq):                              # the page in which a prefix ends holds its last tokens for everyone
                g = s // per
                full, rest = prefix[g] // P, prefix[g] % P
                if rest and s != g * per:
                    for pages in (st["k_pages"], st["v_pages"]):
                        pages[table[s, full], :, :rest] = pages[table[g * per, full], :, :rest]
        if own:
            from paper_2502_00425_amd import binding as mq
            st["cache"] = mq.PagedCache(st["k_pages"], st["v_pages"], st["table"])
    if case["kind"] == "shared":
        st.update(q=_randn(gen, T, hq * D, gain=1.5), out=torch.empty((T, hq * D), dtype=torch.float16, device="cuda"),
                  bounds=(max(rows), int(prefix.max()), max(n - int(prefix[s // per]) for s, n in enumerate(lens))))
        if own:
            from paper_2502_00425_amd import binding as mq
            st["ws"] = torch.empty(mq.paged_attention_shared_workspace_bytes(T, st["cache"], groups, hq, *st["bounds"]),
                                   dtype=torch.uint8, device="cuda")
        return st
    rot = _rotary(case)
    qkv = _randn(gen, T, (hq + 2 * hkv) * D, gain=2.0)          # the qkv linear's output
    axes = _axes_positions(pos, case["axes"])
    st.update(q=qkv[:, :hq * D], k=qkv[:, hq * D:(hq + hkv) * D], v=qkv[:, (hq + hkv) * D:], rope_pos=_cuda(axes), rot=rot,
              q_out=torch.empty((T, hq * D), dtype=torch.float16, device="cuda"), wq=None, wk=None)
    if not case["append"]:
        st["k_out"] = torch.empty((T, hkv * D), dtype=torch.float16, device="cuda")
    if case["norm"]:
        st.update(wq=(0.5 + torch.rand(D, device="cuda", generator=gen)).half(),
                  wk=(0.5 + torch.rand(D, device="cuda", generator=gen)).half())
    if own:
        from paper_2502_00425_amd import binding as mq
        st["turn"] = mq.Rotary(case["rot"], base=rot["base"], halves=case["halves"], sections=rot["sections"],
                               scaling=case["scaling"], factor=rot["factor"], trained=rot["trained"], low=rot["low"],
                               high=rot["high"], scale=rot["scale"])
    return st


def _plan_outputs(n_seq, T):
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"new_state": torch.empty(2, **i32), "new_length": torch.empty(n_seq, **i32), "row_start": torch.empty(n_seq + 1, **i32),
            "pos": torch.empty(T, **i32), "slots": torch.empty(T, dtype=torch.int64, device="cuda")}


# --------------------------------------------------------------------------------- one pass

def _plan_plain(st):
    """Plain form of the bookkeeping: sums along the sequences, pages and rows by index."""
    P, table, ring, T = st["page"], st["table"], st["ring"], st["T"]
    N, dev = ring.numel(), table.device
    length, rows = st["length"].long(), st["rows"].long()
    ended = rows < 0
    have = (length + P - 1) // P
    r = torch.where((rows > 0) & (length + rows <= table.shape[1] * P), rows, 0)
    need = (length + r + P - 1) // P - have
    given = torch.where(ended, (have - torch.minimum(st["shared"].long(), have)).clamp(min=0), 0)
    head, count = st["ring_state"].long()
    back = given.cumsum(0) - given
    width = torch.arange(table.shape[1], device=dev)
    which = ended[:, None] & (width >= st["shared"][:, None]) & (width < have[:, None])
    seq, col = which.nonzero(as_tuple=True)
    ring[(head + count + back[seq] + col - st["shared"].long()[seq]) % N] = table[seq, col]
    there = (count + given.sum()).clamp(max=N)
    served = (r > 0) & (r.cumsum(0) <= T) & (need.cumsum(0) <= there)
    r, need = torch.where(served, r, 0), torch.where(served, need, 0)
    first = need.cumsum(0) - need
    seq, col = ((width >= have[:, None]) & (width < (have + need)[:, None])).nonzero(as_tuple=True)
    table[seq, col] = ring[(head + first[seq] + col - have[seq]) % N]
    taken = need.sum()
    st["new_state"].copy_(torch.stack(((head + taken) % N, there - taken)))
    st["new_length"].copy_(torch.where(ended, 0, length + r))
    start = torch.cat((torch.zeros(1, dtype=torch.long, device=dev), r.cumsum(0)))
    st["row_start"].copy_(start)
    row = torch.arange(T, device=dev)
    of = torch.searchsorted(start[1:].contiguous(), row, right=True)
    inside = of < len(r)
    of = of.clamp(max=len(r) - 1)
    pos = length[of] + st["order"].long()
    st["pos"].copy_(torch.where(inside, pos, -1))
    st["slots"].copy_(torch.where(inside, table[of, pos // P].long() * P + pos % P, -1))
    return st["row_start"], st["pos"], st["slots"], st["new_length"], table, ring, st["new_state"]


def _frequencies(case, rot, dev):
    """Radians a position per pair, in 64 bits."""
    R, base, s = case["rot"], rot["base"], rot["factor"]
    j = torch.arange(R // 2, dtype=torch.float64, device=dev)
    if case["scaling"] == "base":
        base = base * s ** (R / (R - 2))
    f = base ** (-2.0 * j / R)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "turns":
        turns = rot["trained"] * f / (2 * math.pi)
        keep = ((turns - rot["low"]) / (rot["high"] - rot["low"])).clamp(0, 1)
        f = f / s * (1 - keep) + f * keep
    return f


def _rotate(st, x, heads, w):
    """Plain form of the norm and the rotation: angles in 64 bits, the rest in 32."""
    case, rot, T, R = st["case"], st["rot"], x.shape[0], st["case"]["rot"]
    x = x.float().view(T, heads, D)
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w.float()
    f = _frequencies(case, rot, x.device)
    angle = torch.cat([st["rope_pos"][a].double()[:, None] * part for a, part in enumerate(f.split(rot["sections"]))], dim=1)
    c, s = (torch.cos(angle) * rot["scale"]).float()[:, None, :], (torch.sin(angle) * rot["scale"]).float()[:, None, :]
    y = x.clone()
    if case["halves"]:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = a * c - b * s, a * s + b * c
    return y.view(T, heads * D)


def _rotary_plain(st):
    st["q_out"].copy_(_rotate(st, st["q"], st["hq"], st["wq"]))
    k = _rotate(st, st["k"], st["hkv"], st["wk"]).half()
    if not st["case"]["append"]:
        st["k_out"].copy_(k)
        return st["q_out"], st["k_out"]
    row = torch.arange(st["T"], device=k.device)
    seq = torch.searchsorted(st["start"][1:].contiguous(), row, right=True)
    pos = st["pos"].long()
    page, slot = st["table"][seq, pos // st["page"]].long(), pos % st["page"]
    st["k_pages"][page, :, slot] = k.view(-1, st["hkv"], D)
    st["v_pages"][page, :, slot] = st["v"].reshape(-1, st["hkv"], D)
    return st["q_out"], st["k_pages"], st["v_pages"]


def _shared_plain(st):
    """Plain form of the attention: per sequence, some key/value heads at a time."""
    hq, hkv = st["hq"], st["hkv"]
    G, at = hq // hkv, 0
    for s, (n, length) in enumerate(zip(st["rows"], st["lens"])):
        ids = st["table"][s, :_pages_of(length, st["page"])].long()
        q = st["q"][at:at + n].float().view(n, hkv, G, D).permute(1, 0, 2, 3).reshape(hkv, n * G, D)
        seen = torch.arange(length, device=q.device)[None, :] <= st["pos"][at:at + n].repeat_interleave(G)[:, None]
        k = st["k_pages"][ids].float().permute(1, 3, 0, 2).reshape(hkv, D, -1)[:, :, :length].contiguous()
        v = st["v_pages"][ids].float().permute(1, 0, 2, 3).reshape(hkv, -1, D)[:, :length].contiguous()
        step = max(1, min(hkv, (1 << 29) // (n * G * length)))
        for h in range(0, hkv, step):
            z = torch.matmul(q[h:h + step], k[h:h + step]) * (1.0 / math.sqrt(D))
            z = torch.where(seen, z, float("-inf"))
            p = torch.exp(z - z.amax(dim=-1, keepdim=True))
            o = torch.matmul(p, v[h:h + step]) / p.sum(dim=-1, keepdim=True)
            heads = o.view(-1, n, G, D).permute(1, 0, 2, 3).reshape(n, -1)
            st["out"][at:at + n, h * G * D:h * G * D + heads.shape[1]] = heads.half()
        at += n
    return st["out"]


def _sample_plain(st):
    """Plain form of the choice, in 64 bits: rows sorted, filters as truth values, sums along the vocabulary."""
    V = st["logits"].shape[1]
    col = torch.arange(V, device=st["logits"].device)[None, :]
    for a in range(0, st["logits"].shape[0], 32):
        b = slice(a, a + 32)
        z = st["logits"][b].double()
        t = st["temperature"][b].double()[:, None]
        k, p, m, u = (st[x][b][:, None] for x in ("top_k", "top_p", "min_p", "u"))
        z, at = torch.sort(z, dim=1, descending=True, stable=True)
        greedy = t <= 0
        w = torch.exp((z - z[:, :1]) / torch.where(greedy, 1.0, t))
        w = torch.where((col < k) | (k <= 0), w, 0.0)
        w = torch.where(greedy & (col > 0), 0.0, w)
        before = w.cumsum(1) - w
        w = torch.where((before < p.double() * w.sum(1, keepdim=True)) | (p >= 1) | (col == 0), w, 0.0)
        w = torch.where((w >= m.double()) | (m <= 0), w, 0.0)
        w = torch.zeros_like(w).scatter_(1, at, w)
        mass = w.cumsum(1)
        total = mass[:, -1:].contiguous()
        token = torch.searchsorted(mass, u.double() * total, right=True)
        st["token"][b] = token[:, 0]
        st["logprob"][b] = torch.log(w.gather(1, token) / total)[:, 0]
    return st["token"], st["logprob"]


def run(st):
    if not own:
        return {"plan": _plan_plain, "rotary": _rotary_plain, "shared": _shared_plain, "sample": _sample_plain}[st["kind"]](st)
    from paper_2502_00425_amd import binding as mq
    if st["kind"] == "plan":
        mq.step_plan(st["length"], st["rows"], st["table"], st["page"], st["ring"], st["ring_state"], st["T"], shared_dev=st["shared"],
                     order_dev=st["order"], length_out=st["new_length"], state_out=st["new_state"], row_start=st["row_start"],
                     pos=st["pos"], slots=st["slots"])
        return st["row_start"], st["pos"], st["slots"], st["new_length"], st["table"], st["ring"], st["new_state"]
    if st["kind"] == "shared":
        return mq.paged_attention_shared(st["q"], st["cache"], st["start"], st["pos"], st["group_start"], st["prefix"], st["hq"],
                                         *st["bounds"], out=st["out"], workspace=st["ws"])
    if st["kind"] == "sample":
        return mq.sample(st["logits"], st["temperature"], st["top_k"], st["top_p"], st["min_p"], st["u"], out=st["token"],
                         logprob=st["logprob"], workspace=st["ws"])
    if not st["case"]["append"]:
        return mq.rotary_apply(st["q"], st["k"], st["rope_pos"], st["turn"], st["hq"], st["hkv"], st["wq"], st["wk"], eps=EPS,
                               q_out=st["q_out"], k_out=st["k_out"])
    mq.rotary_append(st["q"], st["k"], st["v"], st["cache"], st["start"], st["pos"], st["turn"], st["hq"], st["wq"], st["wk"],
                     eps=EPS, rope_pos_dev=st["rope_pos"], q_out=st["q_out"])
    return st["q_out"], st["k_pages"], st["v_pages"]


def work(case):
    if case["kind"] == "sample":
        per = 2 if case["dtype"] == "fp16" else 4
        return {"bytes": case["rows"] * (case["V"] * per + 28), "flops": case["rows"] * case["V"] * 2}
    P = case["page"]
    if case["kind"] == "plan":
        length, rows = _plan_rows(case)
        T = int(rows[rows > 0].sum())
        pages = sum(_pages_of(int(n + r), P) - _pages_of(int(n), P) for n, r in zip(length, rows) if r > 0)
        pages += sum(max(0, _pages_of(int(n), P) - i % 3) for i, (n, r) in enumerate(zip(length, rows)) if r < 0)
        return {"bytes": case["n_seq"] * 20 + 16 * T + 8 * pages, "flops": 4 * T}
    hq, hkv, rows = case["hq"], case["hkv"], _chunk_rows(case)
    T = sum(rows)
    if case["kind"] == "rotary":
        heads = hq + (2 if case["append"] else 1) * hkv
        return {"bytes": T * (heads * D * 4 + 4 * case["axes"] + (4 if case["append"] else 0)),
                "flops": T * (hq + hkv) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    lens = [max(r, n) for r, n in zip(rows, _spread(case["suf_min"], case["suf_max"], len(rows)))]
    slots = case["groups"] * case["prefix"] + sum(lens)
    seen = sum(r * (case["prefix"] + n) - r * (r - 1) // 2 for r, n in zip(rows, lens))
    return {"bytes": slots * hkv * D * 4 + T * (hq * D * 4 + 4) + 4 * (slots // P), "flops": 4 * D * hq * seen}


# ------------------------------------------------------------------------- from the definitions

def _exact_plan(case, st):
    """Sequence by sequence, page by page."""
    P, T = case["page"], st["T"]
    length, rows, shared, order = (st[k].cpu().numpy().tolist() for k in ("length", "rows", "shared", "order"))
    table, ring = st["table"].cpu().numpy(), st["ring"].cpu().numpy()
    N, (head, count) = len(ring), st["ring_state"].tolist()
    for s, r in enumerate(rows):
        if r < 0:
            for page in range(shared[s], _pages_of(length[s], P)):
                ring[(head + count) % N] = table[s, page]
                count += 1
    start, pos, slots, new, open_, want = [0], [], [], [], True, 0
    for s, r in enumerate(rows):
        if r < 0:
            new.append(0)
            start.append(start[-1])
            continue
        first, last = _pages_of(length[s], P), _pages_of(length[s] + r, P)
        open_ = open_ and start[-1] + r <= T and last - first <= count
        r = r if open_ else 0
        for page in range(first, last if open_ else first):
            table[s, page] = ring[head]
            head, count = (head + 1) % N, count - 1
        for i in range(r):
            at = length[s] + order[start[-1] + i]
            pos.append(at)
            slots.append(int(table[s, at // P]) * P + at % P)
        new.append(length[s] + r)
        start.append(start[-1] + r)
    pad = [-1] * (T - len(pos))
    i32 = torch.int32
    return (torch.tensor(start, dtype=i32), torch.tensor(pos + pad, dtype=i32), torch.tensor(slots + pad, dtype=torch.int64),
            torch.tensor(new, dtype=i32), torch.from_numpy(table), torch.from_numpy(ring), torch.tensor([head, count], dtype=i32))


def _exact_rotate(case, st, x, heads, w):
    """Row block by row block: the definition as a product with unit complex numbers."""
    rot, R = st["rot"], case["rot"]
    half, base = R // 2, rot["base"]
    if case["scaling"] == "base":
        base = math.exp(math.log(base) + math.log(rot["factor"]) * R / (R - 2.0))
    theta = []
    for j in range(half):
        f = math.exp(-math.log(base) * j / half)
        if case["scaling"] == "linear":
            f /= rot["factor"]
        elif case["scaling"] == "turns":
            wave = 2 * math.pi / f
            g = min(1.0, max(0.0, (rot["trained"] / wave - rot["low"]) / (rot["high"] - rot["low"])))
            f = f * g + (f / rot["factor"]) * (1 - g)
        theta.append(f)
    theta = torch.tensor(theta, dtype=torch.float64, device=x.device)
    axis = torch.tensor(sum([[a] * n for a, n in enumerate(rot["sections"])], []), device=x.device)
    out = torch.empty((x.shape[0], heads * D), dtype=torch.float64, device=x.device)
    first = torch.arange(half, device=x.device) if case["halves"] else torch.arange(0, R, 2, device=x.device)
    second = first + (half if case["halves"] else 1)
    for a in range(0, x.shape[0], 1024):
        u = x[a:a + 1024].double().reshape(-1, heads, D)
        if w is not None:
            u = u / torch.sqrt(u.square().sum(dim=2, keepdim=True) / D + EPS) * w.double()
        angle = st["rope_pos"][:, a:a + 1024].double()[axis].t().contiguous() * theta[None, :]
        z = torch.complex(u[..., first], u[..., second]) * torch.polar(torch.full_like(angle, rot["scale"]), angle)[:, None, :]
        u = u.clone()
        u[..., first], u[..., second] = z.real, z.imag
        out[a:a + 1024] = u.reshape(-1, heads * D)
    return out


def _exact_shared(case, st):
    hq, hkv, P, at = st["hq"], st["hkv"], st["page"], 0
    out = torch.empty((st["T"], hq, D), dtype=torch.float64, device="cuda")
    for s, (n, length) in enumerate(zip(st["rows"], st["lens"])):
        slot = torch.arange(length, device="cuda")
        page = st["table"][s].long()[torch.div(slot, P, rounding_mode="floor")]
        for g in range(hkv):
            k, v = st["k_pages"][page, g, slot % P].double(), st["v_pages"][page, g, slot % P].double()
            kt = k.t().contiguous()
            for h in range(g * (hq // hkv), (g + 1) * (hq // hkv)):
                z = (st["q"][at:at + n, h * D:(h + 1) * D].double() @ kt) / math.sqrt(D)
                z.masked_fill_(slot[None, :] > st["pos"][at:at + n, None], float("-inf"))
                out[at:at + n, h] = torch.exp(z - torch.logsumexp(z, dim=1, keepdim=True)) @ v
        at += n
    return out.reshape(st["T"], hq * D)


def _exact_sample(case, st):
    """Row by row on the host: the kept tokens as a set, then the draw along the vocabulary."""
    logits = st["logits"].double().cpu().numpy()
    t, k, p, m, u = (st[x].cpu().numpy().tolist() for x in ("temperature", "top_k", "top_p", "min_p", "u"))
    token, logprob = [], []
    for z, ti, ki, pi, mi, ui in zip(logits, t, k, p, m, u):
        if ti <= 0:
            token.append(int(np.argmax(z)))
            logprob.append(0.0)
            continue
        w = np.exp((z - z.max()) / ti)
        order = np.argsort(-z, kind="stable")
        kept = order[:ki] if ki > 0 else order
        if pi < 1:
            mass = np.cumsum(w[kept])
            kept = kept[:1 + int(np.searchsorted(mass[:-1], pi * mass[-1], side="left"))]
        if mi > 0:
            kept = kept[w[kept] >= mi]
        kept = np.sort(kept)
        mass = np.cumsum(w[kept])
        at = min(int(np.searchsorted(mass, ui * mass[-1], side="right")), len(kept) - 1)
        token.append(int(kept[at]))
        logprob.append(math.log(w[kept[at]] / mass[-1]))
    return torch.tensor(token, dtype=torch.int32), torch.tensor(logprob, dtype=torch.float64)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "plan":
        return _exact_plan(case, st)
    if case["kind"] == "shared":
        return _exact_shared(case, st)
    if case["kind"] == "sample":
        return _exact_sample(case, st)
    q = _exact_rotate(case, st, st["q"], st["hq"], st["wq"])
    k = _exact_rotate(case, st, st["k"], st["hkv"], st["wk"])
    if not case["append"]:
        return q, k
    kp, vp, at = st["k_pages"].double(), st["v_pages"].double(), 0
    for s, n in enumerate(st["rows"]):
        p = st["pos"][at:at + n].long()
        page = st["table"][s].long()[torch.div(p, st["page"], rounding_mode="floor")]
        kp[page, :, p % st["page"]] = k[at:at + n].view(n, -1, D)
        vp[page, :, p % st["page"]] = st["v"][at:at + n].double().reshape(n, -1, D)
        at += n
    return q, kp, vp
