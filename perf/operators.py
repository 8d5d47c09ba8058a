"""The serving-step operators of a decoder layer as timed cases: what lies between the output of
the qkv linear and the input of the o linear when sequences have a cache, and adapters beside a linear.

A case is a dict of plain values.  ``listed()`` holds the named ones, ``draw(rng)`` gives another of the
same ranges, ``prepare(case, seed)`` makes what a program holds before the call, ``run(state)`` is one
pass: in elementary torch operations (``own`` false) or through the package's entry points (``own``
true).  ``work(case)`` counts the bytes and operations that a pass cannot do without and ``exact(case,
seed)`` gives the results from the definitions in 64 bits.  Kinds of work:

  norm    RMS norm of queries and keys per head and their rotary embedding in one pass, rows of a prompt
  append  the same behind the qkv linear of a serving step, keys and values written to their cache pages
  attend  attention of each sequence's new rows over its cached pages: one row (decode), a few, a chunk
  lora    low-rank adapters of many requests added to the output of a shared projection

Head layouts and projections are those of the package's workloads (7B-class: 28 query heads on 4, 3584
channels; 72B-class: 64 on 8, 8192 channels), in draws also generic ones.  Keys and values of a cache are fp16
[pages, kv heads, page size, 128]; slot j of a sequence is row j % size of page table[j // size], and a token's slot
is its original position, whatever row order its chunk has.  A row sees the slots up to its own position.
"""
import math

import numpy as np
import torch

own = False

D = 128
BASE = 10000.0
EPS = 1e-6
QKV_7B, DOWN_7B, O_7B, GATE_UP_7B = (3584, 4608), (18944, 3584), (3584, 3584), (3584, 37888)
QKV_72B, DOWN_72B = (8192, 10240), (29568, 8192)


def listed():
    return [
        # A short mixed prompt, ragged: launch latency counts.
        {"name": "norm_7b_t77", "kind": "norm", "hq": 28, "hkv": 4, "T": 77, "spans": 1},
        # A long context of several images on the large shapes, the largest call of this pass.
        {"name": "norm_72b_t16384", "kind": "norm", "hq": 64, "hkv": 8, "T": 16384, "spans": 4},
        # Token-by-token generation of one sequence: the smallest call there is.
        {"name": "append_7b_b1", "kind": "append", "hq": 28, "hkv": 4, "n_seq": 1, "rows": 1, "kv_min": 1281, "kv_max": 1281,
         "page": 16, "spans": 0, "norm": True},
        # A prompt with one image entering its cache in one step, rows in AIFS order.
        {"name": "append_7b_t4096", "kind": "append", "hq": 28, "hkv": 4, "n_seq": 1, "rows": 4096, "kv_min": 4096,
         "kv_max": 4096, "page": 64, "spans": 1, "norm": True},
        # One sequence behind a usual prompt: few heads, a short cache, latency counts.
        {"name": "decode_7b_b1_kv1281", "kind": "attend", "hq": 28, "hkv": 4, "n_seq": 1, "rows": 1, "kv_min": 1281,
         "kv_max": 1281, "page": 16, "spans": 0},
        # A batch of generating sequences of very different lengths on the large shapes.
        {"name": "decode_72b_b32_kv16384", "kind": "attend", "hq": 64, "hkv": 8, "n_seq": 32, "rows": 1, "kv_min": 500,
         "kv_max": 16384, "page": 64, "spans": 0},
        # Drafted tokens checked in one step: a few rows a sequence.
        {"name": "draft_7b_b8_r5_kv4096", "kind": "attend", "hq": 28, "hkv": 4, "n_seq": 8, "rows": 5, "kv_min": 300,
         "kv_max": 4096, "page": 16, "spans": 0},
        # Follow-up questions with an image each, ragged, on top of what three conversations have cached.
        {"name": "chunk_7b_b3_r777_kv5000", "kind": "attend", "hq": 28, "hkv": 4, "n_seq": 3, "rows": 777, "kv_min": 900,
         "kv_max": 5000, "page": 16, "spans": 1},
        # The last chunk of a long multi-image prompt on the large shapes: the largest call.
        {"name": "chunk_72b_r4096_kv16384", "kind": "attend", "hq": 64, "hkv": 8, "n_seq": 1, "rows": 4096, "kv_min": 16384,
         "kv_max": 16384, "page": 64, "spans": 1},
        # Four generating requests with an adapter each on the qkv linear.
        {"name": "lora_7b_qkv_t4", "kind": "lora", "K": 3584, "N": 4608, "T": 4, "rank": 16, "adapters": 4, "run": 1,
         "spans": 0},
        # A wide batch of generating requests, some without an adapter, on the long side of the MLP.
        {"name": "lora_72b_down_t48", "kind": "lora", "K": 29568, "N": 8192, "T": 48, "rank": 16, "adapters": 12, "run": 1,
         "spans": 0},
        # A step of several prompts, rows of a prompt side by side, at a higher rank.
        {"name": "lora_7b_qkv_t4096_r64", "kind": "lora", "K": 3584, "N": 4608, "T": 4096, "rank": 64, "adapters": 5,
         "run": 900, "spans": 1},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "append", "attend", "attend", "attend", "lora", "lora"))
    hq, hkv = rng.choice(((28, 4), (28, 4), (64, 8), (64, 8), (16, 16), (12, 2), (5, 1)))
    page = rng.choice((16, 32, 64, 128))
    if kind == "norm":
        return {"kind": kind, "hq": hq, "hkv": hkv, "T": _log_int(rng, 1, 16384), "spans": rng.randint(0, 4)}
    if kind == "append":
        rows = _log_int(rng, 1, 2048)
        kv = max(rows, _log_int(rng, 1, 8192))
        return {"kind": kind, "hq": hq, "hkv": hkv, "n_seq": _log_int(rng, 1, max(1, min(64, 4096 // rows))), "rows": rows,
                "kv_min": rng.randint(1, kv), "kv_max": kv, "page": page, "spans": rng.randint(0, 3), "norm": rng.random() < 0.7}
    if kind == "attend":
        form = rng.choice(("decode", "decode", "few", "chunk", "chunk"))
        if form == "chunk":
            rows, kv = _log_int(rng, 16, 3000), _log_int(rng, 64, 12000)
            n_seq = rng.randint(1, max(1, min(6, 3000 // rows)))
        else:
            rows = 1 if form == "decode" else rng.randint(2, 9)
            kv, n_seq = _log_int(rng, 16, 16384), _log_int(rng, 1, 64)
            n_seq = max(1, min(n_seq, 32 * 16384 // kv))
        kv = max(kv, rows)
        return {"kind": kind, "hq": hq, "hkv": hkv, "n_seq": n_seq, "rows": rows, "kv_min": rng.randint(1, kv), "kv_max": kv,
                "page": page, "spans": rng.randint(0, 3) if form == "chunk" else 0}
    K, N = rng.choice((QKV_7B, DOWN_7B, O_7B, GATE_UP_7B, QKV_72B, DOWN_72B))
    T = _log_int(rng, 1, 4096 if N < 20000 else 1024)
    return {"kind": kind, "K": K, "N": N, "T": T, "rank": rng.choice((8, 16, 16, 32, 64, 128)),
            "adapters": rng.randint(1, 16), "run": 1 if T <= 64 else rng.choice((1, T, max(1, T // rng.randint(2, 9)))),
            "spans": 0 if T <= 64 else rng.randint(0, 2)}


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


def _layout(case):
    """Per sequence (rows, cached tokens with them), the first row of each and every row's position."""
    lens = _spread(case["kv_min"], case["kv_max"], case["n_seq"])
    rows = [min(case["rows"] if case["rows"] < 16 else max(1, case["rows"] - 37 * i), n) for i, n in enumerate(lens)]
    start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    pos = np.concatenate([n - r + _perm(r, case["spans"]) for r, n in zip(rows, lens)]).astype(np.int32)
    return rows, lens, start, pos


def _adapter_rows(case):
    """Adapter of every row: runs of equal ones in turn, every fifth run without (-1)."""
    i = np.arange(case["T"]) // case["run"]
    return np.where(i % 5 == 4, -1, (i * 7 + 3) % case["adapters"]).astype(np.int32)


def _randn(gen, *shape, gain=1.0):
    out = torch.empty(shape, dtype=torch.float16, device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - a)
        flat[a:a + n] = (torch.randn(n, dtype=torch.float32, device="cuda", generator=gen) * gain).half()
    return out


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    st = {"case": case, "kind": case["kind"]}
    if case["kind"] == "lora":
        T, K, N, r = case["T"], case["K"], case["N"], case["rank"]
        ids, perm = _adapter_rows(case), _perm(T, case["spans"])
        st.update(T=T, ids=_cuda(ids), perm=_cuda(perm) if case["spans"] else None,
                  rows={int(a): _cuda(np.flatnonzero(ids == a)) for a in np.unique(ids) if a >= 0},
                  x=_randn(gen, T, K), base=_randn(gen, T, N),
                  a=_randn(gen, case["adapters"], r, K, gain=1.0 / math.sqrt(K)),
                  b=_randn(gen, case["adapters"], N, r, gain=1.0 / math.sqrt(r)),
                  scale=0.25 + torch.rand(case["adapters"], device="cuda", generator=gen),
                  y=torch.empty((T, N), dtype=torch.float16, device="cuda"))
        if own:
            from paper_2502_00425_amd import binding as mq
            st["ws"] = torch.empty(mq.lora_workspace_bytes(T, K, r), dtype=torch.uint8, device="cuda")
        return st
    hq, hkv = case["hq"], case["hkv"]
    if case["kind"] == "norm":
        T = case["T"]
        pos = _perm(T, case["spans"])
    else:
        rows, lens, start, pos = _layout(case)
        T, P = int(start[-1]), case["page"]
        need = [-(-n // P) for n in lens]
        n_pages = sum(need) + 3
        pages = torch.randperm(n_pages, device="cuda", generator=gen, dtype=torch.int32)
        table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = pages[at:at + n]
            at += n
        st.update(table=table, start=_cuda(start), rows=rows, lens=lens, page=P,
                  k_pages=_randn(gen, n_pages, hkv, P, D), v_pages=_randn(gen, n_pages, hkv, P, D))
        if own:
            from paper_2502_00425_amd import binding as mq
            st["cache"] = mq.PagedCache(st["k_pages"], st["v_pages"], table)
    st.update(T=T, hq=hq, hkv=hkv, pos=_cuda(pos))
    if case["kind"] == "attend":
        st.update(q=_randn(gen, T, hq * D, gain=1.5), out=torch.empty((T, hq * D), dtype=torch.float16, device="cuda"))
        if own:
            from paper_2502_00425_amd import binding as mq
            st["bounds"] = (max(rows), max(lens))
            st["ws"] = torch.empty(mq.paged_attention_workspace_bytes(T, st["cache"], hq, *st["bounds"]),
                                   dtype=torch.uint8, device="cuda")
        return st
    qkv = _randn(gen, T, (hq + 2 * hkv) * D, gain=2.0)          # the qkv linear's output
    st.update(q=qkv[:, :hq * D], k=qkv[:, hq * D:(hq + hkv) * D], v=qkv[:, (hq + hkv) * D:],
              q_out=torch.empty((T, hq * D), dtype=torch.float16, device="cuda"))
    if case["kind"] == "norm":
        st["k_out"] = torch.empty((T, hkv * D), dtype=torch.float16, device="cuda")
    if case.get("norm", True):
        st.update(wq=(0.5 + torch.rand(D, device="cuda", generator=gen)).half(),
                  wk=(0.5 + torch.rand(D, device="cuda", generator=gen)).half())
    else:
        st.update(wq=None, wk=None)
    return st


# --------------------------------------------------------------------------------- one pass

def _norm_rope(x, heads, w, pos):
    """Plain form of the norm and the rotation: angles in 64 bits, the rest in 32."""
    T = x.shape[0]
    x = x.float().view(T, heads, D)
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w.float()
    theta = BASE ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=x.device) / D)
    angle = pos.double()[:, None] * theta
    c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    even, odd = x[..., 0::2], x[..., 1::2]
    return torch.stack((even * c - odd * s, even * s + odd * c), dim=-1).view(T, heads * D)


def _attend(st):
    """Plain form of the attention: per sequence, some key/value heads at a time."""
    hq, hkv, P = st["hq"], st["hkv"], st["page"]
    G, at = hq // hkv, 0
    for s, (n, length) in enumerate(zip(st["rows"], st["lens"])):
        ids = st["table"][s, :-(-length // P)].long()
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


def _plain(st):
    if st["kind"] == "lora":
        y = st["base"].float()
        for a, rows in st["rows"].items():
            x = st["x"][rows if st["perm"] is None else st["perm"][rows]].float()
            h = torch.matmul(x, st["a"][a].float().t())
            y[rows] += st["scale"][a] * torch.matmul(h, st["b"][a].float().t())
        st["y"].copy_(y)
        return st["y"]
    if st["kind"] == "attend":
        return _attend(st)
    st["q_out"].copy_(_norm_rope(st["q"], st["hq"], st["wq"], st["pos"]))
    k = _norm_rope(st["k"], st["hkv"], st["wk"], st["pos"]).half()
    if st["kind"] == "norm":
        st["k_out"].copy_(k)
        return st["q_out"], st["k_out"]
    row = torch.arange(st["T"], device=k.device)
    seq = torch.searchsorted(st["start"][1:].contiguous(), row, right=True)
    pos = st["pos"].long()
    page, slot = st["table"][seq, pos // st["page"]].long(), pos % st["page"]
    st["k_pages"][page, :, slot] = k.view(-1, st["hkv"], D)
    st["v_pages"][page, :, slot] = st["v"].reshape(-1, st["hkv"], D)
    return st["q_out"], st["k_pages"], st["v_pages"]


def run(st):
    if not own:
        return _plain(st)
    from paper_2502_00425_amd import binding as mq
    if st["kind"] == "lora":
        return mq.lora_apply(st["x"], st["ids"], st["a"], st["b"], st["scale"], st["base"], perm_dev=st["perm"],
                             out=st["y"], workspace=st["ws"])
    if st["kind"] == "attend":
        return mq.paged_attention(st["q"], st["cache"], st["start"], st["pos"], st["hq"], *st["bounds"], out=st["out"],
                                  workspace=st["ws"])
    if st["kind"] == "norm":
        return mq.qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["pos"], st["hq"], st["hkv"], eps=EPS, base=BASE,
                               q_out=st["q_out"], k_out=st["k_out"])
    mq.kv_append(st["q"], st["k"], st["v"], st["cache"], st["start"], st["pos"], st["hq"], st["wq"], st["wk"], eps=EPS,
                 base=BASE, q_out=st["q_out"])
    return st["q_out"], st["k_pages"], st["v_pages"]


def work(case):
    if case["kind"] == "lora":
        T, K, N, r = case["T"], case["K"], case["N"], case["rank"]
        ids = _adapter_rows(case)
        used, rows = len(set(ids[ids >= 0].tolist())), int((ids >= 0).sum())
        return {"bytes": 2 * (rows * K + 2 * T * N + used * r * (K + N)) + 4 * T + 4 * used, "flops": 2 * rows * r * (K + N)}
    hq, hkv = case["hq"], case["hkv"]
    if case["kind"] == "norm":
        return {"bytes": case["T"] * ((hq + hkv) * D * 4 + 4) + 4 * D, "flops": case["T"] * (hq + hkv) * D * 7}
    rows, lens, start, pos = _layout(case)
    T = int(start[-1])
    if case["kind"] == "append":
        return {"bytes": T * ((hq + 2 * hkv) * D * 4 + 8), "flops": T * (hq + hkv) * D * (7 if case["norm"] else 3)}
    return {"bytes": sum(lens) * hkv * D * 4 + T * (hq * D * 4 + 4) + 4 * sum(-(-n // case["page"]) for n in lens),
            "flops": 4 * D * hq * int((pos.astype(np.int64) + 1).sum())}


# ------------------------------------------------------------------------- from the definitions

def _exact_norm_rope(x, heads, w, pos):
    """Row by row block of the definition, as a product with the 2 x 2 rotations in complex numbers."""
    out = torch.empty((x.shape[0], heads * D), dtype=torch.float64, device=x.device)
    j = torch.arange(0, D, 2, dtype=torch.float64, device=x.device)
    theta = torch.exp(j * (-math.log(BASE) / D))
    for a in range(0, x.shape[0], 1024):
        u = x[a:a + 1024].double().reshape(-1, heads, D)
        if w is not None:
            u = u / torch.sqrt(u.square().sum(dim=2, keepdim=True) / D + EPS) * w.double()
        z = torch.view_as_complex(u.reshape(-1, heads, D // 2, 2).contiguous())
        turn = torch.polar(torch.ones_like(theta)[None, :], pos[a:a + 1024, None].double() * theta[None, :])
        out[a:a + 1024] = torch.view_as_real(z * turn[:, None, :]).reshape(-1, heads * D)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "lora":
        y = st["base"].double()
        ids = st["ids"].tolist()
        for i0 in range(0, case["T"], 512):
            part = ids[i0:i0 + 512]
            src = torch.arange(i0, i0 + len(part), device="cuda") if st["perm"] is None else st["perm"][i0:i0 + 512].long()
            x = st["x"][src].double()
            for a in sorted(set(part)):
                if a >= 0:
                    here = torch.tensor([i for i, b in enumerate(part) if b == a], device="cuda")
                    low = x[here] @ st["a"][a].double().t().contiguous()
                    y[i0 + here] += (low @ st["b"][a].double().t().contiguous()) * st["scale"][a].double()
        return y
    if case["kind"] != "attend":
        q = _exact_norm_rope(st["q"], st["hq"], st["wq"], st["pos"])
        k = _exact_norm_rope(st["k"], st["hkv"], st["wk"], st["pos"])
        if case["kind"] == "norm":
            return q, k
        kp, vp = st["k_pages"].double(), st["v_pages"].double()
        at = 0
        for s, n in enumerate(st["rows"]):
            p = st["pos"][at:at + n].long()
            page = st["table"][s].long()[torch.div(p, st["page"], rounding_mode="floor")]
            kp[page, :, p % st["page"]] = k[at:at + n].view(n, -1, D)
            vp[page, :, p % st["page"]] = st["v"][at:at + n].double().reshape(n, -1, D)
            at += n
        return q, kp, vp
    hq, hkv, P, at = st["hq"], st["hkv"], st["page"], 0
    out = torch.empty((st["T"], hq, D), dtype=torch.float64, device="cuda")
    for s, (n, length) in enumerate(zip(st["rows"], st["lens"])):
        slot = torch.arange(length, device="cuda")
        page = st["table"][s].long()[torch.div(slot, P, rounding_mode="floor")]
        for g in range(hkv):
            k, v = st["k_pages"][page, g, slot % P].double(), st["v_pages"][page, g, slot % P].double()
            kt = k.t().contiguous()
            for h in range(g * (hq // hkv), (g + 1) * (hq // hkv)):
                for a in range(at, at + n, 4096):
                    b = min(a + 4096, at + n)
                    z = (st["q"][a:b, h * D:(h + 1) * D].double() @ kt) / math.sqrt(D)
                    z.masked_fill_(slot[None, :] > st["pos"][a:b, None], float("-inf"))
                    out[a:b, h] = torch.exp(z - torch.logsumexp(z, dim=1, keepdim=True)) @ v
        at += n
    return out.reshape(st["T"], hq * D)
