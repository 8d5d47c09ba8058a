"""A serving loop around attention layers as a program runs it: the step's plan, norm and rotation with the write to the pages, attention over
a shared prefix, logits and the next token, prefill and tokens, eagerly and from one captured graph, against the oracle."""
import numpy as np
import pytest

from oracle import mquant_oracle as orc
from serving import D, attention_bound

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
HQ, HKV, PAGE, V = 8, 2, 16, 1003


@pytest.fixture(scope="module")
def mq():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2502_00425_amd import binding
    return binding


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Loop:
    """Device state and the step.  Sequences 0 .. 3 begin with the same `prefix` tokens (one group), 4 and 5 with none; a row's embedding is
    that of its token and what follows is a single attention layer whose output is multiplied with the vocabulary."""

    def __init__(self, mq, n_seq, prefix, n_pages, T, rot):
        rng = np.random.default_rng(1)
        self.mq, self.T, self.rot, self.n_seq, self.prefix = mq, T, rot, n_seq, prefix
        self.embed = dev(rng.standard_normal((V, (HQ + 2 * HKV) * D)).astype(np.float16))
        self.head = dev((rng.standard_normal((HQ * D, V)) * 0.2).astype(np.float16))
        self.wk = dev(rng.uniform(0.5, 1.5, D).astype(np.float16))
        self.kp = torch.full((n_pages, HKV, PAGE, D), float("nan"), dtype=torch.float16, device="cuda")
        self.vp = torch.full_like(self.kp, float("inf"))
        whole = prefix // PAGE
        table = np.full((n_seq, 12), -3, dtype=np.int32)
        order = rng.permutation(n_pages).astype(np.int32)
        table[:4, :whole] = order[:whole]
        self.table = dev(table)
        ring = np.roll(np.concatenate([order[whole:], np.full(whole, -9, np.int32)]), 5)
        self.ring, self.state = dev(ring), dev(np.array([5, n_pages - whole], dtype=np.int32))
        self.length = dev(np.zeros(n_seq, dtype=np.int32))
        self.shared = dev(np.where(np.arange(n_seq) < 4, whole, 0).astype(np.int32))
        self.group_start, self.prefixes = dev(np.array([0, 4], np.int32)), dev(np.array([prefix], np.int32))
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.rows, self.tokens, self.u = i32(n_seq), i32(T), torch.zeros(T, dtype=torch.float32, device="cuda")
        self.start, self.pos, self.slots = i32(n_seq + 1), i32(T), torch.zeros(T, dtype=torch.int64, device="cuda")
        self.cache = mq.PagedCache(self.kp, self.vp, self.table)
        self.out = torch.zeros((T, HQ * D), dtype=torch.float16, device="cuda")
        self.next, self.logprob = i32(T), torch.zeros(T, dtype=torch.float32, device="cuda")
        self.settings = [dev(np.resize(np.array(c, d), T)) for c, d in zip(
            zip((1.0, 0, 1.0, 0.0), (0.8, 40, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.2, 0, 0.7, 0.01)), (np.float32, np.int32, np.float32, np.float32))]
        self.ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
        self.qkv = torch.zeros((T, (HQ + 2 * HKV) * D), dtype=torch.float16, device="cuda")
        self.logits = torch.zeros((T, V), dtype=torch.float16, device="cuda")

    def step(self):
        """Entries of the library and the products around them, on the current stream; nothing is read back."""
        mq = self.mq
        mq.step_plan(self.length, self.rows, self.table, PAGE, self.ring, self.state, self.T, self.shared, None, self.length, self.state,
                     self.start, self.pos, self.slots)
        torch.index_select(self.embed, 0, self.tokens, out=self.qkv)
        q, k, v = self.qkv[:, :HQ * D], self.qkv[:, HQ * D:(HQ + HKV) * D], self.qkv[:, (HQ + HKV) * D:]
        mq.rotary_append(q, k, v, self.cache, self.start, self.pos, self.rot, HQ, None, self.wk, q_out=q)
        mq.paged_attention_shared(q, self.cache, self.start, self.pos, self.group_start, self.prefixes, HQ, out=self.out, workspace=self.ws)
        torch.mm(self.out, self.head, out=self.logits)
        mq.sample(self.logits, *self.settings, self.u, self.next, self.logprob, self.ws)


def test_prefill_and_tokens_from_one_graph(mq):
    """The prefix by a sequence of its own, then steps of all: prompts, tokens, one that ends, and one that begins in its pages.  Every step is
    run eagerly on one loop and replayed from a graph on another with the same state: the same bits; and against the oracle: plan equal,
    pages and attention within their bounds, tokens equal from the logits that were computed."""
    rng = np.random.default_rng(5)
    n_seq, prefix, T, n_pages = 6, 37, 48, 40
    rot = mq.Rotary(64, base=5e5, halves=True, scaling="turns", factor=4.0, trained=32.0, low=0.5, high=4.0, scale=1.25)
    freq = orc.rotary_frequencies(64, 5e5, "turns", 4.0, 32.0, 0.5, 4.0)
    loops = [Loop(mq, n_seq, prefix, n_pages, T, rot) for _ in range(2)]
    whole = prefix // PAGE
    # the shared pages are filled through a table of one sequence; what the prefix has in a page of its own, each sequence writes itself
    shared_tokens = rng.integers(0, V, whole * PAGE)
    for loop in loops:
        x = loop.embed[dev(shared_tokens)]
        one = mq.PagedCache(loop.kp, loop.vp, loop.table[:1].contiguous())
        mq.rotary_append(x[:, :HQ * D], x[:, HQ * D:(HQ + HKV) * D], x[:, (HQ + HKV) * D:], one, dev(np.array([0, whole * PAGE], np.int32)),
                         dev(np.arange(whole * PAGE, dtype=np.int32)), rot, HQ, None, loop.wk)
        loop.length.copy_(dev(np.where(np.arange(n_seq) < 4, whole * PAGE, 0).astype(np.int32)))
    eager, replayed = loops
    for t, f in zip((eager.kp, eager.vp), (replayed.kp, replayed.vp)):
        assert torch.equal(t.view(torch.int16), f.view(torch.int16))
    same_rest = rng.integers(0, V, prefix % PAGE)
    prompts = [np.concatenate([same_rest, rng.integers(0, V, n)]) for n in (3, 1, 2, 4)] + [rng.integers(0, V, n) for n in (5, 7)]
    steps = [np.array([len(p) for p in prompts], np.int32)] + [np.ones(n_seq, np.int32) for _ in range(3)] + [
        np.array([1, -1, 1, 0, 1, -1], np.int32), np.array([1, 0, 1, 1, 1, 9], np.int32), np.array([1, 0, 1, 1, 1, 1], np.int32),
        np.array([1, 0, 1, 1, 30, 20], np.int32), np.array([2, 2 + prefix % PAGE, 2, 2, 2, 2], np.int32)]
    graph, last = None, [0] * n_seq
    for number, rows in enumerate(steps):
        tokens = np.zeros(T, np.int32)
        at = 0
        for s, n in enumerate(np.maximum(rows, 0)):
            if at + n > T:
                break
            new = prompts[s] if number == 0 else rng.integers(0, V, n) if n > 1 else [last[s]]
            if number == len(steps) - 1 and s == 1:            # begins behind the shared pages again, with what the prefix has in a page of its own
                new = np.concatenate([same_rest, new[:2]])
            tokens[at:at + n] = new
            at += n
        u = rng.random(T, dtype=np.float32)
        if number == len(steps) - 1:
            eager.length[1] = replayed.length[1] = whole * PAGE
        before = [x.cpu().numpy().copy() for x in (eager.length, eager.table, eager.ring, eager.state)]
        for loop in loops:
            loop.rows.copy_(dev(rows)), loop.tokens.copy_(dev(tokens)), loop.u.copy_(dev(u))
        eager.step()
        if graph is None:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                for _ in range(2):                                     # the library product's own scratch
                    torch.mm(replayed.out, replayed.head, out=replayed.logits)
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                replayed.step()
        graph.replay()
        torch.cuda.synchronize()
        # ---- the plan
        want = orc.step_plan(before[0], rows, before[1], PAGE, before[2], before[3], T, eager.shared.cpu().numpy(), None)
        start, pos = (x.cpu().numpy() for x in (eager.start, eager.pos))
        for got, ref in zip((eager.start, eager.pos, eager.slots, eager.length, eager.state, eager.table, eager.ring), (*want, before[1], before[2])):
            assert np.array_equal(got.cpu().numpy(), ref), number
        n = int(start[-1])
        assert n > 0 and (number != len(steps) - 2 or n < rows.clip(0).sum())          # the last but one asks for more than a step has
        for name in ("length", "state", "table", "ring", "start", "pos", "slots", "kp", "vp"):
            a, b = getattr(eager, name), getattr(replayed, name)
            assert torch.equal(a.view(torch.int16) if a.is_floating_point() else a, b.view(torch.int16) if b.is_floating_point() else b), (number, name)
        for name in ("out", "next", "logprob"):
            assert torch.equal(getattr(eager, name)[:n], getattr(replayed, name)[:n]), (number, name)
        # ---- pages: 24 roundings of fp32 (2^-19 of the pair) and one of fp16
        x = eager.embed.cpu().numpy()[tokens[:n]]
        k64 = orc.rotary_f64(x[:, HQ * D:(HQ + HKV) * D], eager.wk.cpu().numpy(), pos[:n], HKV, freq, True, scale=1.25)
        kp, vp, slots, table = (t.cpu().numpy() for t in (eager.kp, eager.vp, eager.slots, eager.table))
        got = kp[slots[:n] // PAGE, :, slots[:n] % PAGE].reshape(n, -1).astype(np.float64)
        h = np.abs(k64).reshape(n, HKV, D)
        pair = h.copy()
        pair[:, :, :32] = pair[:, :, 32:64] = h[:, :, :32] + h[:, :, 32:64]
        assert (np.abs(got - k64) <= 2.0 ** -11 * np.abs(k64) + 2.0 ** -25 + 2.0 ** -19 * np.sqrt(2) * pair.reshape(n, -1)).all(), number
        assert np.array_equal(vp[slots[:n] // PAGE, :, slots[:n] % PAGE].reshape(n, -1), x[:, (HQ + HKV) * D:])
        # ---- attention, from the pages and queries as they are
        q = eager.qkv[:, :HQ * D].cpu().numpy()
        st = {"T": T, "hq": HQ, "hkv": HKV, "q": q, "kp": kp, "vp": vp, "table": table, "start": start, "pos": pos}
        ref = orc.paged_attention_f64(q, kp, vp, table, start, pos, HQ)
        err, tol = np.abs(eager.out.cpu().numpy().astype(np.float64) - ref)[:n], attention_bound(st, ref)[:n]
        assert (err <= tol).all(), (number, (err - tol).max())
        # ---- tokens, from the logits as they are
        logits, drawn = eager.logits.cpu().numpy().astype(np.float64), eager.next.cpu().numpy()
        cols = [c.cpu().numpy() for c in eager.settings]
        for i in range(n):
            token, _ = orc.sample_f64(logits[i], float(cols[0][i]), int(cols[1][i]), float(cols[2][i]), float(cols[3][i]), float(u[i]))
            assert drawn[i] == token, (number, i)
        for s in range(n_seq):
            if start[s + 1] > start[s]:
                last[s] = int(drawn[start[s + 1] - 1])
