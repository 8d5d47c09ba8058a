"""Attention of sequences that begin with the same tokens, against the fp64 oracle of the attention by itself over every sequence's own
pages, within serving.attention_bound."""
import numpy as np
import pytest

from loop import make_shared
from oracle import mquant_oracle as orc
from serving import D, attention_bound

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mq():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2502_00425_amd import binding
    return binding


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def args_of(mq, st):
    return (dev(st["q"]), mq.PagedCache(dev(st["kp"]), dev(st["vp"]), dev(st["table"])), dev(st["start"]), dev(st["pos"]),
            dev(st["group_start"]), dev(st["prefix"]), st["hq"])


def bounds_of(st):
    rows, behind = 1, 1
    for s, mine in orc.sequence_rows(st["start"], st["T"]):
        if len(mine) == 0:
            continue
        g = np.searchsorted(st["group_start"], s, side="right") - 1
        p = st["prefix"][g] if 0 <= g < len(st["prefix"]) else 0
        rows, behind = max(rows, len(mine)), max(behind, int(st["pos"][mine].max()) + 1 - int(p))
    return rows, int(max([1, *st["prefix"]])), behind


def check(st, out, rows=None, what=""):
    plain = {**st, "table": st["full"]}
    ref = orc.paged_attention_f64(st["q"], st["kp"], st["vp"], st["full"], st["start"], st["pos"], st["hq"], rows=rows)
    mine = ~np.isnan(ref[:, 0])
    got = out.cpu().numpy().astype(np.float64)
    assert np.isfinite(got[mine]).all(), what
    err, tol = np.abs(got - ref)[mine], attention_bound(plain, ref, rows=rows)[mine]
    worst = np.unravel_index((err - tol).argmax(), err.shape)
    assert (err <= tol).all(), f"{what}: {err[worst]:.3e} > {tol[worst]:.3e} at {worst}"


STEPS = {                      # groups, query heads, kv heads, page
    "two_tokens": ([(1, [(1, 2), (1, 2)])], 28, 4, 16),
    "one_sequence": ([(100, [(1, 131)])], 28, 4, 16),
    "decode": ([(1280, [(1, 1290), (1, 1340), (1, 1281), (1, 1300)])], 28, 4, 16),
    "decode_in_a_page": ([(1003, [(1, 1010), (1, 1290), (1, 1004)])], 28, 4, 64),
    "many": ([(300, [(1, 301 + 7 * i) for i in range(40)])], 64, 8, 16),
    "few_queries_each_part": ([(200, [(1, 230), (2, 260)])], 16, 16, 16),
    "drafts": ([(513, [(5, 600), (3, 520), (4, 517)])], 28, 4, 16),
    "questions": ([(700, [(150, 900), (33, 733), (60, 800)])], 28, 4, 16),
    "long_questions": ([(3000, [(40, 3100), (35, 3050)])], 28, 4, 64),
    "many_rows_each": ([(257, [(220, 480), (200, 460), (210, 900)]), (100, [(180, 300), (190, 290)])], 16, 16, 16),
    "mixed_lengths": ([(256, [(1, 300), (100, 400), (2, 258), (0, 256), (1, 2000)])], 7, 1, 32),
    "groups": ([(64, [(1, 70), (1, 90)]), (333, [(3, 400)]), (0, [(1, 30), (2, 5)]), (1000, [(1, 1001), (40, 1100), (1, 1003)])], 12, 2, 16),
    "inside_the_prefix": ([(500, [(1, 500), (3, 260), (1, 1), (2, 503), (40, 480)])], 28, 4, 16),
    "all_inside_the_prefix": ([(500, [(1, 500), (1, 400)])], 28, 4, 16),
    "no_rows": ([(90, [(0, 90), (0, 100)]), (64, [(1, 66), (0, 70), (3, 68)])], 28, 4, 16),
    "empty_group": ([(90, [(1, 95)]), (64, []), (128, [(1, 129), (1, 140)])], 28, 4, 128),
    "borders_of_tiles": ([(p, [(1, p + 1), (2, p + 70)]) for p in (31, 32, 33, 63, 64, 65, 127, 128, 129)], 14, 2, 16),
    "borders_of_tiles_chunks": ([(p, [(40, p + 40), (33, p + 70)]) for p in (31, 32, 33, 63, 64, 65, 127, 128, 129)], 14, 2, 16),
    "long": ([(9000, [(1, 9100), (1, 9001), (1, 12000)])], 28, 4, 64),
    "heads_of_their_own": ([(150, [(1, 160 + i) for i in range(60)])], 8, 8, 16),
}


@pytest.mark.parametrize("name", list(STEPS))
@pytest.mark.parametrize("known", [True, False])
def test_steps(mq, name, known):
    st = make_shared(np.random.default_rng(len(name)), *STEPS[name], before=2, behind=3, spans=[(3, 20)])
    args = args_of(mq, st)
    out = torch.full((st["T"], st["hq"] * D + 4), 3.0, dtype=torch.float16, device="cuda")
    mq.paged_attention_shared(*args, *(bounds_of(st) if known else ()), out=out)
    check(st, out[:, :st["hq"] * D], what=name)
    others = np.setdiff1d(np.arange(st["T"]), np.concatenate([r for _, r in orc.sequence_rows(st["start"], st["T"])]))
    assert (out[others] == 3).all() and (out[:, st["hq"] * D:] == 3).all()       # rows of no sequence stay as they were


@pytest.mark.parametrize("name", ["decode", "drafts", "questions", "mixed_lengths", "groups", "many", "inside_the_prefix"])
def test_bounds_that_the_data_exceed(mq, name):
    st = make_shared(np.random.default_rng(1), *STEPS[name])
    rows, prefix, behind = bounds_of(st)
    for bounds in ((1, 1, 1), (rows, 1, behind), (1, prefix, 1), (rows, prefix, 2 ** 31 - 1), (rows, 2 ** 31 - 1, behind), (10 ** 6, prefix, 7)):
        check(st, mq.paged_attention_shared(*args_of(mq, st), *bounds), what=f"{name} {bounds}")


def test_sequences_of_no_group(mq):
    groups = [(0, [(1, 40)]), (200, [(1, 230), (4, 250)]), (0, [(50, 90), (1, 300)])]
    st = make_shared(np.random.default_rng(2), groups, 28, 4, 16, alone=(1, 1))
    assert st["group_start"].tolist() == [1, 3]
    for bounds in ((), bounds_of(st)):
        check(st, mq.paged_attention_shared(*args_of(mq, st), *bounds))


def test_no_groups_is_the_attention_by_itself(mq):
    st = make_shared(np.random.default_rng(3), [(0, [(1, 200), (60, 90), (3, 1500)])], 28, 4, 16)
    q, cache, start, pos, _, _, hq = args_of(mq, st)
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    check(st, mq.paged_attention_shared(q, cache, start, pos, torch.zeros(1, dtype=torch.int32, device="cuda"), e, hq))
    out = torch.empty((st["T"], hq * D), dtype=torch.float16, device="cuda")
    ws = torch.empty(mq.paged_attention_shared_workspace_bytes(st["T"], cache, 0, hq), dtype=torch.uint8, device="cuda")
    assert mq.lib.mquant_paged_attention_shared(q.data_ptr(), q.stride(0), cache.address, start.data_ptr(), pos.data_ptr(), None, None, 0, out.data_ptr(),
                                                out.stride(0), st["T"], hq, 0, 0, 0, ws.data_ptr(), ws.numel(), None) == mq.OK
    torch.cuda.synchronize()
    check(st, out)


def test_prefixes_out_of_range_and_rows_that_see_nothing(mq):
    rng = np.random.default_rng(4)
    st = make_shared(rng, [(64, [(1, 64), (2, 40)]), (0, [(1, 30)])], 28, 4, 16, poison=False)
    st["pos"][0] = -3
    st["prefix"][1] = -17
    check(st, mq.paged_attention_shared(*args_of(mq, st)))
    # a prefix beyond the table counts as all of it: every sequence is read through the first one's pages
    same = make_shared(rng, [(64, [(1, 64), (2, 64), (1, 60)])], 28, 4, 16, poison=False)
    same["prefix"][0] = 2 ** 31 - 1
    check(same, mq.paged_attention_shared(*args_of(mq, same)))


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), 3e38])
def test_scratch_holds_anything(mq, fill):
    for name in ("decode", "groups", "questions", "inside_the_prefix", "mixed_lengths"):
        st = make_shared(np.random.default_rng(5), *STEPS[name])
        args, bounds = args_of(mq, st), bounds_of(st)
        need = mq.paged_attention_shared_workspace_bytes(st["T"], args[1], len(st["prefix"]), st["hq"], *bounds)
        ws = torch.full((need // 4,), fill, dtype=torch.float32, device="cuda")
        check(st, mq.paged_attention_shared(*args, *bounds, workspace=ws), what=name)


def test_strides_streams_and_repeats(mq):
    st = make_shared(np.random.default_rng(6), *STEPS["groups"])
    wide = torch.full((st["T"], st["hq"] * D + 40), 9.0, dtype=torch.float16, device="cuda")
    q, *rest = args_of(mq, st)
    wide[:, 8:8 + st["hq"] * D] = q
    want = mq.paged_attention_shared(q, *rest)
    mine = torch.from_numpy(np.concatenate([r for _, r in orc.sequence_rows(st["start"], st["T"])])).cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs += [mq.paged_attention_shared(wide[:, 8:8 + st["hq"] * D], *rest) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(o[mine], want[mine]) for o in outs)


def test_two_graphs_that_share_a_workspace(mq):
    """Replayed in turn with other queries and positions between."""
    steps = [make_shared(np.random.default_rng(7 + i), *STEPS[name]) for i, name in enumerate(("decode", "drafts"))]
    args = [args_of(mq, st) for st in steps]
    need = max(mq.paged_attention_shared_workspace_bytes(st["T"], a[1], 1, st["hq"], *bounds_of(st)) for st, a in zip(steps, args))
    ws, graphs, outs = torch.empty(need, dtype=torch.uint8, device="cuda"), [], []
    for st, a in zip(steps, args):
        outs.append(torch.empty((st["T"], st["hq"] * D), dtype=torch.float16, device="cuda"))
        mq.paged_attention_shared(*a, *bounds_of(st), out=outs[-1], workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mq.paged_attention_shared(*a, *bounds_of(st), out=outs[-1], workspace=ws)
        graphs.append(g)
    rng = np.random.default_rng(9)
    for _ in range(3):
        for st, a in zip(steps, args):
            st["q"] = rng.standard_normal(st["q"].shape).astype(np.float16)
            st["pos"] = np.maximum(st["pos"] - rng.integers(0, 3, st["T"]).astype(np.int32), 0)
            a[0].copy_(dev(st["q"])), a[3].copy_(dev(st["pos"]))
        for g in graphs:
            g.replay()
        for st, out in zip(steps, outs):
            check(st, out)


def test_seeded_sweep(mq):
    rng = np.random.default_rng(11)
    for _ in range(25):
        hq, hkv = [(28, 4), (8, 8), (12, 2), (5, 1), (64, 8)][rng.integers(5)]
        groups = []
        for _ in range(rng.integers(1, 4)):
            p = int(rng.integers(0, 900))
            members = []
            for _ in range(rng.integers(1, 6)):
                n = int(rng.choice([0, 1, 1, 2, 7, 30]))
                members.append((n, n + int(rng.integers(0, p + 300))))
            groups.append((p, members))
        st = make_shared(rng, groups, hq, hkv, int(rng.choice([16, 32, 64])))
        if st["T"]:
            check(st, mq.paged_attention_shared(*args_of(mq, st), *(bounds_of(st) if rng.random() < 0.5 else ())), what=str(groups))


def test_routes(mq):
    """Which kernels the groups' rows and the bounds choose."""
    from kernel_trace import kernels
    for name, bounds, want in (("decode", True, ["shared_few_kernel<2>", "shared_combine_kernel"]),
                               ("many", True, ["shared_both_kernel<1>", "shared_combine_kernel"]),
                               ("drafts", True, ["shared_both_kernel<3>", "shared_combine_kernel"]),
                               ("questions", True, ["shared_whole_kernel<2>"]),
                               ("long_questions", True, ["shared_whole_kernel<2>", "paged_combine_kernel<true>"]),
                               ("questions", False, ["shared_both_kernel<3>", "shared_suffix_kernel", "shared_combine_kernel"]),
                               ("mixed_lengths", True, ["shared_both_kernel<3>", "shared_suffix_kernel", "shared_combine_kernel"])):
        st = make_shared(np.random.default_rng(10), *STEPS[name], poison=False)
        args = args_of(mq, st)
        names = kernels(lambda: mq.paged_attention_shared(*args, *(bounds_of(st) if bounds else ())))
        assert [n for n in names if n.startswith(("shared", "paged"))] == want, (name, names)


@pytest.mark.parametrize("name", ["decode_in_a_page", "questions", "many_rows_each"])
def test_pages_beyond_32_bits(mq, name):
    """The same step with its pages at the end of a pool of more than 2^31 values each: the same bits."""
    st = make_shared(np.random.default_rng(21), *STEPS[name])
    args, bounds = args_of(mq, st), bounds_of(st)
    want = mq.paged_attention_shared(*args, *bounds)
    _, hkv, page, _ = st["kp"].shape
    far = (1 << 31) // (hkv * page * D) + 1
    pools = []
    for a in ("kp", "vp"):
        pool = torch.empty((far + len(st[a]), hkv, page, D), dtype=torch.float16, device="cuda")
        pool[far:] = dev(st[a])
        pools.append(pool)
    table = np.where(st["table"] >= 0, st["table"] + far, st["table"]).astype(np.int32)
    cache = mq.PagedCache(*pools, dev(table))
    assert torch.equal(mq.paged_attention_shared(args[0], cache, *args[2:], *bounds), want)
