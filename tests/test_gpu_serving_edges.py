"""Edges of the serving calls: state that is carried from step to step, refused steps, numbers at the ends of their ranges."""
import math

import numpy as np
import pytest
import torch

from tests import serving_reference as R
from tests.test_gpu_serving import B, Case, context, ctx, dev, plan_outputs  # noqa: F401  (B and ctx: fixtures)

pytestmark = pytest.mark.gpu


# ---- state from step to step ------------------------------------------------------------------------------------------
def paged_cache(ctx, requests=3, n_pages=16, max_len=96):  # noqa: F811
    from paper_2511_15015_amd.serving import PagedCache
    return PagedCache(ctx, layers=1, requests=requests, max_tokens=64, max_len=max_len, n_pages=n_pages, page_size=16, kv_heads=1, head_dim=64)


def refuse_all(cache, drafts, max_n=None):
    """A verification that accepts nothing (p is 0 at every token); drafts: how many each request brings."""
    requests, n = len(drafts), sum(drafts)
    max_n = max(drafts) if max_n is None else max_n
    tokens, accepted = dev(np.full((requests, max_n + 1), -7)), dev(np.full(requests, -7))
    p, u = torch.zeros((n + requests, 8), device="cuda"), torch.full((n + requests,), 0.5, device="cuda")
    cache.verify(p, None, dev(np.zeros(n)), dev(np.concatenate([[0], np.cumsum(drafts)])), max_n, u[:n], u[n:], tokens, accepted)
    return tokens, accepted


def plan_of(cache, new, state, drops):
    """cache.plan against the reference; -> its state"""
    T = sum(max(n, 0) for n in new)
    want = R.plan(cache.page_size, T, cache.free_list.numel(), np.array(new), state["lens"], np.array(drops), int(state["free"][0]),
                  state["free_list"], state["table"])
    cache.plan(dev(new), T)
    torch.cuda.synchronize()
    for name in ("lens", "free", "free_list", "table", "q_offsets", "status"):
        assert np.array_equal(getattr(cache, name).cpu().numpy(), want[name]), (name, getattr(cache, name), want[name])
    assert np.array_equal(cache.slots[:T].cpu().numpy(), want["slots"]) and np.array_equal(cache.positions[:T].cpu().numpy(), want["positions"])
    return want


def state_of(cache):
    return {k: getattr(cache, k).cpu().numpy().astype(int) for k in ("lens", "free", "free_list", "table")}


def test_dropped_tokens_are_taken_back_once(ctx):  # noqa: F811
    """Steps without a verification behind one that left drops: each of them sees the drops of the verification before it, once."""
    c = paged_cache(ctx)
    s = plan_of(c, [18, 5, 20], state_of(c), [0, 0, 0])
    refuse_all(c, [2, 0, 3])
    assert c.drops.tolist() == [2, 0, 3]
    s = plan_of(c, [1, 1, 0], s, [2, 0, 3])
    assert c.drops.tolist() == [0, 0, 0]
    s = plan_of(c, [1, 1, 1], s, [0, 0, 0])
    s = plan_of(c, [0, 0, 0], s, [0, 0, 0])
    assert c.lens.tolist() == [18, 7, 18]


def test_a_place_is_taken_again_after_a_request_that_ended_with_drops(ctx):  # noqa: F811
    c = paged_cache(ctx)
    s = plan_of(c, [18, 5, 20], state_of(c), [0, 0, 0])
    refuse_all(c, [1, 3, 0])
    s = plan_of(c, [-1, -1, 1], s, [1, 3, 0])
    s = plan_of(c, [5, 2, 1], s, [0, 0, 0])
    assert c.status.tolist()[2:] == [0, 0] and c.lens.tolist() == [5, 2, 22]


def test_drops_are_kept_by_a_step_that_is_refused(ctx):  # noqa: F811
    c = paged_cache(ctx, requests=2, n_pages=4)
    s = plan_of(c, [20, 32], state_of(c), [0, 0])
    refuse_all(c, [2, 0])
    s = plan_of(c, [1, 1], s, [2, 0])                            # a page is missing
    assert c.status.tolist()[2] == 1 and c.drops.tolist() == [2, 0]
    s = plan_of(c, [1, -1], s, [2, 0])
    assert c.lens.tolist() == [19, 0] and c.drops.tolist() == [0, 0]


def test_drops_of_a_plan_with_outputs_of_its_own_stay(ctx):  # noqa: F811
    """dx_pages_plan reads its drops (several caches may share them, a step may be planned twice)."""
    o, fl, tb = plan_outputs(1, 3), dev(np.arange(4)), dev([[3, -1]])
    new, lens, drops, free = dev([3]), dev([9]), dev([2]), dev([3])
    for _ in range(2):
        ctx.dx_pages_plan(new, lens, drops, free, fl, tb, 16, o["lens"], o["free"], o["q_offsets"], o["slots"], o["positions"], o["status"])
        assert o["lens"].tolist() == [10] and drops.tolist() == [2] and o["slots"].tolist() == [55, 56, 57]


def test_drops_in_replays_of_a_graph(B):  # noqa: F811
    """A captured step whose verification leaves drops for the next replay's plan, beside eager steps without a verification."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = paged_cache(context(B, stream.cuda_stream), max_len=96, n_pages=30)
        new, drafts, V = dev([0, 0, 0]), 3, 8
        p, u = torch.zeros((3 * drafts + 3, V), device="cuda"), torch.full((3 * drafts + 3,), 0.5, device="cuda")
        offsets, draft = dev(np.arange(4) * drafts), dev(np.zeros(3 * drafts))
        tokens, accepted = dev(np.zeros((3, drafts + 1))), dev(np.zeros(3))

        def step():
            c.plan(new, 12)
            c.verify(p, None, draft, offsets, drafts, u[:9], u[9:], tokens, accepted)

        def start():
            for t in (c.lens, c.drops):
                t.zero_()
            c.free.fill_(30)
            c.free_list.copy_(torch.arange(30))

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        start()
        with torch.cuda.graph(g, stream=stream):
            step()
        rng = np.random.default_rng(2)
        start()
        lens, drops = np.zeros(3, int), np.zeros(3, int)
        for i in range(12):
            new.copy_(dev([4, 4, 4]))
            good = [int(x) for x in rng.integers(0, drafts + 1, 3)]          # drafts to accept
            p.zero_()
            for b in range(3):
                p[b * (drafts + 1):b * (drafts + 1) + good[b], 0] = 1
            g.replay()
            torch.cuda.synchronize()
            lens, drops = lens - drops + 4, drafts - np.array(good)
            assert c.status.tolist()[2:] == [0, 0] and c.lens.tolist() == lens.tolist() and c.drops.tolist() == drops.tolist()
            if i % 3 == 1:                                                   # a chunk with nothing to judge
                n = [int(x) for x in rng.integers(0, 4, 3)]
                c.plan(dev(n), sum(n))
                torch.cuda.synchronize()
                lens, drops = lens - drops + n, drops * 0
                assert c.lens.tolist() == lens.tolist() and c.drops.tolist() == [0, 0, 0]
        c.ctx.close()


def test_refusals_of_planning_in_place(B, ctx):  # noqa: F811
    p = dev(np.zeros(64)).data_ptr()

    def plan(n=1, T=1, P=16, n_pages=4, stride=2, new=p, lens=p, drops=p, free=p, status=p):
        return ctx.lib.dx_pages_plan_in_place(ctx.h, n, T, P, n_pages, stride, new, lens, drops, free, p, p, p, p, p, status)

    for kw, word in (({"n": 1501}, "B="), ({"n": -1}, "B="), ({"T": -1}, "T="), ({"P": 8}, "page_size"), ({"n_pages": 0}, "n_pages"), ({"stride": 0}, "table_stride"),
                     ({"n_pages": 1 << 27}, "n_pages"), ({"new": None}, "null"), ({"lens": None}, "null"), ({"free": None}, "null"), ({"status": None}, "null")):
        assert plan(**kw) == B.DX_ERR_INVALID
        text = ctx.lib.dx_last_error(ctx.h).decode()
        assert text.startswith("dx_pages_plan_in_place") and word in text, text


def test_a_refused_step_leaves_drops_and_verdicts_of_the_step_before(ctx):  # noqa: F811
    """Drops are waiting, a step lacks pages and goes through attention and verification all the same, a request ends, the step is
    taken again: lengths and pages as if it had not been tried."""
    ends = []
    for tried in (False, True):
        c = paged_cache(ctx, requests=2, n_pages=4)
        s = plan_of(c, [20, 32], state_of(c), [0, 0])
        s = plan_of(c, [3, 0], s, [0, 0])
        refuse_all(c, [2, 0])
        if tried:
            s = plan_of(c, [3, 1], s, [2, 0])
            assert c.status.tolist()[2] == 1
            q, out = torch.randn((4, 1, 64), device="cuda").to(torch.bfloat16), torch.full((4, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
            k = c.k.clone()
            c.write(0, q, q)
            c.attend(0, q, out, 3, 0.1)
            assert (out == 7).all() and torch.equal(k, c.k)
            tokens, accepted = refuse_all(c, [1, 0])
            assert c.drops.tolist() == [2, 0] and accepted.tolist() == [0, 0] and (tokens == -1).all()
        s = plan_of(c, [3, -1], s, [2, 0])
        tokens, accepted = refuse_all(c, [2, 0])
        assert c.drops.tolist() == [2, 0] and (tokens[:, 0] >= 0).all()
        s = plan_of(c, [1, 0], s, [2, 0])
        ends.append({k: v.tolist() for k, v in state_of(c).items()})
    assert ends[0]["lens"] == [23, 0] and ends[0] == ends[1]


def test_verification_behind_an_accepted_plan(ctx):  # noqa: F811
    """dx_draft_verify_planned and dx_draft_verify say the same where the step was accepted; what is refused writes nothing else."""
    rng = np.random.default_rng(7)
    ns, V = [3, 0, 2, 4], 9001
    n, rows = sum(ns), sum(ns) + len(ns)
    p, q = (torch.softmax(3 * torch.from_numpy(rng.standard_normal((x, V)).astype(np.float32)).cuda(), 1) for x in (rows, n))
    draft, offsets, u = dev(rng.integers(0, V, n)), dev(np.concatenate([[0], np.cumsum(ns)])), torch.rand(rows, device="cuda")
    for status in ([5, 6, 0, 0], [0, 0, 1, 0], [0, 0, 0, 2], [5, 6, 0, 0]):
        outs = []
        for call in (ctx.dx_draft_verify, lambda *a: ctx.dx_draft_verify_planned(dev(status), *a)):
            o = [dev(np.full(s, -7)) for s in ((4, 5), 4, 4)]
            call(p, q, draft, offsets, 4, u[:n], u[n:], *o)
            outs.append([t.tolist() for t in o])
        if status[2:] == [0, 0]:
            assert outs[0] == outs[1]
        else:
            assert outs[1] == [[[-1] * 5] * 4, [0] * 4, [-7] * 4]


def test_refusals_of_verification_behind_a_plan(B, ctx):  # noqa: F811
    p, f = dev(np.zeros(64)).data_ptr(), torch.zeros(64, device="cuda").data_ptr()

    def verify(status=p, n=1, drafts=1, most=1, V=8, pp=f, draft=p):
        return ctx.lib.dx_draft_verify_planned(ctx.h, status, pp, f, draft, p, n, drafts, most, V, f, f, p, p, None)

    for kw, word in (({"status": None}, "status"), ({"n": -1}, "B="), ({"V": 0}, "V="), ({"most": 256}, "max_n"), ({"drafts": 2}, "n_drafts"),
                     ({"pp": None}, "null"), ({"draft": None}, "null")):
        assert verify(**kw) == B.DX_ERR_INVALID
        text = ctx.lib.dx_last_error(ctx.h).decode()
        assert text.startswith("dx_draft_verify_planned") and word in text, text


def test_drafts_beyond_the_most_are_dropped_too(ctx):  # noqa: F811
    """The step has appended every draft: those behind the first max_n are not judged, and the next plan takes them back."""
    c = paged_cache(ctx)
    s = plan_of(c, [18, 5, 20], state_of(c), [0, 0, 0])
    tokens, accepted = refuse_all(c, [4, 1, 1], max_n=2)             # all refused
    assert accepted.tolist() == [0, 0, 0] and c.drops.tolist() == [4, 1, 1]
    s = plan_of(c, [5, 1, 1], s, [4, 1, 1])
    p, u = torch.ones((7, 8), device="cuda"), torch.full((7,), 0.5, device="cuda")
    tokens, accepted = dev(np.zeros((3, 3))), dev(np.zeros(3))
    c.verify(p, None, dev([1, 2, 3, 4]), dev([0, 4, 4, 4]), 2, u[:4], u[4:], tokens, accepted)   # all that are judged accepted
    assert accepted.tolist() == [2, 0, 0] and tokens[0, :2].tolist() == [1, 2] and c.drops.tolist() == [2, 0, 0]
    plan_of(c, [1, 0, 0], s, [2, 0, 0])


@pytest.mark.parametrize("page", [-1, -(1 << 27), 40, 1 << 27, (1 << 27) + 3, 1 << 28, 2 ** 31 - 1])
def test_plan_gives_no_slot_in_a_page_that_is_none(ctx, page):  # noqa: F811
    """A table entry that the step keeps, or a free page, that is no page of the cache: its tokens get no slot, and no one else's."""
    for where in ("kept", "free"):
        o, fl, tb = plan_outputs(2, 9), dev(np.arange(40)), dev([[7, -1], [8, -1]])
        if where == "kept":
            tb[0, 0] = page
        else:
            fl[39] = page                                       # the first one taken
        new, lens = dev([5, 4]), dev([9, 16] if where == "kept" else [16, 9])
        ctx.dx_pages_plan(new, lens, None, dev([40]), fl, tb, 16, o["lens"], o["free"], o["q_offsets"], o["slots"], o["positions"], o["status"])
        fine = [39 * 16 + i for i in range(4)] if where == "kept" else [8 * 16 + 9 + i for i in range(4)]
        assert o["status"].tolist() == [1, 0, 0, 0] and o["slots"].tolist() == [-1] * 5 + fine
        assert o["positions"].tolist() == ([9, 10, 11, 12, 13, 16, 17, 18, 19] if where == "kept" else [16, 17, 18, 19, 20, 9, 10, 11, 12])


# ---- numbers at the ends of their ranges ------------------------------------------------------------------------------
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 3, 1 << 30])
def test_attention_window_of_any_size(B, ctx, window):  # noqa: F811
    """A window that is no window, where the first tokens of a request have no keys (their positions are below zero)."""
    for new in ([8, 1], [90, 3]):
        for fmt in ("bf16", "fp8"):
            c = Case(B, 8, 2, 64, 16, fmt, [100, 40], new, seed=1)
            c.lens[0] = new[0] - 5
            got = c.run(ctx, window)
            c.check(got, window)
            assert torch.isinf(got[1][:5]).all() and torch.isfinite(got[1][5:]).all()


def far_scores(B, fmt, D, new, top, alike):  # noqa: F811
    """Scores that are exact in fp32 and of the size of `top` (all alike, or key 0 alone far above the others), and the bounds for them:
    nothing but probabilities of equal keys or of one key enters, whatever the scores' size."""
    P = 16
    c = Case(B, 4, 1, D, P, fmt, [new + 2], [new], seed=D + new)
    half = 2.0 ** (math.frexp(abs(top))[1] // 2)
    if fmt == "fp8":
        c.ks.fill_(half)
        code, k = 0x3F, 1.875 * half                             # (1.875 in e4m3)
        low = 0x37 if top > 0 else 0x47                          # half of it, double
        raw = c.ck
    else:
        code, k = 255 / 128 * half, 255 / 128 * half
        low = code / 2 if top > 0 else code * 2
        raw = c.ck.view(torch.bfloat16)
    real = raw != 127 if fmt == "fp8" else ~torch.isnan(raw)
    raw[real] = code if alike else low
    c.k = torch.full_like(c.k, k if alike else k / 2 if top > 0 else k * 2)
    page = int(c.table[0, 0])
    raw[page, :, :, 0], c.k[page * P] = code, k                  # key 0
    c.q[:] = 2.0 ** math.frexp(abs(top) / half)[1] / D * math.copysign(1, top) / 4
    c.scale = 1.0
    ref = R.attention(c.q.double(), c.k, c.v, c.table, c.q_offsets, c.lens, c.P, c.n_pages, c.scale, 0)
    b_out, b_lse = R.attention_bounds(*ref[:3], torch.zeros_like(ref[3]), ref[4], D)
    return c, ref, b_out, b_lse


def check_far_scores(ctx, c, ref, b_out, b_lse):  # noqa: F811
    out, lse = c.run(ctx)
    assert torch.isfinite(lse).all() and torch.isfinite(out).all()
    over = ((out.double() - ref[0]).abs() / b_out).max().item(), ((lse.double() - ref[1]).abs() / b_lse).max().item()
    assert max(over) <= 1, over


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_scores_far_from_zero(B, ctx, fmt, D, new):  # noqa: F811
    """Beyond 2^31 half a unit in the last place of a score is more than the exponents there are."""
    for top in (2.0 ** 20, 2.0 ** 30, 2.0 ** 35, 2.0 ** 60, 2.0 ** 120):
        for sign in (1, -1):
            for alike in (True, False):
                print("far", fmt, D, new, top * sign, alike, flush=True)
                check_far_scores(ctx, *far_scores(B, fmt, D, new, top * sign, alike))


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_scores_near_the_lowest_number(B, ctx, D, new):  # noqa: F811
    """Every score is -1.98 * 2^126, -2.4e38 in base 2: a number still."""
    case = far_scores(B, "bf16", D, new, -1.99 * 2.0 ** 127, True)
    assert -2.0 ** 127 < case[1][1].min() <= case[1][1].max() < -1.9 * 2.0 ** 126
    check_far_scores(ctx, *case)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("heads,kv,D", [(8, 8, 64), (24, 8, 64), (32, 4, 128), (6, 1, 256)])
def test_attention_values_that_are_no_numbers_reach_the_rows_that_see_them(B, ctx, fmt, heads, kv, D):  # noqa: F811
    """NaN and infinities in values of the new tokens (and under a window of old ones): a row that does not see such a token is as
    without it, one that does gets what the sum gives, in that channel and no other."""
    P = 16
    steps = [([150, 40], [3, 6], 0), ([333, 20], [61, 1], 0), ([300], [300], 0), ([700, 90], [130, 5], 100), ([500], [70], 33)]
    steps += [([60, 33] * 40, [5, 1] * 40, 0), ([60, 33] * 35 + [400], [5, 2] * 35 + [400], 0)]      # more requests than a wavefront has lanes
    if D == 128:
        steps.append(([4070], [4070], 0))                        # several whole tiles to a block
    for lens, new, window in steps:
        c = Case(B, heads, kv, D, P, fmt, lens, new, seed=heads + lens[0])
        rng = np.random.default_rng(lens[0])
        odd = torch.zeros_like(c.v)                              # what is no number, by slot, head and channel
        for b, n in enumerate(lens):
            first = max(n - new[b] - (window or 1), 0)
            for j in rng.choice(np.arange(first, n), min(7, n - first), replace=False):
                slot, h, d = int(c.table[b, j // P]) * P + int(j) % P, int(rng.integers(kv)), int(rng.integers(D))
                what, bits = [(math.inf, 0x7F80), (-math.inf, 0xFF80 - 65536), (math.nan, 0x7FC1)][int(rng.integers(3))]
                if fmt == "fp8":
                    what, bits = math.nan, int(rng.choice([127, 255]))
                odd[slot, h, d] = what
                c.cv[slot // P, h, slot % P // c.X, d, slot % c.X] = bits
                c.v[slot, h, d] = 0
        print("no numbers", fmt, heads, kv, D, lens, new, window, flush=True)
        out, lse = c.run(ctx, window)
        ref = R.attention(c.q.double(), c.k, c.v, c.table, c.q_offsets, c.lens, P, c.n_pages, c.scale, window)
        b_out, b_lse = R.attention_bounds(*ref, D)
        want = ref[0].clone()
        for b, n in enumerate(lens):
            j = np.arange(n)
            slot = torch.from_numpy(c.table[b, j // P] * P + j % P).cuda()
            pos = torch.arange(n - new[b], n, device="cuda")[:, None]
            jt = torch.from_numpy(j).cuda()
            see = ((jt <= pos) & ((jt > pos - window) if window else (jt >= 0))).double()
            for h in range(heads):
                x = odd[slot, h // (heads // kv)]
                up, down = see @ (~(x < 0) & (x != 0)).double(), see @ (~(x > 0) & (x != 0)).double()      # (NaN: both)
                rows = want[c.q_offsets[b]:c.q_offsets[b + 1], h]
                rows[(up > 0) & (down == 0)] = math.inf
                rows[(up == 0) & (down > 0)] = -math.inf
                rows[(up > 0) & (down > 0)] = math.nan
        fine = torch.isfinite(want)
        assert not fine.all() and torch.isfinite(lse).all()
        assert ((out.double() - want).abs() <= b_out)[fine].all(), ((out.double() - want).abs() / b_out)[fine].max()
        assert torch.equal(torch.nan_to_num(out.double(), 7.0, 8.0, 9.0)[~fine], torch.nan_to_num(want, 7.0, 8.0, 9.0)[~fine])
        assert ((lse.double() - ref[1]).abs() <= b_lse).all()


# ---- a chunk beside more requests than a wavefront has lanes -----------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("heads,kv,D", [(8, 2, 64), (16, 4, 128), (6, 1, 256)])
@pytest.mark.parametrize("n", [65, 257, 1000])
def test_attention_chunks_beside_many_requests(B, ctx, fmt, heads, kv, D, n):  # noqa: F811
    """Chunks of several tiles at the first, a middle and the last request, requests without tokens between."""
    rng = np.random.default_rng(n + D)
    for chunks, window in (({0: 301}, 0), ({n // 2: 133}, 50), ({n - 1: 402}, 0), ({0: 77, n // 2: 250, n - 1: 129}, 0)):
        new = [chunks.get(b, int(rng.integers(0, 3))) for b in range(n)]
        lens = [max(x, 1) + int(rng.integers(0, 60)) for x in new]
        for b in rng.choice(n, n // 10, replace=False):
            if b not in chunks:
                new[b], lens[b] = 0, int(rng.integers(0, 2)) * 9
        print("chunks", fmt, heads, kv, D, n, chunks, window, flush=True)
        c = Case(B, heads, kv, D, 16, fmt, lens, new, seed=n)
        c.check(c.run(ctx, window), window)


@pytest.mark.parametrize("live", ["first", "last", "spread"])
def test_attention_places_without_a_request_cost_next_to_nothing(B, ctx, live):  # noqa: F811
    """4 live requests in 1024 places against the same 4 alone, which is bound by latency: no block may walk over the others.  (Four
    times as long is allowed; a walk takes twenty times as long.)"""
    n = 1024
    at = {"first": [0, 1, 2, 3], "last": [n - 4, n - 3, n - 2, n - 1], "spread": [5, 300, 301, 900]}[live]
    times = []
    for places in (4, n):
        where = range(4) if places == 4 else at
        lens, new = [0] * places, [0] * places
        for b in where:
            lens[b], new[b] = 400, 1
        c = Case(B, 32, 4, 128, 16, "bf16", lens, new, seed=1)
        c.check(c.run(ctx))
        args = c.cache, c.q, dev(c.q_offsets), dev(c.lens), dev(c.table), 1, c.scale, 0, torch.empty_like(c.q)
        took = []
        for _ in range(7):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            for _ in range(20):
                ctx.dx_paged_attention(*args)
            end.record()
            torch.cuda.synchronize()
            took.append(start.elapsed_time(end) / 20)
        times.append(sorted(took)[3])
    print("places", live, times, flush=True)
    assert times[1] <= 4 * times[0], times


