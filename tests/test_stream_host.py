"""Host side of the stream operators: the pages' book-keeping against the oracle's, the division of a planned step, and
what is refused.  No GPU is touched."""
import numpy as np
import pytest

from oracle import layer as OL
from oracle import stream as OS
from paper_2411_16102_amd import binding, workloads as W
from stream_cases import make_batch


# ---- the oracle against other formulas ---------------------------------------------------
def test_oracle_attention_without_a_limit_is_causal_attention():
    rng = np.random.default_rng(1)
    q, K, V = rng.standard_normal((5, 4, 8)), rng.standard_normal((30, 2, 8)), rng.standard_normal((30, 2, 8))
    out, _ = OS.window_attention(q, K, V, 25, 1000, 0)
    np.testing.assert_allclose(out, OL.attention(q, K, V, 25), atol=1e-13)
    # all of it from sinks
    out, _ = OS.window_attention(q, K, V, 25, 1, 1000)
    np.testing.assert_allclose(out, OL.attention(q, K, V, 25), atol=1e-13)
    # a window of one token: its value
    out, _ = OS.window_attention(q, K, V, 25, 1, 0)
    np.testing.assert_allclose(out[3], V[28].repeat(2, axis=0), atol=1e-13)


@pytest.mark.parametrize("first,window,sinks", [(25, 7, 2), (-3, 4, 1), (0, 1, 0), (12, 30, 14), (40, 5, 33)])
def test_oracle_attention_is_what_every_row_sees(first, window, sinks):
    rng = np.random.default_rng(first + 9)
    n = max(0, first + 6)
    q, K, V = rng.standard_normal((6, 4, 8)), rng.standard_normal((n, 2, 8)), rng.standard_normal((n, 2, 8))
    out, weight = OS.window_attention(q, K, V, first, window, sinks)
    for j in range(6):
        see = [t for t in range(n) if OS.visible(first + j, t, window, sinks)]
        for h in range(4):
            if not see:
                assert not out[j, h].any() and not weight[j, h].any()
                continue
            e = np.exp([K[t, h // 2] @ q[j, h] / 8 ** 0.5 for t in see])
            np.testing.assert_allclose(out[j, h], sum(w * V[t, h // 2] for w, t in zip(e, see)) / e.sum(), atol=1e-13)
            np.testing.assert_allclose(weight[j, h], sum(w * abs(V[t, h // 2]) for w, t in zip(e, see)) / e.sum(), atol=1e-13)


def test_oracle_rope_of_equal_axes_is_rope():
    rng = np.random.default_rng(2)
    v, pos = rng.standard_normal((6, 3, 16)), np.array([0, 1, 5, 100, 7, 3])
    got = OS.rope_axes(v, np.stack([pos] * 3), np.arange(8) % 3, 10000.0)
    np.testing.assert_allclose(got, OL.rope(v, pos, 10000.0), atol=1e-12)


# ---- pages ---------------------------------------------------------------------------------
def _same(p, o):
    ids = sorted(o.seqs)
    start, pages = p.tables(ids)
    assert p.lengths(ids).tolist() == [o.seqs[i][0] for i in ids]
    assert [pages[start[k]:start[k + 1]].tolist() for k in range(len(ids))] == [o.seqs[i][1] for i in ids]
    assert p.stats() == {"free": len(o.free_pages()), "sequences": len(ids)}


@pytest.mark.parametrize("seed", range(8))
def test_pages_follow_the_oracle(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(4, 60))
    p, o = binding.Pages(n), OS.Pages(n)
    for _ in range(60):
        ids = sorted(o.seqs)
        some = [i for i in rng.permutation(ids)[:rng.integers(0, 4)]] if ids else []
        some = [int(i) for i in some]
        what = rng.integers(0, 7)
        if what == 0:
            assert p.open(2).tolist() == o.open(2)
        elif what == 1 and some:
            k = int(rng.integers(0, 3))
            assert p.fork(some, k).tolist() == o.fork(some, k)
        elif what in (2, 3, 4):
            more = rng.integers(0, 40, len(some)).tolist()
            want = o.extend(some, more)
            if want is None:
                with pytest.raises(binding.BlendStepError, match="are free") as e:
                    p.extend(some, more)
                assert e.value.code == -2
            else:
                src, dst = p.extend(some, more)
                assert list(zip(src.tolist(), dst.tolist())) == want
                assert not set(src.tolist()) & set(dst.tolist()) and len(set(dst.tolist())) == len(dst)
        elif what == 5:
            w, s = int(rng.integers(1, 40)), int(rng.integers(0, 20))
            p.trim(some, w, s)
            o.trim(some, w, s)
        elif rng.random() < 0.5:
            p.free(some)
            o.free(some)
        else:
            src, dst, live = p.compact()
            assert (list(zip(src.tolist(), dst.tolist())), live) == o.compact()
        _same(p, o)


def test_pages_refusals_change_nothing():
    p = binding.Pages(4)
    a, b = p.open(2).tolist()
    p.extend([a], 50)
    before = p.tables([a, b])[1].tolist()
    for call, match in ((lambda: p.extend([a, a], 1), "twice"), (lambda: p.extend([7], 1), "no sequence"), (lambda: p.extend([a], -1), "further tokens"),
                        (lambda: p.extend([b], 17), "are free"), (lambda: p.free([b, b]), "twice"), (lambda: p.free([-1]), "no sequence"),
                        (lambda: p.trim([a], 0), "window"), (lambda: p.fork([9], 1), "no sequence"), (lambda: p.fork([a], -1), "children")):
        with pytest.raises(binding.BlendStepError, match=match):
            call()
        assert p.tables([a, b])[1].tolist() == before and p.stats() == {"free": 0, "sequences": 2}
    with pytest.raises(binding.BlendStepError):
        binding.Pages(-1)
    assert binding.Pages(0).stats()["free"] == 0


# ---- plans -----------------------------------------------------------------------------------
SHAPE = W.LayerShape(256, 8, 2, 64, 256)


@pytest.fixture(scope="module")
def host_layer():
    return binding.Layer(SHAPE, device=-1)


def test_plan_names_the_pages_that_rows_see(host_layer):
    # one row at 999: window of 100 tokens 900 .. 999 (pages 56 .. 62), sinks 0 .. 19 (pages 0, 1)
    plan = host_layer.window_plan(make_batch([(1, 1000)]), 100, 20)
    assert plan.division().pages == 9
    # sinks that meet the window, a window longer than the context, an idle slot
    assert plan.update(make_batch([(1, 1000)]), 100, 950).division().pages == 63
    assert plan.update(make_batch([(1, 1000)]), 1 << 30, 1 << 30).division().pages == 63
    assert plan.update(make_batch([(1, 0)]), 100, 4).division().pages == 0
    d = plan.update(make_batch([]), 5, 0).division()
    assert d.units == 0 and d.pages == 0


def test_pages_that_are_given_up_are_not_needed(host_layer):
    # pages 2 .. 55 of the example above
    b = make_batch([(1, 1000)], given_up={0: range(2, 56)})
    assert host_layer.window_plan(b, 100, 20).division().pages == 9
    for window, sinks in ((101 + 4, 20), (100, 33)):
        with pytest.raises(binding.BlendStepError, match="given up"):
            host_layer.window_plan(b, window, sinks)
    with pytest.raises(binding.BlendStepError, match="appends to page 62"):
        host_layer.window_plan(make_batch([(1, 1000)], given_up={0: [62]}), 100, 20)


def test_pages_trimmed_behind_the_window_are_never_needed_again(host_layer):
    # a sequence grows token by token, and by chunks, and is trimmed before every step
    rng = np.random.default_rng(5)
    for window, sinks in ((1, 0), (16, 0), (17, 4), (40, 17), (33, 64)):
        pages = binding.Pages(40)
        ids = pages.open(1)
        for _ in range(60):
            pages.trim(ids, window, sinks)
            rows = int(rng.choice([1, 1, 1, 5, 40]))
            try:
                pages.extend(ids, rows)
            except binding.BlendStepError:
                break
            start, table = pages.tables(ids)
            b = make_batch([(rows, int(pages.lengths(ids)[0]))])
            b.page_start, b.page_ids, b.n_pages = start, table, 40
            host_layer.window_plan(b, window, sinks)


def test_plan_refusals(host_layer):
    good = make_batch([(3, 40), (1, 17), (2, 1)])
    plan = host_layer.window_plan(good, 8, 1)

    def refused(match, batch=good, window=8, sinks=1, **kw):
        with pytest.raises(binding.BlendStepError, match=match) as e:
            plan.update(batch, window, sinks, **kw)
        assert e.value.code == -1
        with pytest.raises(binding.BlendStepError, match="nothing is planned"):
            plan.division()

    refused("at least 1", window=0)
    refused("at least 0", sinks=-1)
    b = good.copy(); b.page_ids[0] = b.n_pages
    refused("outside the pool", b)
    b = good.copy(); b.page_ids[0] = -2
    refused("outside the pool", b)
    b = good.copy(); b.page_ids[2] = b.page_ids[0]
    refused("referenced more than once", b)
    b = good.copy(); b.kv_len[1] = 33
    refused("exceeds its 2 pages", b)
    b = good.copy(); b.kv_len[1] = -1
    refused("out of range", b)
    b = good.copy(); b.row_start[1] = 5
    refused("row_start not monotone", b)
    b = good.copy(); b.n_rows = 7
    refused("row_start ends at", b)
    pos, axis = np.zeros((2, 6), dtype=np.int32), np.zeros(32, dtype=np.int32)
    p = pos.copy(); p[1, 5] = 16384
    refused("outside \\[0, 16384\\)", positions=p, axis_of_pair=axis)
    p = pos.copy(); p[0, 0] = -1
    refused("outside", positions=p, axis_of_pair=axis)
    a = axis.copy(); a[31] = 2
    refused("axis_of_pair\\[31\\]=2", positions=pos, axis_of_pair=a)
    refused("n_axes 9", positions=np.zeros((9, 6), dtype=np.int32), axis_of_pair=axis)
    plan.update(good, 8, 1, positions=pos, axis_of_pair=axis)
    # a host-only context plans, but runs nothing
    lib = host_layer.lib
    assert lib.bs_window_attention(plan.h, 16, 512, 16, 512, 16, None) == -1 and "host-only" in host_layer.last_error()
    assert lib.bs_rope_append(plan.h, 16, 768, 16, 512, 16, None) == -1 and "host-only" in host_layer.last_error()
    assert lib.bs_w4_linear(host_layer.h, 16, 64, 16, 1, 16, 64, 64, 0, 16, 16, None) == -1 and "host-only" in host_layer.last_error()


def test_bytes_of_a_laid_out_weight(host_layer):
    lib = host_layer.lib
    assert lib.bs_w4_bytes(16, 128, 128, 0) == 1024 + 32
    assert lib.bs_w4_bytes(17, 160, 32, 1) == 2 * (2 * 1024 + 8 * (32 + 16))
    for n, k, g in ((16, 128, 16), (16, 130, 64), (-1, 128, 64), (16, -64, 64), (1 << 40, 128, 64)):
        assert lib.bs_w4_bytes(n, k, g, 0) == 0
