"""Appending rows to a paged cache and attention of one new token over it, against plain forms in 64 bits."""
import math
import threading
from dataclasses import replace

import pytest
import torch

from paper_2511_17560_b200 import workloads as W
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MAX_POS = 5000
SHAPES = {"g1_64": (8, 8, 64), "g2": (4, 2, 128), "g7": (7, 1, 128), "g4": (32, 8, 128), "g7x4": (28, 4, 128), "g10_64": (20, 2, 64),
          "g24": (24, 1, 128), "g16": (32, 2, 128), "g32_64": (64, 2, 64), "g8_64": (16, 2, 64)}


@pytest.fixture(scope="module")
def a3():
    from paper_2511_17560_b200 import a3
    return a3


_engines = {}


def engine(a3, shape, layout=0):
    if (shape, layout) not in _engines:
        hq, hkv, d = SHAPES[shape]
        m = replace(W.TINY, n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, d_model=128, d_ff=128, rope_layout=layout, rope_theta=1e4)
        _engines[shape, layout] = a3.A3(m, W.make_weights_device(m, torch.device(DEV), 0), MAX_POS)
    return _engines[shape, layout]


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(torch.bfloat16)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make_pool(g, n, size, heads, d, packed, fill=None, interleaved=False):
    shape = (n, 2 if interleaved else 1, size, heads, d)
    k, v = (torch.full(shape, fill, device=DEV) if fill is not None else torch.randn(shape, generator=g, device=DEV) * (30 if packed else 1)
            for _ in range(2))
    dtype = torch.float8_e4m3fn if packed else torch.bfloat16
    k, v = k.to(dtype), v.to(dtype)
    if interleaved:  # keys and values of a page side by side in one pool
        k, v = k[:, 0], k[:, 1]
    else:
        k, v = k[:, 0], v[:, 0]
    scale = lambda: 0.01 + 0.02 * torch.rand(heads, generator=g, device=DEV)  # noqa: E731
    return (k, v, scale(), scale()) if packed else (k, v, None, None)


def make_table(g, lens, size, extra=2, width=None):
    counts = [-(-n // size) for n in lens]
    order = torch.randperm(sum(counts) + extra, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), width or max(1, max(counts))), -7, dtype=torch.int32, device=DEV)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    return table, sum(counts) + extra


def bits(t):
    return t.contiguous().view(torch.uint8)


# ------------------------------------------------------------------ append


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("shape,layout,size,mode", [
    ("g4", 0, 16, "slot"), ("g4", 1, 16, "gap"), ("g1_64", 0, 1, "delta"), ("g1_64", 1, 24, "slot"), ("g7", 0, 33, "back"),
    ("g7x4", 0, 64, "plain"), ("g24", 0, 7, "slot")])
def test_append(a3, shape, layout, size, mode, packed):
    hq, hkv, d = SHAPES[shape]
    eng, g = engine(a3, shape, layout), gen(size + 7 * packed)
    lens, new = [1, 130, 37, 0, 64], [1, 90, 37, 0, 5]
    table, n_pages = make_table(g, lens, size)
    kp, vp, ks, vs = make_pool(g, n_pages, size, hkv, d, packed)
    cache = a3.PagedCache(kp, vp, ks, vs)
    seq = ints(sum(([s] * c for s, c in enumerate(new)), []) + [-1, -5])
    slot = ints(sum((list(range(n - c, n)) for n, c in zip(lens, new)), []) + [0, 1 << 30])
    order = torch.randperm(len(seq), generator=g, device=DEV)  # rows in any order
    seq, slot = seq[order], slot[order]
    pos = {"slot": None, "gap": slot % 2000 + 2999, "delta": torch.full_like(slot, 4999), "back": -(slot % 4000) - 1, "plain": None}[mode]
    M = len(seq)
    wide = randn(g, M, hq + 2 * hkv + 1, d, std=2.0)
    wide[:, 0, :2] = 0.0  # a gap in front of the queries
    q, k, v = wide[:, 1:hq + 1], wide[:, hq + 1:hq + hkv + 1], wide[:, hq + hkv + 1:]
    before = [t.clone() for t in (kp, vp)]
    q_out = torch.full((M, hq, d), 77.0, dtype=torch.bfloat16, device=DEV)
    got_q = eng.paged_append(cache, table, seq, slot, k, v, q_rows=q, row_pos=pos, rotate=mode != "plain", q_out=q_out)
    assert eng.device_status() == 0 and got_q is q_out
    live = torch.nonzero(seq >= 0)[:, 0]
    p = (slot if pos is None else pos)[live]
    if mode == "plain":
        p = torch.zeros_like(p)
    page, entry = table[seq[live].long(), (slot[live] // size).long()].long(), (slot[live] % size).long()
    want_q, mag = R.turned(q[live], p, 1e4, layout)
    # products, cosines and the sum in fp32: 2^-22 of the magnitudes; one rounding to bf16
    assert ((q_out[live].double() - want_q).abs() <= want_q.abs() * 2.0 ** -8 + mag * 2.0 ** -22).all()
    assert (q_out[seq < 0] == 77.0).all()
    want_k, mag = R.turned(k[live], p, 1e4, layout)
    for pool, old, scale, want, m in ((kp, before[0], ks, want_k, mag), (vp, before[1], vs, v[live].double(), torch.zeros_like(mag))):
        got = pool.view(torch.uint8)[page, entry].view(pool.dtype).double()
        if packed:
            want, m = want / scale.double()[:, None], m / scale.double()[:, None]
            want = want.clamp(-R.E4M3_MAX, R.E4M3_MAX)
            # half a step of e4m3: 2^-4 of the value, 2^-10 below its smallest normal number
            assert ((got - want).abs() <= (want.abs() * 2.0 ** -4).clamp(min=2.0 ** -10) + m * 2.0 ** -21).all()
            assert (got[want.abs() == R.E4M3_MAX].abs() == R.E4M3_MAX).all()  # what is beyond the largest value is the largest value
        else:
            assert ((got - want).abs() <= want.abs() * 2.0 ** -8 + m * 2.0 ** -22).all()
        rest = torch.ones(pool.shape[:2], dtype=torch.bool, device=DEV)
        rest[page, entry] = False
        assert torch.equal(pool.view(torch.uint8)[rest], old.view(torch.uint8)[rest])  # nothing else was touched


def test_append_in_place_one_row_and_none(a3):
    eng, g = engine(a3, "g4"), gen(1)
    hq, hkv, d = SHAPES["g4"]
    kp, vp, _, _ = make_pool(g, 3, 16, hkv, d, False)
    cache, table = a3.PagedCache(kp, vp), ints([[2, 0]])
    q, k, v = randn(g, 1, hq, d), randn(g, 1, hkv, d), randn(g, 1, hkv, d)
    apart = eng.paged_append(cache, table, ints([0]), ints([17]), k, v, q_rows=q)
    assert eng.paged_append(cache, table, ints([0]), ints([17]), k, v, q_rows=q, q_out=q) is q
    assert torch.equal(apart, q)
    old = kp.clone()
    assert eng.paged_append(cache, table, ints([]), ints([]), k[:0], v[:0]) is None
    assert torch.equal(kp, old) and torch.equal(vp[0, 1], v[0]) and eng.device_status() == 0


def test_append_values_that_are_no_numbers(a3):
    eng, g = engine(a3, "g4"), gen(2)
    _, hkv, d = SHAPES["g4"]
    for packed in (False, True):
        kp, vp, ks, vs = make_pool(g, 1, 16, hkv, d, packed)
        k, v = randn(g, 1, hkv, d), randn(g, 1, hkv, d)
        v[0, 0, 0], v[0, 0, 1], v[0, 0, 2] = math.nan, math.inf, -math.inf
        eng.paged_append(a3.PagedCache(kp, vp, ks, vs), ints([[0]]), ints([0]), ints([3]), k, v)
        got = vp[0, 3, 0, :3].float()
        most = R.E4M3_MAX if packed else math.inf
        assert got[0].isnan() and got[1] == most and got[2] == -most


def test_append_leaves_out_rows_that_lead_nowhere(a3):
    """Sequence, slot, page and position beyond their ranges: such a row is left out as a whole and flagged, the others go in."""
    eng, g = engine(a3, "g4"), gen(3)
    hq, hkv, d = SHAPES["g4"]
    for seq, slot, pos in ((2, 0, 0), (0, 32, 0), (0, -1, 0), (1, 16, 0), (1, 0, 0), (0, 0, MAX_POS), (0, 0, -MAX_POS), (0, 0, -2 ** 31), (0, 2 ** 31 - 1, 0)):
        kp, vp, _, _ = make_pool(g, 3, 16, hkv, d, False)
        old = kp.clone(), vp.clone()
        table = ints([[2, 1], [3, -1]])  # sequence 1: pages outside the pool
        q, k, v = randn(g, 2, hq, d), randn(g, 2, hkv, d), randn(g, 2, hkv, d)
        q_out = torch.full_like(q, 5.0)
        eng.paged_append(a3.PagedCache(kp, vp), table, ints([seq, 0]), ints([slot, 20]), k, v, q_rows=q, row_pos=ints([pos, 1]), q_out=q_out)
        assert eng.device_status() == a3.DEV_BAD_POSITION
        assert (q_out[0] == 5.0).all() and torch.equal(vp[1, 4], v[1])
        rest = torch.ones(3, 16, dtype=torch.bool, device=DEV)
        rest[1, 4] = False
        assert torch.equal(kp[rest], old[0][rest]) and torch.equal(vp[rest], old[1][rest])


# ------------------------------------------------------------------ attention


def check_attention(a3, eng, cache, table, lens, q, scale=None):
    hq, d = q.shape[1:]
    out, lse = eng.paged_attention(cache, table, ints(lens), q, scale=scale, want_lse=True)
    assert eng.device_status() == 0
    for s, n in enumerate(lens):
        if n == 0:
            assert (out[s] == 0).all() and (lse[s] == -math.inf).all()
            continue
        k, v = R.gathered(cache.k_pages, cache.k_scale, table[s], n), R.gathered(cache.v_pages, cache.v_scale, table[s], n)
        want, want_lse, tol, tol_lse = R.attention(q[s], k, v, d ** -0.5 if scale is None else scale, cache.k_scale is not None, hq)
        err = (out[s].double() - want).abs()
        assert (err <= tol).all(), (s, n, (err - tol).max().item())
        err = (lse[s].double() - want_lse).abs()
        assert (err <= tol_lse).all(), (s, n, (err - tol_lse).max().item())
    return out, lse


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_attention_shapes(a3, shape, packed):
    hq, hkv, d = SHAPES[shape]
    eng, g = engine(a3, shape), gen(len(shape) + packed)
    lens = [1, 15, 16, 17, 0, 63, 64, 65, 500, 31, 0]
    table, n = make_table(g, lens, 16)
    cache = a3.PagedCache(*make_pool(g, n, 16, hkv, d, packed))
    check_attention(a3, eng, cache, table, lens, randn(g, len(lens), hq, d, std=2.0))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("size,lens", [
    (1, [7, 1, 100]), (3, [1000]), (16, [5153]), (24, [0, 0, 2500, 0, 1, 0]), (64, [4096, 1, 4097]), (200, [199, 200, 201, 20000]),
    (16, [1] * 700), (16, list(range(300))), (32, [0] * 9), (128, [70000, 3, 70001])])
def test_attention_lengths_and_pages(a3, size, lens, packed):
    hq, hkv, d = SHAPES["g4"] if sum(lens) < 100000 else SHAPES["g2"]
    eng, g = engine(a3, "g4" if hkv == 8 else "g2"), gen(size)
    table, n = make_table(g, lens, size)
    cache = a3.PagedCache(*make_pool(g, n, size, hkv, d, packed))
    check_attention(a3, eng, cache, table, lens, randn(g, len(lens), hq, d, std=2.0))


@pytest.mark.parametrize("packed,lens", [(False, [50000, 1, 0, 40000, 25000, 33]), (True, [120000, 0, 100001, 5000])])
def test_attention_with_late_parts(a3, packed, lens):
    """So many tiles that a tenth of them is left to late parts; and the same table with so few that there are none of them."""
    hq, hkv, d = SHAPES["g4"]
    eng, g = engine(a3, "g4"), gen(22)
    tile = 32 if packed else 16
    warps = torch.cuda.get_device_properties(0).multi_processor_count // hkv * 8
    assert sum(-(-n // tile) for n in lens) >= 48 * warps  # from there on there are late parts
    table, n = make_table(g, lens, 32)
    cache = a3.PagedCache(*make_pool(g, n, 32, hkv, d, packed))
    q = randn(g, len(lens), hq, d, std=2.0)
    check_attention(a3, eng, cache, table, lens, q)
    check_attention(a3, eng, cache, table, [n // 1000 for n in lens], q)


def test_attention_reads_nothing_behind_a_sequence(a3):
    """Entries behind the last slot hold NaN, table entries behind the last page name no page; pages apart, queries in a wider buffer."""
    for packed in (False, True):
        hq, hkv, d = SHAPES["g4"]
        eng, g = engine(a3, "g4"), gen(11)
        lens = [1, 33, 16, 250, 0]
        table, n = make_table(g, lens, 16, width=40)
        kp, vp, ks, vs = make_pool(g, n, 16, hkv, d, packed, interleaved=True)
        assert kp.stride(0) == 2 * 16 * hkv * d
        used = torch.zeros(n, 16, dtype=torch.bool, device=DEV)
        for s, m in enumerate(lens):
            t = torch.arange(m, device=DEV)
            used[table[s].long()[t // 16], t % 16] = True
        for p in (kp, vp):
            p.view(torch.uint8)[~used] = 0x7F if packed else 0xFF  # NaN
        wide = randn(g, len(lens), hq + 3, d, std=2.0)
        check_attention(a3, eng, a3.PagedCache(kp, vp, ks, vs), table, lens, wide[:, 2:hq + 2])


def test_attention_scales_and_extreme_values(a3):
    eng, g = engine(a3, "g4"), gen(12)
    hq, hkv, d = SHAPES["g4"]
    lens = [100, 700]
    table, n = make_table(g, lens, 16)
    for packed in (False, True):
        pool = make_pool(g, n, 16, hkv, d, packed)
        cache = a3.PagedCache(*pool)
        for scale in (-0.1, 0.0, 1.0):
            check_attention(a3, eng, cache, table, lens, randn(g, 2, hq, d), scale=scale)
        # queries of far-apart magnitudes per head, one head all zeros
        q = randn(g, 2, hq, d) * (10.0 ** torch.linspace(-30, 1, hq, device=DEV))[:, None].to(torch.bfloat16)
        q[:, 3] = 0
        check_attention(a3, eng, cache, table, lens, q.contiguous())
        q[1, 5, 0] = math.nan  # stays in its head
        out, lse = eng.paged_attention(cache, table, ints(lens), q, want_lse=True)
        assert out[1, 5].isnan().all() and lse[1, 5].isnan()
        out[1, 5], lse[1, 5] = 0, 0
        assert out.isfinite().all() and lse.isfinite().all()


def test_attention_of_rising_logits(a3):
    """Every tile raises the maximum: the accumulators are rescaled each time; then the other way round."""
    eng, g = engine(a3, "g4"), gen(13)
    hq, hkv, d = SHAPES["g4"]
    for sign in (1, -1):
        kp, vp, _, _ = make_pool(g, 130, 16, hkv, d, False)
        table = torch.arange(130, dtype=torch.int32, device=DEV)[None]
        kp[..., 0] = sign * (torch.arange(130 * 16, device=DEV).view(130, 16, 1) / 50.0).to(torch.bfloat16)
        q = randn(g, 1, hq, d, std=0.1)
        q[..., 0] = 20.0
        check_attention(a3, eng, a3.PagedCache(kp, vp), table, [2080], q)


def test_attention_flags_lengths_and_pages_out_of_range(a3):
    eng, g = engine(a3, "g4"), gen(14)
    hq, hkv, d = SHAPES["g4"]
    kp, vp, _, _ = make_pool(g, 4, 16, hkv, d, False)
    cache, q = a3.PagedCache(kp, vp), randn(g, 3, hq, d)
    table = ints([[0, 1], [2, 3], [1, 0]])
    good, _ = eng.paged_attention(cache, table, ints([20, 32, 5]), q)
    assert eng.device_status() == 0
    out, lse = eng.paged_attention(cache, table, ints([20, 33, -1]), q, want_lse=True)
    assert eng.device_status() == a3.DEV_BAD_POSITION
    assert torch.equal(out[0], good[0]) and (out[1:] == 0).all() and (lse[1:] == -math.inf).all()
    out, _ = eng.paged_attention(cache, ints([[0, 4], [2, 3], [-1, 0]]), ints([20, 32, 5]), q)
    assert eng.device_status() == a3.DEV_BAD_POSITION
    assert torch.equal(out[1], good[1]) and (out[2] == 0).all() and out.isfinite().all()


def test_attention_beyond_32_bit_offsets(a3):
    """A pool of 4.5 GiB of keys and as much of values: offsets in bytes and, in 8 bits, in elements pass 32 bits."""
    eng, g = engine(a3, "g4"), gen(15)
    hq, hkv, d = SHAPES["g4"]
    for packed in (False, True):
        n = (9 << 29) // (16 * hkv * d * (1 if packed else 2))
        kp, vp = (torch.zeros((n, 16, hkv, d), dtype=torch.uint8 if packed else torch.bfloat16, device=DEV) for _ in range(2))
        if packed:
            kp, vp = kp.view(torch.float8_e4m3fn), vp.view(torch.float8_e4m3fn)
        scales = (torch.full((hkv,), 0.05, device=DEV),) * 2 if packed else ()
        cache, table = a3.PagedCache(kp, vp, *scales), ints([[n - 1, 3, n - 2], [n // 2, n - 5, 0]])
        M = 96
        seq, slot = ints([0] * 48 + [1] * 48), ints(list(range(48)) * 2)
        k, v = randn(g, M, hkv, d), randn(g, M, hkv, d)
        eng.paged_append(cache, table, seq, slot, k, v, rotate=False)
        if not packed:
            assert torch.equal(kp[n - 1], k[:16]) and torch.equal(vp[n - 5], v[64:80])
        check_attention(a3, eng, cache, table, [48, 41], randn(g, 2, hq, d))
        del kp, vp, cache


def test_results_repeat_bit_for_bit_and_follow_captured_lengths(a3):
    """The same call twice; captured, with lengths, slots and rows changed between replays; two graphs at once."""
    hq, hkv, d = SHAPES["g4"]
    eng, g = engine(a3, "g4"), gen(16)
    full = [300, 2000, 64, 900, 1]
    table, n = make_table(g, full, 16)
    kp, vp, _, _ = make_pool(g, n, 16, hkv, d, False)
    cache, other = a3.PagedCache(kp, vp), a3.PagedCache(kp.clone(), vp.clone())
    seq, slot, lens = ints(range(5)), ints([0] * 5), ints([1] * 5)
    q, k, v = randn(g, 5, hq, d), randn(g, 5, hkv, d), randn(g, 5, hkv, d)

    def step(c):
        return eng.paged_attention(c, table, lens, eng.paged_append(c, table, seq, slot, k, v, q_rows=q), want_lse=True)

    step(cache), step(other)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in (cache, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(c))
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for trial in range(4):
        now = [0, 1999, 63, 17 * trial, 0] if trial else [5, 7, 0, 1, 0]
        slot.copy_(ints(now))
        lens.copy_(ints([t + 1 for t in now]) * ints([1, 1, 1, 1, trial % 2]))
        k.copy_(randn(g, 5, hkv, d))
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
                graph.replay()
        torch.cuda.synchronize()
        want = step(cache)
        again = step(cache)
        for a, b, c, e in zip(want, again, *outs):
            assert torch.equal(bits(a), bits(b)) and torch.equal(bits(a), bits(c)) and torch.equal(bits(a), bits(e))
    assert eng.device_status() == 0


def test_calls_on_another_stream(a3):
    hq, hkv, d = SHAPES["g2"]
    eng, g = engine(a3, "g2"), gen(17)
    lens = [3000, 5]
    table, n = make_table(g, lens, 16)
    cache = a3.PagedCache(*make_pool(g, n, 16, hkv, d, False))
    q = randn(g, 2, hq, d)
    want, _ = eng.paged_attention(cache, table, ints(lens), q)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    lens = ints(lens)
    torch.cuda.synchronize()
    for _ in range(20):
        for st in streams:
            with torch.cuda.stream(st):
                got.append(eng.paged_attention(cache, table, lens, q)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(want, o) for o in got)


def test_calls_from_two_threads(a3):
    """Each thread decodes on a stream and a pool of its own through one engine; the calls let the other thread run while they launch."""
    hq, hkv, d = SHAPES["g4"]
    eng, g = engine(a3, "g4"), gen(23)
    sets = []
    for i in range(2):
        lens = [700 + 900 * i, 3, 2500]
        table, n = make_table(g, lens, 16)
        kp, vp, _, _ = make_pool(g, n, 16, hkv, d, False)
        sets.append((a3.PagedCache(kp, vp), table, ints(range(3)), ints([x - 1 for x in lens]), ints(lens), randn(g, 3, hq, d), randn(g, 3, hkv, d),
                     randn(g, 3, hkv, d), randn(g, 3, 20000), ints([0, 19999, 5])))

    def step(cache, table, seq, slot, lens, q, k, v, x, t):
        return (*eng.paged_attention(cache, table, lens, eng.paged_append(cache, table, seq, slot, k, v, q_rows=q), want_lse=True), *eng.token_logprobs(x, t, 4))

    want = [step(*s) for s in sets]
    torch.cuda.synchronize()
    got = [[], []]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            got[i] = [step(*sets[i]) for _ in range(200)][-20:]
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    for i in range(2):
        assert len(got[i]) == 20 and all(torch.equal(bits(a), bits(b)) for step_out in got[i] for a, b in zip(want[i], step_out))
    assert eng.device_status() == 0


def test_attention_without_pages(a3):
    """A page table of no columns: every sequence is padding."""
    eng, g = engine(a3, "g4"), gen(20)
    hq, hkv, d = SHAPES["g4"]
    kp, vp, _, _ = make_pool(g, 1, 16, hkv, d, False)
    for n in (1, 3, 400):
        q = randn(g, n, hq, d)
        out, lse = eng.paged_attention(a3.PagedCache(kp, vp), torch.empty((n, 0), dtype=torch.int32, device=DEV), ints([0] * n), q, want_lse=True)
        assert (out == 0).all() and (lse == -math.inf).all() and eng.device_status() == 0
    out, _ = eng.paged_attention(a3.PagedCache(kp, vp), torch.empty((0, 4), dtype=torch.int32, device=DEV), ints([]), q[:0])
    assert out.shape == (0, hq, d)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("shape", ["g4", "g2", "g10_64"])
def test_attention_where_a_cluster_has_a_sequence(a3, shape, packed):
    """Page tables as wide as one, two, four and eight CTAs take, and wider; in each, lengths that leave CTAs of a cluster, or all, without keys."""
    hq, hkv, d = SHAPES[shape]
    eng, g = engine(a3, shape), gen(24)
    for n in (1, 3):
        for width in (40, 100, 300, 1300, 2600, 5100, 6200):
            table, pages = make_table(g, [width] * n, 16)
            cache = a3.PagedCache(*make_pool(g, pages, 16, hkv, d, packed))
            for lens in ([width] * n, [1, 0, width // 2][:n], [0, 17, width - 1][:n], [33, 32, 31][:n]):
                q = randn(g, n, hq, d, std=2.0)
                check_attention(a3, eng, cache, table, lens, q)
                first = eng.paged_attention(cache, table, ints(lens), q, want_lse=True)
                for a, b in zip(first, eng.paged_attention(cache, table, ints(lens), q, want_lse=True)):
                    assert torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("packed", [False, True])
def test_attention_where_one_cta_or_many_have_a_sequence(a3, packed):
    """The same sequences behind page tables of different widths: alone in a CTA each, and on the line of all CTAs."""
    hq, hkv, d = SHAPES["g4"]
    eng, g = engine(a3, "g4"), gen(21)
    lens = [600, 1, 0, 17, 333]
    narrow, n = make_table(g, lens, 16, width=40)
    cache = a3.PagedCache(*make_pool(g, n, 16, hkv, d, packed))
    q = randn(g, 5, hq, d, std=2.0)
    lib = a3._load()
    assert lib.a3_paged_attention_workspace_bytes(eng._h, cache._ref, 5, 40) == 0
    wide = torch.full((5, 200), -3, dtype=torch.int32, device=DEV)
    wide[:, :40] = narrow
    assert lib.a3_paged_attention_workspace_bytes(eng._h, cache._ref, 5, 200) > 0
    a3.launch_count(reset=True)
    check_attention(a3, eng, cache, narrow, lens, q)
    assert a3.launch_count() == 1
    check_attention(a3, eng, cache, wide, lens, q)
    assert a3.launch_count() == 3


# ------------------------------------------------------------------ values far apart, and infinite ones


@pytest.mark.parametrize("lens", [[1000], [3000] * 200, [20000, 5]])
def test_attention_in_8_bits_of_many_small_weights(a3, lens):
    """The first key far above all others, whose weights are e^-gap of its own and whose values are 1 where its own is 0: the output is what the small
    weights add up to, w n' / (1 + w n').  A weight is off by 2^-11 of itself or, where fp16 has fewer bits for it, by half a step of 2^-24 beside a largest
    weight of 2^7 at least: 2^-32.  The logits' own errors are R.attention's."""
    hq, hkv, d = SHAPES["g2"]
    eng, g = engine(a3, "g2"), gen(30)
    table, n = make_table(g, lens, 32)
    f8 = torch.float8_e4m3fn
    for gap in (17.5, 12.0, 14.5, 20.0):
        kp, vp = torch.zeros((n, 32, hkv, d), device=DEV), torch.ones((n, 32, hkv, d), device=DEV)
        for s in range(len(lens)):
            kp[table[s, 0].long(), 0, :, 0] = 4.0
            vp[table[s, 0].long(), 0] = 0.0
        one = torch.ones(hkv, device=DEV)
        cache = a3.PagedCache(kp.to(f8), vp.to(f8), one, one)
        q = torch.zeros((len(lens), hq, d), dtype=torch.bfloat16, device=DEV)
        q[..., 0] = 1.0
        out, lse = eng.paged_attention(cache, table, ints(lens), q, scale=gap / 4, want_lse=True)
        assert eng.device_status() == 0
        for s, m in enumerate(lens):
            small = (m - 1) * math.exp(-gap)
            want = small / (1 + small)
            delta = gap * d * 2.0 ** -23 + (m + 8) * 2.0 ** -24
            tol = want * (2.0 ** -8 + 2.0 ** -11 + 2 * delta) + m * 2.0 ** -32
            assert ((out[s].double() - want).abs() <= tol).all(), (gap, s, m, out[s, 0, 0].item(), want)
            assert ((lse[s].double() - gap - math.log1p(small)).abs() <= delta + 32 * 2.0 ** -22).all()


@pytest.mark.parametrize("lens", [[40], [700, 3], [2500, 2], [9000, 0, 17]])
def test_attention_of_infinite_values(a3, lens):
    """A value of +inf makes that dimension +inf wherever its weight is above 0, -inf likewise, both together NaN; the other dimensions are as before."""
    hq, hkv, d = SHAPES["g4"]
    eng, g = engine(a3, "g4"), gen(31)
    table, n = make_table(g, lens, 16)
    kp, vp, _, _ = make_pool(g, n, 16, hkv, d, False)
    cache, q = a3.PagedCache(kp, vp), randn(g, len(lens), hq, d)
    clean, clean_lse = eng.paged_attention(cache, table, ints(lens), q, want_lse=True)
    for where in (0, 33, lens[0] - 1):
        at = (table[0, where // 16].long(), where % 16)
        old = vp[at].clone()
        vp[at[0], at[1], :, 5], vp[at[0], at[1], :, 100], vp[at[0], at[1], :, 64] = math.inf, -math.inf, math.inf
        other = (table[0, (lens[0] - 2) // 16].long(), (lens[0] - 2) % 16)
        old2 = vp[other].clone()
        vp[other[0], other[1], :, 64] = -math.inf
        out, lse = eng.paged_attention(cache, table, ints(lens), q, want_lse=True)
        assert eng.device_status() == 0
        assert (out[0, :, 5] == math.inf).all() and (out[0, :, 100] == -math.inf).all() and out[0, :, 64].isnan().all()
        out[0, :, [5, 64, 100]] = clean[0, :, [5, 64, 100]]
        assert torch.equal(bits(out), bits(clean)) and torch.equal(bits(lse), bits(clean_lse))
        vp[other], vp[at] = old2, old
    # a weight of 0 beside a value near the largest number adds nothing
    q[0, :, 0] = 4.0
    kp[table[0, 0].long(), 1], kp[table[0, 0].long(), 1, :, 0] = 0.0, -400.0
    vp[table[0, 0].long(), 1] = 3e38
    check_attention(a3, eng, cache, table, lens, q)


def test_profiles_tell_decoding_from_fusion(a3):
    """Each of the decoding calls is a class of its own, with a record for every launch."""
    hq, hkv, d = SHAPES["g2"]
    m = replace(W.TINY, n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, d_model=128, d_ff=128)
    eng, g = a3.A3(m, W.make_weights_device(m, torch.device(DEV), 0), 64), gen(32)
    kp, vp, _, _ = make_pool(g, 4, 16, hkv, d, False)
    cache, q, k = a3.PagedCache(kp, vp), randn(g, 1, hq, d), randn(g, 1, hkv, d)
    narrow, wide = ints([[1, 2]]), ints([[1] * 4000])
    eng.profile_enable(64)
    a3.launch_count(reset=True)
    eng.paged_append(cache, narrow, ints([0]), ints([3]), k, k, q_rows=q)
    eng.paged_attention(cache, narrow, ints([4]), q)
    eng.paged_attention(cache, wide, ints([4]), q)  # two launches
    eng.token_logprobs(torch.zeros((2, 100), device=DEV))
    got = {name: e["launches"] for name, e in eng.profile_read().items() if e["launches"]}
    assert got == {"paged_append": 1, "paged_attention": 3, "token_logprobs": 1} and a3.launch_count() == 5
    eng.profile_enable(0)
    eng.close()


# ------------------------------------------------------------------ refusals


def test_refusals_of_the_library(a3):
    """What the host can see is refused before any launch."""
    import ctypes as C
    eng, g = engine(a3, "g4"), gen(18)
    hq, hkv, d = SHAPES["g4"]
    kp, vp, _, _ = make_pool(g, 4, 16, hkv, d, False)
    cache, lib = a3.PagedCache(kp, vp), a3._load()
    q, k, v, o = randn(g, 1, hq, d), randn(g, 1, hkv, d), randn(g, 1, hkv, d), randn(g, 1, hq, d)
    one, zero = ints([1]), ints([0])
    wide = 1 << 12  # pages of a table that a sequence alone in a CTA is not meant for
    table = torch.zeros((1, wide), dtype=torch.int32, device=DEV)
    nbytes = lib.a3_paged_attention_workspace_bytes(eng._h, cache._ref, 1, wide)
    assert nbytes > 0 and lib.a3_paged_attention_workspace_bytes(eng._h, cache._ref, 1, 1) == 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    p = lambda t: t.data_ptr()  # noqa: E731
    whole = lambda kw: [0 if v is None else v for v in kw.values()]  # noqa: E731
    good = dict(t=p(table), len=p(one), q=p(q), o=p(o), lse=None, ws=p(ws), b=nbytes, qs=hq * d, n=1, w=wide, scale=0.1, r=0)
    attend = lambda h=eng._h, c=C.addressof(cache.desc), **kw: lib.a3_paged_attention(h, c, R.PAGED_QUERIES.pack(*whole({**good, **kw})), 0)  # noqa: E731
    assert attend() == 0 and attend(w=1, ws=None, b=0) == 0 and lib.a3_paged_attention(eng._h, cache._ref, None, 0) == -1 and lib.a3_paged_append(eng._h, cache._ref, None, 0) == -1
    a3.launch_count(reset=True)
    kept = []

    def desc(**kw):
        kept.append(a3.PagedCacheDesc(*{**{f: getattr(cache.desc, f) for f, _ in a3.PagedCacheDesc._fields_}, **kw}.values()))
        return C.addressof(kept[-1])

    bad_caches = [dict(k_pages=None), dict(v_pages=p(vp) + 2), dict(n_pages=0), dict(page_size=0), dict(page_stride=16 * hkv * d * 2 - 16),
                  dict(page_stride=16 * hkv * d * 2 + 8), dict(type=1), dict(page_stride=1 << 62)]
    for kw in [dict(h=None), dict(c=None), dict(t=None), dict(n=-1), dict(w=-1), dict(len=None), dict(q=None), dict(q=p(q) + 2), dict(qs=hq * d - 8),
               dict(qs=hq * d + 4), dict(qs=1 << 32), dict(scale=math.inf), dict(scale=math.nan), dict(o=None), dict(o=p(o) + 8), dict(ws=None), dict(ws=p(ws) + 16)]:
        assert attend(**kw) == -1, kw
    for kw in bad_caches:
        assert attend(c=desc(**kw)) == -1, kw
    assert attend(c=desc(type=2)) == -2 and attend(b=nbytes - 1) == -3 and attend(n=0) == 0
    assert attend(w=1 << 27) == -6 and attend(n=1 << 10, w=(1 << 20) + 1) == -6
    good_a = dict(t=p(table), seq=p(zero), slot=p(zero), pos=None, q=p(q), k=p(k), v=p(v), o=p(o), qs=hq * d, ks=hkv * d, vs=hkv * d, os=hq * d,
                  n=1, w=1, M=1, rot=1)
    append = lambda h=eng._h, c=C.addressof(cache.desc), **kw: lib.a3_paged_append(h, c, R.PAGED_ROWS.pack(*whole({**good_a, **kw})), 0)  # noqa: E731
    for kw in [dict(h=None), dict(c=None), dict(t=None), dict(n=-1), dict(w=-1), dict(seq=None), dict(slot=None), dict(k=None), dict(v=None),
               dict(q=None), dict(o=None), dict(M=-1), dict(k=p(k) + 2), dict(ks=hkv * d - 8), dict(vs=hkv * d + 1), dict(qs=8), dict(os=hq * d + 4), dict(ks=1 << 32)]:
        assert append(**kw) == -1, kw
    for kw in bad_caches:
        assert append(c=desc(**kw)) == -1, kw
    assert append(M=0) == 0 and a3.launch_count() == 0
    assert append() == 0 and append(q=None, o=None) == 0 and eng.device_status() == 0


# ------------------------------------------------------------------ together


def test_decoding_after_fusion(a3):
    """A fused request's cache goes into pages as it is, further tokens are decoded over the pages, and their log probabilities taken.
    Each layer of a step against a3_recompute_layer, which runs the same row over the contiguous cache."""
    m, r = W.request_for("tiny_gqa")
    dev = torch.device(DEV)
    weights = W.make_weights_device(m, dev, 3)
    n, steps, size = r.n, 3, 16
    eng = a3.A3(m, weights, n + steps)
    g = gen(19)
    L, Hq, Hkv, D = m.n_layers, m.n_q_heads, m.n_kv_heads, m.head_dim
    ck, cv, x0 = [], [], randn(g, n, m.d_model)
    for o, t in zip(r.offsets, r.chunk_lens):
        k, v = (torch.zeros((L, t, Hkv, D), dtype=torch.bfloat16, device=dev) for _ in range(2))
        eng.precompute_chunk(x0[o:o + t].clone(), k, v)
        ck.append(k), cv.append(v)
    K, V = (torch.zeros((L, n, Hkv, D), dtype=torch.bfloat16, device=dev) for _ in range(2))
    req, out = eng.make_request(a3.chunk_table(ck, cv, r.offsets), len(ck), max(r.chunk_lens), r.n_ctx, r.n_question, x0, K, V)
    eng.fuse_request(req)
    # two sequences share the request's pages (their own from the first decoded token on)
    n_pages = -(-n // size) + 4
    kp, vp = (torch.full((L, n_pages, size, Hkv, D), math.nan, dtype=torch.bfloat16, device=dev) for _ in range(2))
    caches = [a3.PagedCache(kp[l], vp[l]) for l in range(L)]
    common = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    table = common[None, :-(-n // size) + 1].repeat(2, 1).contiguous()
    table[1, n // size:] = common[-3:][: table.shape[1] - n // size]
    slots = torch.arange(n, dtype=torch.int32, device=dev)
    tail = slots[n // size * size:]  # the last page's rows go to both
    for l in range(L):
        eng.paged_append(caches[l], table, torch.cat([torch.zeros_like(slots), torch.ones_like(tail)]), torch.cat([slots, tail]),
                         torch.cat([K[l], K[l][tail.long()]]), torch.cat([V[l], V[l][tail.long()]]), rotate=False)
    for l in range(L):
        assert torch.equal(kp[l].flatten(0, 1)[(table[0].long()[slots.long() // size] * size + slots % size)], K[l])
    flat = [torch.cat([t, torch.zeros((L, steps, Hkv, D), dtype=torch.bfloat16, device=dev)], 1).contiguous() for t in (K, V)]
    norm, head = torch.ones(m.d_model, dtype=torch.bfloat16, device=dev), randn(g, m.vocab, m.d_model, std=0.05)
    table_t = randn(g, m.vocab, m.d_model)
    row = out["x"][-1]
    for step in range(steps):
        logits, token = eng.first_token(row, norm, head)
        logprob, entropy, ids, lps = eng.token_logprobs(logits[None], token, 5)
        lp, h, tol, tol_h = R.logprobs(logits[None])
        assert ids[0, 0] == token[0] and torch.equal(ids.long(), R.ranked(logits[None], 5))
        assert ((lps.double() - lp.gather(1, ids.long())).abs() <= tol.gather(1, ids.long())).all() and logprob[0] == lps[0, 0]
        assert ((entropy.double() - h).abs() <= tol_h).all()
        x = table_t[token.long()].repeat(2, 1)
        ref = x[:1].clone()
        at = n + step
        for l, w in enumerate(weights):
            def rms(y, gain):
                y = y.double()
                return (y * (y.square().mean(-1, keepdim=True) + m.rms_eps).rsqrt() * gain.double()).to(torch.bfloat16)

            lin = lambda y, name: y.double() @ w[name].double().T  # noqa: E731, B023
            a = rms(x, w["attn_norm"])
            qkv = torch.cat([lin(a, f) for f in ("wq", "wk", "wv")], 1).to(torch.bfloat16).view(2, Hq + 2 * Hkv, D)
            q = eng.paged_append(caches[l], table, ints([0, 1]), ints([at, at]), qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], q_rows=qkv[:, :Hq])
            o, _ = eng.paged_attention(caches[l], table, ints([at + 1] * 2), q)
            assert torch.equal(o[0], o[1])  # the same keys from different pages
            x = (x.double() + lin(o.flatten(1), "wo")).to(torch.bfloat16)
            b = rms(x, w["mlp_norm"])
            gate, up = lin(b, "w_gate"), lin(b, "w_up")
            x = (x.double() + lin((gate * torch.sigmoid(gate) * up).to(torch.bfloat16), "w_down")).to(torch.bfloat16)
            eng.recompute_layer(l, ref, ints([at]), flat[0][l][:at + 1], flat[1][l][:at + 1])
            # keys: rounded twice here (projection and rotation, 2^-8 of the pair each), once there, on hidden rows whose own
            # distance is what the layers before have made of such roundings: 2^-6 of the row's norm for each layer
            for pool, have in ((kp, flat[0]), (vp, flat[1])):
                new = pool[l][table[0].long()[at // size], at % size]
                assert (new.double() - have[l][at].double()).norm() <= (l + 1) * 2.0 ** -6 * have[l][at].double().norm()
            assert (x[0].double() - ref[0].double()).norm() <= (l + 1) * 2.0 ** -6 * ref[0].double().norm()
        row = x[0]
    assert eng.device_status() == 0
    eng.close()
