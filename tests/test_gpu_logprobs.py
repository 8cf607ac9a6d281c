"""Log probabilities of given tokens, entropies and the best alternatives, against plain forms in 64 bits."""
import math
from dataclasses import replace

import pytest
import torch

from paper_2511_17560_b200 import workloads as W
from tests import paged_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def a3():
    from paper_2511_17560_b200 import a3
    return a3


@pytest.fixture(scope="module")
def eng(a3):
    m = replace(W.TINY, n_layers=1, d_model=128, d_ff=128, n_q_heads=2, n_kv_heads=2)
    return a3.A3(m, W.make_weights_device(m, torch.device(DEV), 0), 8)


def check(eng, x, targets, n, status=0):
    logprob, entropy, ids, lps = eng.token_logprobs(x, targets, n)
    assert eng.device_status() == status
    lp, h, tol, tol_h = R.logprobs(x)
    if targets is not None:
        at = targets.long().clamp(min=0)[:, None]
        want, t = lp.gather(1, at)[:, 0], tol.gather(1, at)[:, 0]
        want, t = torch.where(targets < 0, 0.0, want), torch.where(targets < 0, 0.0, t)
        gone = want.isinf()  # a token that is ruled out
        assert (logprob[gone] == -math.inf).all()
        assert ((logprob.double() - want).abs() <= t)[~gone].all()
    else:
        assert logprob is None
    assert ((entropy.double() - h).abs() <= tol_h).all(), ((entropy.double() - h).abs() - tol_h).max()
    if n:
        best = R.ranked(x, n)
        assert torch.equal(ids.long(), best)
        want, t = lp.gather(1, best), tol.gather(1, best)
        gone = want.isinf()
        assert (lps[gone] == -math.inf).all() and ((lps.double() - want).abs() <= t)[~gone].all()
    else:
        assert ids is None and lps is None


def rows(M, V, dtype, seed=0, std=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn((M, V), generator=g, device=DEV) * std).to(dtype), torch.randint(V, (M,), generator=g, device=DEV).to(torch.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,V,n", [(1, 1, 1), (3, 2, 2), (2, 5, 0), (4, 31, 31), (2, 32, 32), (7, 257, 5), (1, 1000, 32), (1, 4097, 20),
                                   (5, 9001, 1), (64, 16384, 7), (300, 32001, 32), (1, 128256, 20), (65, 152064, 20), (297, 128256, 3), (20, 40000, 0)])
def test_rows(eng, M, V, n, dtype):
    x, t = rows(M, V, dtype, M + V)
    check(eng, x, t, n)


def test_rows_apart_and_unaligned(eng):
    for dtype in (torch.float32, torch.bfloat16):
        wide, t = rows(9, 5003, dtype, 1)
        for first in range(0, 9):
            check(eng, wide[:, first:first + 4987], (t % 4987).contiguous(), 6)


def test_ties_go_to_the_lower_id(eng):
    """Few distinct values, and rows of one value: more elements at the bound than are kept apart."""
    for V in (100, 5000, 128256):
        g = torch.Generator(device=DEV).manual_seed(V)
        x = torch.randint(-3, 3, (3, V), generator=g, device=DEV).to(torch.bfloat16)
        x[1] = 2.5
        x[2] = torch.where(torch.rand(V, generator=g, device=DEV) < 0.5, 0.0, -0.0).to(torch.bfloat16)  # both zeros are alike
        check(eng, x, torch.zeros(3, dtype=torch.int32, device=DEV), 20)
        check(eng, x.float(), None, 32)
        check(eng, x[:1].float().repeat(400, 1), None, 4)


def test_sorted_rows(eng):
    for V in (3000, 128256):
        up = torch.linspace(-20, 20, V, device=DEV)
        check(eng, torch.stack([up, up.flip(0), -up.abs()]), None, 32)
        blocks = torch.zeros(2, V, device=DEV)
        blocks[0, V // 2:V // 2 + 900] = torch.linspace(5, 6, 900, device=DEV)  # the best ones are neighbours
        blocks[1, :4096:512] = 7.0
        check(eng, blocks, None, 32)
        check(eng, blocks.bfloat16(), None, 32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ruled_out_tokens(eng, dtype):
    """-inf almost everywhere: fewer tokens are left than alternatives asked for; and rows of the type's lowest value."""
    for V, left in ((50, 1), (6000, 3), (128256, 2), (128256, 40), (128256, 1000)):
        x, t = rows(3, V, dtype, V + left)
        keep = torch.zeros((3, V), dtype=torch.bool, device=DEV)
        for r in range(3):
            keep[r, torch.randperm(V, device=DEV)[:left]] = True
        keep[2] = False
        keep[2, V - left:] = True  # all at the end, where the elements behind the last whole vector are
        x[~keep] = -math.inf
        check(eng, x, t, 20)
        x = torch.where(keep, x, torch.full_like(x, torch.finfo(dtype).min))
        check(eng, x, t, 20)
    check(eng, torch.full((2, 700), torch.finfo(dtype).min, dtype=dtype, device=DEV), None, 9)


def test_ruled_out_beside_the_lowest_values(eng):
    """A largest logit so low that the type has no number far below it: -inf still adds nothing at all."""
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        low = torch.finfo(dtype).min
        for top in (low, low * (1 - torch.finfo(dtype).eps), low * 0.998, low * 0.99):
            x = torch.full((2, 20000), -math.inf, dtype=dtype, device=DEV)
            t = torch.tensor([4321, 0], dtype=torch.int32, device=DEV)
            x[torch.arange(2), t.long()] = top
            logprob, entropy, ids, lps = eng.token_logprobs(x, t, 2)
            assert eng.device_status() == 0
            assert logprob.tolist() == [0, 0] and entropy.tolist() == [0, 0] and lps.tolist() == [[0, -math.inf]] * 2
            assert ids.tolist() == [[4321, 0], [0, 1]]


def test_nearly_certain_tokens(eng):
    """One logit far above the others: what is missing from 1, and the entropy, come from the others alone.  Those that share the
    largest one's thread (1 in 512) are lost below 2^-24, hence 1 %."""
    x, _ = rows(4, 32000, torch.float32, 5, std=1.0)
    t = torch.tensor([5, 31999, 0, 16000], dtype=torch.int32, device=DEV)
    x[torch.arange(4), t.long()] = torch.tensor([25.0, 35.0, 45.0, 60.0], device=DEV)
    logprob, entropy, ids, lps = eng.token_logprobs(x, t, 2)
    lp = torch.log_softmax(x.double(), 1)
    s = torch.where(torch.arange(32000, device=DEV) == t[:, None], 0.0, (x.double() - x.double().amax(1, keepdim=True)).exp()).sum(1)
    h = torch.log1p(s) - (lp.exp() * (x.double() - x.double().amax(1, keepdim=True))).sum(1)
    assert ((logprob.double() + torch.log1p(s)).abs() <= 0.01 * s).all()
    assert ((entropy.double() - h).abs() <= 0.01 * h).all()
    assert torch.equal(ids[:, 0], t) and torch.equal(lps[:, 0], logprob)


def test_large_values(eng):
    x, t = rows(3, 20000, torch.float32, 6, std=1000.0)
    check(eng, x, t, 5)
    x, t = rows(3, 20000, torch.float32, 7)
    x += torch.tensor([[1e4], [-1e4], [3e5]], device=DEV)
    check(eng, x, t, 5)


def test_rows_without_a_distribution(a3, eng):
    for V in (40, 5000, 128256):
        for dtype in (torch.float32, torch.bfloat16):
            x, t = rows(5, V, dtype, V)
            x[0, V // 2] = math.nan
            x[1, V - 1] = math.inf
            x[2] = -math.inf
            x[3, 1:] = -math.inf
            x[3, 7], x[3, 3] = math.nan, math.nan
            logprob, entropy, ids, lps = eng.token_logprobs(x, t, 12)
            assert eng.device_status() == a3.DEV_NONFINITE_SCORE
            assert logprob[:4].isnan().all() and entropy[:4].isnan().all() and lps[:4].isnan().all()
            clean = x.clone()
            clean[0, V // 2] = -math.inf
            clean[3] = torch.where(x[3].isnan(), -math.inf, x[3])
            assert torch.equal(ids[0].long(), R.ranked(clean[:1], 12)[0])  # NaN is not among the first
            assert ids[1, 0] == V - 1 and ids[2].tolist() == list(range(12))
            assert ids[3].tolist() == [0, 1, 2, 4, 5, 6] + list(range(8, 14))
            check(eng, x[4:], t[4:], 12)
    x = torch.full((1, 6), -math.inf, device=DEV)
    x[0, 1], x[0, 4] = math.nan, 2.0
    assert eng.token_logprobs(x, None, 6)[2].tolist() == [[4, 0, 2, 3, 5, 1]]
    assert eng.device_status() == a3.DEV_NONFINITE_SCORE


def test_targets_beside_the_vocabulary(a3, eng):
    x, t = rows(4, 300, torch.float32, 8)
    t[0], t[1], t[2] = -1, -100, 299
    check(eng, x, t, 0)
    t[3] = 300
    logprob, entropy, _, _ = eng.token_logprobs(x, t)
    assert eng.device_status() == a3.DEV_BAD_POSITION
    assert logprob[3].isnan() and (logprob[:2] == 0).all() and logprob[2].isfinite() and entropy.isfinite().all()
    none = eng.token_logprobs(x[:0], t[:0], 3)
    assert none[0].shape == (0,) and none[2].shape == (0, 3)


def test_repeats_bit_for_bit_and_captured(eng):
    x, t = rows(33, 50000, torch.bfloat16, 9)
    eng.token_logprobs(x, t, 8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = eng.token_logprobs(x, t, 8)
    for seed in (10, 11):
        y, u = rows(33, 50000, torch.bfloat16, seed)
        x.copy_(y), t.copy_(u)
        graph.replay()
        for a, b in zip(out, eng.token_logprobs(x, t, 8)):
            assert torch.equal(a, b)
        check(eng, x, t, 8)


def test_refusals_of_the_library(a3, eng):
    lib, x = a3._load(), torch.zeros((2, 64), device=DEV)
    f, i, t = torch.zeros((2, 64), device=DEV), torch.zeros((2, 64), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    p = lambda v: v.data_ptr()  # noqa: E731
    good = dict(x=p(x), t=p(t), lp=p(f), e=p(f), ids=p(i), lps=p(f), stride=64, type=0, M=2, V=64, n=3)
    call = lambda h=eng._h, **kw: lib.a3_token_logprobs(h, R.LOGIT_ROWS.pack(*[0 if v is None else v for v in {**good, **kw}.values()]), 0)  # noqa: E731
    assert lib.a3_token_logprobs(eng._h, None, 0) == -1
    a3.launch_count(reset=True)
    for kw in [dict(h=None), dict(x=None), dict(x=p(x) + 2), dict(stride=63), dict(M=-1), dict(V=0), dict(t=None), dict(lp=None), dict(n=-1),
               dict(n=0), dict(ids=None), dict(lps=None), dict(V=2), dict(stride=1 << 41)]:
        assert call(**kw) == -1, kw
    assert call(type=3) == -2 and call(type=-1) == -2 and call(n=33) == -2 and call(M=0) == 0
    assert a3.launch_count() == 0
    assert call() == 0 and call(e=None) == 0 and call(n=0, ids=None, lps=None) == 0 and call(t=None, lp=None) == 0
    assert eng.device_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,V", [(1, 128256), (40, 40000), (400, 4096), (400, 40000), (310, 128256)])
def test_two_tokens_are_left(eng, dtype, M, V):
    """Two finite logits `gap` apart, as a grammar leaves them: neighbours, and as far apart as the elements of one thread lie, with the
    first elements in front of the first 16-byte boundary or not.  With s = exp(-gap): log p = -log1p(s), entropy log1p(s) + gap s / (1 + s).
    The exponential's argument is rounded twice (2^-24 of gap each), the exponential and log1p are off by 2^-22 each, the sums here by 2^-22."""
    size = torch.finfo(dtype).bits // 8
    for first in (0, 1):
        wide = torch.full((M, V + 16), -math.inf, dtype=dtype, device=DEV)
        x = wide[:, first:first + V]
        for apart in [1, 3] + [t * 16 // size for t in (64, 128, 256)]:
            for at, gap in ((0, 18.0), (8, 16.75), (1027, 24.5), (V - 1 - apart, 40.0), (V // 2, 9.0)):
                if at + apart >= V:
                    continue
                for top in (at, at + apart):  # the larger one first, and last
                    wide.fill_(-math.inf)
                    x[:, at] = x[:, at + apart] = 2.0 - gap
                    x[:, top] = 2.0
                    t = torch.full((M,), top, dtype=torch.int32, device=DEV)
                    logprob, entropy, ids, lps = eng.token_logprobs(x, t, 2)
                    s = math.exp(-gap)
                    want, h = -math.log1p(s), math.log1p(s) + gap * s / (1 + s)
                    rel = gap * 2.0 ** -23 + 2.0 ** -20
                    assert ((logprob.double() - want).abs() <= rel * -want).all(), (first, apart, at, gap, logprob[0].item(), want)
                    assert ((entropy.double() - h).abs() <= rel * h).all(), (first, apart, at, gap, entropy[0].item(), h)
                    assert torch.equal(logprob, lps[:, 0]) and (ids == torch.tensor([top, 2 * at + apart - top], device=DEV)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,V", [(1, 512), (400, 512), (400, 20000), (300, 128256), (2, 128256)])
def test_one_token_above_a_full_row(eng, dtype, M, V):
    """One logit `up` above the largest of the others, from hardly likelier to certain.  What the others sum up to is a sum of V / 64 terms at
    most in a thread, each added with 2^-24 of the sum so far.  Where the largest one's 1 is among them, what they add is an eighth of it at
    least: 9 x 2^-24 for each, relative to the others alone."""
    x, t = rows(M, V, dtype, M + V, std=1.0)
    at = t.long()[:, None]
    for up in (0.0, 1.0, 3.0, 6.0, 9.0, 14.0, 20.0, 30.0, 50.0):
        y = x.clone()
        y.scatter_(1, at, (x.float().amax(1, keepdim=True) + up).to(dtype))
        logprob, entropy, _, _ = eng.token_logprobs(y, t, 1)
        d = y.double() - y.double().gather(1, at)
        e = d.exp().scatter(1, at, 0.0)
        s = e.sum(1)
        h = torch.log1p(s) - (e * d).sum(1) / (1 + s)
        rel = (up + 12) * 2.0 ** -23 + 2.0 ** -20 + 9 * (V / 64 + 64) * 2.0 ** -24
        assert ((logprob.double() + torch.log1p(s)).abs() <= rel * s).all(), (up, ((logprob.double() + torch.log1p(s)) / s).abs().max().item())
        assert ((entropy.double() - h).abs() <= rel * (h + s)).all(), (up, ((entropy.double() - h) / h).abs().max().item())


def test_a_shift_of_all_logits_costs_no_time(eng):
    """The alternatives of rows far from zero are found as fast as those of rows around it (once, 1 000 in the logits took several times as long).
    The values of both rows are multiples of 2^-10, so the shift loses nothing."""
    def elapsed(x, n):
        best = []
        for _ in range(7):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(20):
                eng.token_logprobs(x, None, n)
            b.record()
            torch.cuda.synchronize()
            best.append(a.elapsed_time(b))
        return min(best)

    for dtype, shift, M, V in ((torch.float32, 1000.0, 1, 128256), (torch.float32, 6000.0, 300, 30000), (torch.float16, 1000.0, 300, 30000), (torch.float32, 6000.0, 64, 3000)):
        x, _ = rows(M, V, torch.float32, 12, std=2.5)
        x = ((x * 1024).round() / 1024).to(dtype)
        y = (x.float() + shift).to(dtype)
        x = (y.float() - shift).to(dtype)
        check(eng, y, None, 20)
        check(eng, y[:1, 1:4097], None, 20)  # threads without a vector where V allows it
        assert torch.equal(eng.token_logprobs(x, None, 20)[2], eng.token_logprobs(y, None, 20)[2])
        base, shifted = elapsed(x, 20), elapsed(y, 20)
        print(f"{dtype} {M} x {V}: {base / 20 * 1e3:.1f} us, shifted by {shift:.0f} {shifted / 20 * 1e3:.1f} us")
        assert shifted <= 2.5 * base, (dtype, M, V, base, shifted)
