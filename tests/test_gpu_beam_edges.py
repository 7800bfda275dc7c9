"""Beam selection and reordering at the ends of what the documentation allows."""
import math

import pytest
import torch

from test_gpu_beam import check_select, logits_of
from paper_2410_18517_b200 import KvsError, SharedKVCache
from paper_2410_18517_b200 import binding as kb
from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_over_the_largest_vocabulary(dtype):
    """One row of 2^31 - 1 logits (the bound on n_beams * vocab): the last segment ends where 31 bits do."""
    cache = SharedKVCache(1, 1, 1, 64, 1, 1, "bf16")
    V = 2 ** 31 - 1
    x = torch.zeros(1, V, dtype=DT[dtype], device="cuda")
    best = {V - V % 2 ** 23: 6.0, V - 1: 5.0, V - 2: 4.0, 0: 3.0}
    for at, logit in best.items():
        x[0, at] = logit
    s, t, p = cache.beam_select(x, torch.zeros(1, device="cuda"), 1, 6)
    del x
    assert t[0].tolist() == list(best) + [1, 2] and p[0].tolist() == [0] * 6
    lse = math.log(V - 4 + sum(math.exp(v) for v in best.values()))
    want = torch.tensor([v - lse for v in best.values()] + [-lse] * 2, dtype=torch.float64)
    # sums of ones are exact up to 2^24; rescaled a few times per thread that holds one of the four: 2^-22 each, and the
    # score's own rounding (2^-24 of 21.5)
    assert float((s[0].cpu().double() - want).abs().max()) < 16 * 2.0 ** -22
    assert cache.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 6000, 70000])
def test_select_logits_that_differ_by_less_than_scores_show(dtype, V):
    """Logits of a few 1e-20 apart: their fp64 scores are equal.  A beam's go by the logit, beams by their number, whatever
    n_out is: fewer continuations are the first of more."""
    W = 3
    cache = SharedKVCache(1, 1, 1, 64, 2 * W, 1, "bf16")
    x = torch.zeros(2 * W, V)
    for b in range(2 * W):
        for i, at in enumerate((V - 1, V // 2, 7 + b, V // 3)):
            x[b, at] = (i % 3 + 1 + b) * 1e-20 * (-1 if i == 2 else 1)
    x[1, 3], x[4] = 2.0, -math.inf               # a beam with a score that shows, a beam without candidates
    x = x.to(DT[dtype])
    scores = torch.tensor([-1.0, -8.0, -1.0, -0.5, 0.0, -0.5])
    scores[1] = -1.0 + float(torch.logsumexp(x[1].double(), 0) - math.log(V)) - 2.0
    want = []
    for r in range(2):
        every = []
        for w in range(W):
            row = x[r * W + w].double()
            top = row.max()
            base = float(scores[r * W + w]) - float((row - top).exp().sum().log())
            total = base + (row - top)
            every += [(-float(total[v]), w, -float(row[v]), v) for v in range(V) if math.isfinite(float(total[v]))]
        want.append([(v, r * W + w) for _, w, _, v in sorted(every)[:64]])
    got = {}
    for K in (64, 40, 17, 16, 5, 2, 1):
        _, t, p = cache.beam_select(x.cuda(), scores.cuda(), W, K)
        got[K] = [list(zip(t[r].tolist(), p[r].tolist())) for r in range(2)]
        if K == 64:
            assert got[K][1] == want[1]
        for r in range(2):
            assert got[K][r] == got[64][r][:K], (K, r)
    assert cache.device_status() == 0


def test_select_takes_as_many_rows_as_the_header_says():
    """65535 rows, and not one more, though the cache has room for them."""
    cache = SharedKVCache(1, 1, 1, 64, 65536, 1, "bf16")
    x = torch.zeros(65536, 2, device="cuda")
    x[:, 1] = torch.arange(65536, device="cuda") * 1e-4 - 3
    scores = torch.zeros(65536, device="cuda")
    s, t, p = cache.beam_select(x[:65535], scores[:65535], 1, 2)
    want = x[:65535].double().log_softmax(-1).sort(dim=-1, descending=True, stable=True)
    assert torch.equal(t.long(), want.indices) and torch.equal(p[:, 0], torch.arange(65535, device="cuda").int())
    # one exponential below 1 (2^-22; its argument, at most 3.6, rounded twice: 7.2 * 2^-24), a sum (2^-24), and the rounding of
    # the score, below 4.3 in size (4.3 * 2^-24)
    assert float((s.double() - want.values).abs().max()) < 17 * 2.0 ** -24
    with pytest.raises(KvsError) as e:
        cache.beam_select(x, scores, 1, 2)
    assert e.value.status == kb.KVS_ERR_INVALID_ARG
    assert cache.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_of_as_many_requests_as_the_device_has_sms_and_more(dtype):
    n = torch.cuda.get_device_properties(0).multi_processor_count
    cache = SharedKVCache(1, 1, 1, 64, 2 * (2 * n + 1), 1, "bf16")
    for R in (n - 1, n, n + 1, 2 * n + 1):
        x = torch.randn(2 * R, 600, device="cuda", generator=torch.Generator(device="cuda").manual_seed(R)).to(DT[dtype])
        x[:, 77] = x[:, 5]                       # a tie in every row
        scores = -torch.rand(2 * R, device="cuda", generator=torch.Generator(device="cuda").manual_seed(R + 1))
        s, t, p = cache.beam_select(x, scores, 2, 20)
        total = (scores.double()[:, None] + x.double().log_softmax(-1)).view(R, -1)
        want = total.sort(dim=-1, descending=True, stable=True)
        assert float((s.double() - want.values[:, :20]).abs().max()) < 2.0 ** -22 + 32 * 2.0 ** -24 + 16 * 2.0 ** -24
        # the order within a beam is exact; between beams scores may be as close as their error
        chosen = total.gather(1, (t + 600 * (p - 2 * torch.arange(R, device="cuda").int()[:, None])).long())
        assert float((chosen - want.values[:, :20]).abs().max()) < 2.0 ** -21 + 64 * 2.0 ** -24
        assert all(len(set(zip(t[r].tolist(), p[r].tolist()))) == 20 for r in range(0, R, 37))
    assert cache.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [24, 25])
def test_select_either_way_to_the_threshold(dtype, K):
    """Up to 24 continuations the threshold comes from the maxima of four threads, above from each thread's."""
    cache = SharedKVCache(1, 1, 1, 64, 6, 1, "bf16")
    for V in (900, 40001):
        check_select(cache, logits_of(V + K, dtype, 6, V), -torch.arange(6.0).cuda() / 3, 3, K)
    check_select(cache, torch.full((6, 3000), 0.5, dtype=DT[dtype], device="cuda"), torch.zeros(6).cuda(), 3, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V", [(800, 1000), (800, 131072), (4, 1000003)])
def test_select_logarithms_are_good_to_a_few_1e_7(dtype, rows, V):
    """The scores of each row's best token against float64, beside the score's own rounding.  Bound: a term's exponential (2^-22),
    and for each of the 8 levels at which partial sums meet within a block the rescaling of the smaller one, at most half of
    the two (2^-22 of it), and the addition (2^-24).  A thread's own additions, up to 16 turns of 32, err either way and stay
    below what the first term leaves; a sum in order over the row would not."""
    cache = SharedKVCache(1, 1, 1, 64, rows, 1, "bf16")
    x = (torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V)) * 4).to(DT[dtype])
    s, t, _ = cache.beam_select(x, torch.zeros(rows, device="cuda"), 1, 1)
    for i in range(0, rows, 100):
        exact = x[i:i + 100].double().log_softmax(-1).gather(1, t[i:i + 100].long())
        off = (s[i:i + 100].double() - exact).abs() - 2.0 ** -24 * exact.abs()
        assert float(off.max()) < 2.0 ** -22 + 8 * (2.0 ** -23 + 2.0 ** -24)
        if dtype == "f32":                       # (bf16 logits tie)
            assert torch.equal(t[i:i + 100, 0].long(), x[i:i + 100].argmax(-1))
