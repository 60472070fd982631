"""Sampling on the device against the definition in 64 bits: the same token
for every row (a random number within rounding of a border, 1e-9 of the rows'
unit interval at most, would be the only other possibility)."""
import numpy as np
import pytest
import torch

from paper_2608_10139_amd.device import sample

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def reference(x, u, T, top_k=0, top_p=1.0, min_p=0.0):
    """x: one row, float64."""
    x = np.where(np.isnan(x), -np.inf, x)
    m = x.max()
    if m == -np.inf:
        return 0
    if T == 0:
        return int(np.argmax(x))
    with np.errstate(invalid="ignore"):
        w = np.where(x == m, 1.0, np.exp((x - m) / T))
    order = np.argsort(-x, kind="stable")
    n = min(top_k or len(x), int(np.sum(x > -np.inf)))
    c = np.cumsum(w[order[:n]])
    if top_p < 1:
        n = min(n, 1 + int(np.sum(c < top_p * c[-1])))
    kept = np.sort(order[:n])
    kept = kept[w[kept] >= min_p]
    c = np.cumsum(w[kept])
    i = int(np.sum(c <= u * c[-1])) if u < 1 else len(kept)
    return int(kept[min(i, len(kept) - 1)])


def check(x, u, **kw):
    T = kw.pop("temperature", 1.0)
    got = sample(x, u, temperature=T, **kw).cpu().numpy()
    xs = x.double().cpu().numpy()
    us = np.zeros(len(xs)) if u is None else u.double().cpu().numpy()
    want = np.array([reference(r, a, T, **kw) for r, a in zip(xs, us)])
    np.testing.assert_array_equal(got, want)


def rows(n, V, seed, dtype=torch.float32, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn(n, V, generator=g)
    x.scatter_add_(1, torch.randint(0, V, (n, 6), generator=g), 4.0 * torch.rand(n, 6, generator=g))
    return x.to(dtype).cuda(), torch.rand(n, generator=g).cuda()


FILTERS = [dict(), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(top_p=0.3, top_k=40), dict(min_p=0.05),
           dict(top_k=200, top_p=0.95, min_p=0.01), dict(top_p=1e-9), dict(min_p=1.0), dict(top_k=10 ** 6)]


@pytest.mark.parametrize("kw", FILTERS, ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 63, 1000, 32000, 40001])
def test_sample_against_the_definition(V, dtype, kw):
    say("case: sample", V, dtype, kw)
    for T in (1.0, 0.25, 3.0):
        x, u = rows(12, V, V + int(8 * T), dtype)
        check(x, u, temperature=T, **kw)


def test_borders_of_the_random_number():
    say("case: u at its borders")
    x, _ = rows(6, 500, 3)
    u = torch.tensor([0.0, 1.0, 2.0, float("nan"), 1.0 - 2.0 ** -24, -0.5], device="cuda")
    got = sample(x, u, top_k=20).cpu().numpy()
    for r in range(6):
        kept = np.sort(np.argsort(-x[r].double().cpu().numpy(), kind="stable")[:20])
        assert got[r] == (kept[0] if r in (0, 5) else kept[-1])


def test_equal_logits_are_taken_from_the_lowest_ids():
    say("case: ties")
    x = torch.zeros(40, 3001, device="cuda")
    u = torch.rand(40, device="cuda")
    for kw in (dict(), dict(top_k=7), dict(top_p=0.01), dict(top_k=100, top_p=0.5), dict(min_p=1.0)):
        check(x, u, **kw)
    y = torch.randint(-3, 3, (40, 3001), device="cuda").float()
    y[:, 5] = -0.0
    for kw in (dict(top_k=700), dict(top_p=0.6), dict(top_k=701, top_p=0.99)):
        check(y, u, **kw)


def test_infinities_and_nan():
    say("case: infinities and NaN")
    x, u = rows(10, 777, 4)
    x[0] = float("-inf")
    x[1] = float("nan")
    x[2, ::2] = float("-inf")
    x[3, 1::3] = float("nan")
    x[4, 100:103] = float("inf")
    x[5] = float("-inf")
    x[5, 700] = -3.0
    x[6] = torch.finfo(torch.float32).min
    x[7, 3] = torch.finfo(torch.float32).max
    x[8, 9], x[8, 10] = 1e30, -1e30
    x[9] *= 1e-30
    for kw in (dict(), dict(top_k=5), dict(top_p=0.7), dict(top_k=600, top_p=0.9, min_p=0.001), dict(temperature=0.0)):
        check(x, u, **kw)


def test_greedy_needs_no_random_numbers():
    say("case: temperature 0")
    x, _ = rows(33, 4096, 5, torch.float16)
    check(x, None, temperature=0.0)
    check(x, None, temperature=0.0, top_k=3, top_p=0.5)


def test_strided_rows_and_repeats():
    """Rows of a wider, unaligned matrix; twice the same call, and rows one by one."""
    say("case: strides")
    for dtype in (torch.float32, torch.bfloat16):
        wide, u = rows(9, 2003, 6, dtype)
        x = wide[:, 1:1990]
        check(x, u, top_k=30, top_p=0.8)
        a = sample(x, u, top_p=0.9)
        assert torch.equal(a, sample(x, u, top_p=0.9))
        assert torch.equal(a, torch.cat([sample(x[i:i + 1], u[i:i + 1], top_p=0.9) for i in range(9)]))
    assert sample(wide[:0], u[:0]).shape == (0,)


def test_extreme_temperatures():
    say("case: temperatures")
    x, u = rows(8, 5000, 7)
    for T in (1e-6, 1e-3, 50.0, 1e6, 1e30):
        check(x, u, temperature=T, top_k=1000)
        check(x, u, temperature=T, top_p=0.9)


@pytest.mark.parametrize("V", [131071, 262144])
def test_large_vocabularies(V):
    say("case: vocabulary", V)
    x, u = rows(5, V, 8, torch.bfloat16)
    for kw in (dict(), dict(top_k=1000, top_p=0.95), dict(top_p=0.9, min_p=0.002)):
        check(x, u, temperature=1.3, **kw)


def test_frequencies():
    """60,000 draws of a row: counts within five standard deviations of the kept distribution."""
    say("case: frequencies")
    x, _ = rows(1, 50, 9)
    n = 60000
    u = torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    got = np.bincount(sample(x.expand(n, 50), u, top_k=20).cpu().numpy(), minlength=50)
    w = np.exp(x[0].double().cpu().numpy())
    keep = np.argsort(-w)[:20]
    p = np.zeros(50)
    p[keep] = w[keep] / w[keep].sum()
    assert np.all(got[p == 0] == 0)
    assert np.all(np.abs(got - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 1)


def test_captured_sampling_replays():
    say("case: captured sampling")
    x, u = rows(20, 3000, 10)
    out = torch.zeros(20, dtype=torch.int32, device="cuda")
    sample(x, u, top_p=0.9, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sample(x, u, top_p=0.9, top_k=300, out=out)
    for s in range(4):
        y, w = rows(20, 3000, 20 + s)
        x.copy_(y)
        u.copy_(w)
        g.replay()
        want = sample(y, w, top_p=0.9, top_k=300)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("n,V", [(6, 131071), (700, 6000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_hundreds_of_kept_tokens(n, V, dtype):
    say("case: hundreds kept", n, V, dtype)
    x, u = rows(n, V, 11, dtype)
    for k in (129, 500, 1000):
        check(x, u, top_k=k)
        check(x, u, top_k=k, top_p=0.97, temperature=2.0)
        check(x, u, top_k=k, top_p=0.9, min_p=0.01, temperature=2.0)


@pytest.mark.parametrize("n", [4, 600])
def test_kept_tokens_that_lie_or_weigh_alike(n):
    # ids next to each other in a large vocabulary, equal logits, two levels
    say("case: alike", n)
    V = 1 << 17
    x, u = torch.full((n, V), -30.0, device="cuda"), torch.rand(n, generator=torch.Generator().manual_seed(12)).cuda()
    g = torch.Generator("cuda").manual_seed(13)
    x[:, 70000:70900] = torch.randn(n, 900, device="cuda", generator=g)
    x[::2, 70000:70900] = x[::2, 70000:70900].round()
    check(x, u, top_k=700)
    check(x, u, top_k=600, top_p=0.8)
    x[:, 70000:70900] = 1.0
    check(x, u, top_k=800, top_p=0.5)
    x[:, 100:400] = 1.5
    check(x, u, top_k=500, top_p=0.9)


def test_more_rows_than_workgroups():
    say("case: 70,000 rows")
    x, u = rows(700, 60, 14)
    x, u = x.repeat(100, 1), torch.rand(70000, generator=torch.Generator().manual_seed(15)).cuda()
    for kw in (dict(), dict(top_k=7), dict(top_p=0.8, min_p=0.01)):
        got = sample(x, u, **kw)
        want = torch.cat([sample(x[i:i + 700], u[i:i + 700], **kw) for i in range(0, 70000, 700)])
        assert torch.equal(got, want)
        check(x[-40:], u[-40:], **kw)


@pytest.mark.parametrize("n,ks", [(6, (1500, 2000, 4000, 4096, 5000)), (300, (2000, 4000)), (700, (500, 2000))])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_top_k_of_more_candidates_than_are_gathered(n, ks, dtype):
    """Thousands of tokens pass top-k's first bound: the steps start over on the whole row."""
    say("case: top-k of thousands", n, ks, dtype)
    x, u = rows(n, 20000, 17, dtype)
    for k in ks:
        check(x, u, top_k=k)
        check(x, u, top_k=k, top_p=0.97, min_p=1e-4, temperature=2.0)


@pytest.mark.parametrize("n", [2, 256, 1100])
def test_border_of_thousands_of_equal_logits_in_many_rows(n):
    """Levels of more equal logits than are gathered, on as many rows as workgroups are resident: the same tokens each time."""
    say("case: thousands of equal logits", n)
    g = torch.Generator().manual_seed(18)
    x = torch.randint(-2, 2, (n, 9001), generator=g).float()
    x[::3] = 0.5
    x, u = x.cuda(), torch.rand(n, generator=g).cuda()
    for k in (7, 500, 2600):
        got = sample(x, u, top_k=k)
        assert all(torch.equal(got, sample(x, u, top_k=k)) for _ in range(5))
        check(x[-24:], u[-24:], top_k=k)
        want = [reference(r, a, 1.0, k) for r, a in zip(x[:24].double().cpu().numpy(), u[:24].double().cpu().numpy())]
        np.testing.assert_array_equal(got[:24].cpu().numpy(), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_temperatures_up_to_the_largest(dtype):
    # every finite logit weighs the same; -infinity and NaN nothing, and no id is past the row's end
    say("case: temperatures up to the largest", dtype)
    for V in (5, 777, 3001):
        x, u = rows(64, V, 16, dtype)
        x[:, ::3] = float("-inf")
        x[1::2, 1::3] = float("nan")
        u[:4] = torch.tensor([0.0, 0.5, 0.999, 1.0 - 2.0 ** -24])
        for T in (1e200, 1e290, 1e300, 1.7976931348623157e308):
            for kw in (dict(), dict(top_k=300), dict(top_p=0.9), dict(min_p=0.5)):
                check(x, u, temperature=T, **kw)
