"""The 8-bit key/value cache: written and read back, and attention over it,
against a plain form in 64 bits.

Read-back is exact: the whole numbers and scales are defined step by step.
Attention: weights reach the products in 16 bits (half a step each, u_p: fp16
2^-11; a bf16 cache's tail 2^-8) while their sum stays in 32, so the output
moves by at most u_p max|v|; scores of up to 2^6 in 32 bits move a weight by
less than 2^-15, 2^-14 with the sum's; the output's own rounding is u_out |out|."""
import numpy as np
import pytest
import torch

from paper_2608_10139_amd import binding as B
from paper_2608_10139_amd.device import DeviceKvCache
from tests import _kv_ref as R

pytestmark = pytest.mark.gpu
BLOCK = R.BLOCK
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def say(*a):
    print(*a, flush=True)


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).cuda()


def starts(n):
    out = np.zeros(len(n) + 1, np.int64)
    out[1:] = np.cumsum(n)
    return out


class Case:
    """Sequences of the given final lengths in one cache: their rows (host and
    device), blocks in a shuffled order, tails too."""

    def __init__(self, lens, heads, kv, hd, dtype, seed, paged=True, spare=0):
        r = np.random.default_rng(seed)
        self.lens, self.heads, self.kv, self.hd, self.dtype = np.asarray(lens), heads, kv, hd, dtype
        n = len(lens)
        size = np.exp(0.5 * r.standard_normal((1, kv, hd)))
        self.k = [torch.tensor(r.standard_normal((L, kv, hd)) * size, dtype=dtype) for L in lens]
        self.v = [torch.tensor(r.standard_normal((L, kv, hd)) * r.uniform(0.1, 4.0, (1, kv, 1)), dtype=dtype) for L in lens]
        self.q = [torch.tensor(r.standard_normal((L, heads, hd)) * 1.5, dtype=dtype) for L in lens]
        blocks = (self.lens + BLOCK - 1) // BLOCK + spare
        self.start = starts(blocks)
        nb = int(self.start[-1])
        self.blk_start = i32(self.start)
        self.blk_ids = i32(r.permutation(nb)) if paged else None
        self.tail_ids = i32(r.permutation(n)) if paged else None
        self.cache = DeviceKvCache(max(nb, 1), max(n, 1), kv, hd, dtype)

    def batch(self, length, new, single=False):
        length, new = np.asarray(length), np.asarray(new)
        return self.cache.batch(i32(length), self.blk_start, int(max(self.lens.max(initial=0), 1)),
                                cu=None if single else i32(starts(new)), blk_ids=self.blk_ids, tail_ids=self.tail_ids)

    def rows(self, what, length, new):
        """The last new[i] of the first length[i] rows of every sequence, in a wider matrix's columns."""
        x = getattr(self, what)
        parts = [x[i][L - m:L] for i, (L, m) in enumerate(zip(length, new))]
        flat = torch.cat(parts) if parts else x[0][:0]
        n, h = flat.shape[0], flat.shape[1]
        wide = torch.full((n, (h + 2) * self.hd), 7.0, dtype=self.dtype)
        wide[:, self.hd:(h + 1) * self.hd] = flat.reshape(n, -1)
        return wide.cuda()[:, self.hd:(h + 1) * self.hd].unflatten(1, (h, self.hd))

    def write(self, length, new, single=False):
        self.cache.write(self.batch(length, new, single), self.rows("k", length, new), self.rows("v", length, new))

    def ok(self):
        assert int(self.cache.status.item()) == 0

    def held(self, i, L=None):
        """What the cache should hold of sequence i once L tokens are in: (k, v) float64."""
        L = self.lens[i] if L is None else L
        return tuple(R.held(x[i][:L].float().numpy()) for x in (self.k, self.v))

    def check_read(self, length):
        k, v = self.cache.read(self.batch(length, length))
        at = starts(length)
        for i, L in enumerate(length):
            for got, want in zip((k, v), self.held(i, L)):
                want = torch.from_numpy(want).to(torch.float32).to(self.dtype)   # exact in 32 bits, rounded once
                assert torch.equal(got[at[i]:at[i + 1]].cpu(), want), f"sequence {i} of {L} tokens"
        self.ok()

    def check_attend(self, length, new, out, out_dtype=None):
        u_p, u_o = U[self.dtype], U[out_dtype or self.dtype]
        at = starts(new)
        out = out.double().cpu().numpy()
        for i, (L, m) in enumerate(zip(length, new)):
            if m == 0:
                continue
            want, top = R.attend(self.q[i][L - m:L].float().numpy(), *self.held(i, L), np.arange(L - m, L))
            tol = (u_p + 2.0 ** -14) * top[:, :, None] + u_o * np.abs(want) + 1e-7
            err = np.abs(out[at[i]:at[i + 1]] - want)
            assert np.all(err <= tol), f"sequence {i} of {L} tokens: {np.nanmax(err / tol):.2f} of the bound"
        self.ok()


LENS = [1, 31, 32, 33, 0, 64, 65, 100, 257, 2]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kv,hd", [(8, 64), (3, 128), (1, 64)])
def test_written_rows_read_back(kv, hd, dtype):
    say("case: write and read", kv, hd, dtype)
    c = Case(LENS, kv, kv, hd, dtype, 1)
    c.write(c.lens, c.lens)
    c.check_read(c.lens)


@pytest.mark.parametrize("hd", [64, 128])
def test_what_is_held_does_not_depend_on_the_calls(hd):
    """Rows in pieces of many sizes, then one by one: the same bytes as at once."""
    say("case: pieces", hd)
    lens = np.array([97, 160, 64, 33, 70])
    one, many = (Case(lens, 2, 2, hd, torch.float16, 2, spare=s) for s in (0, 0))
    one.write(lens, lens)
    held = np.zeros(len(lens), np.int64)
    r = np.random.default_rng(3)
    while np.any(held < lens - 3):
        new = np.minimum(r.integers(0, 70, len(lens)), np.maximum(lens - 3 - held, 0))
        held = held + new
        many.write(held, new)
    for _ in range(3):
        held = held + 1
        many.write(held, np.ones_like(held), single=True)
    for a, b in ((one.cache.k, many.cache.k), (one.cache.v, many.cache.v), (one.cache.k_scale, many.cache.k_scale),
                 (one.cache.v_scale, many.cache.v_scale)):
        assert torch.equal(a, b)
    many.check_read(lens)


def test_scales_of_extreme_blocks():
    """Zeros, the largest numbers, subnormals, one large value among small ones, infinity and NaN."""
    say("case: extreme blocks")
    for dtype, big in ((torch.float16, 65504.0), (torch.bfloat16, 3.0e38)):
        c = Case([7 * 32], 1, 1, 64, dtype, 4, paged=False)
        k = c.k[0]
        k[:32] = 0.0
        k[32:64] = (k[32:64].double() / k[32:64].double().abs().max() * big).to(dtype)
        k[64:96] *= 2.0 ** -22 if dtype == torch.float16 else 2.0 ** -130
        k[96:128] *= 1e-3
        k[100, 0, 5] = 500.0
        k[128 + 3, 0, 9] = float("inf")
        k[160 + 31, 0, 63] = float("nan")
        c.write(c.lens, c.lens)
        got = c.cache.read(c.batch(c.lens, c.lens))[0].cpu()
        want = torch.from_numpy(c.held(0)[0]).to(torch.float32).to(dtype)
        assert torch.equal(got[:128], want[:128]) and torch.equal(got[192:], want[192:])
        assert torch.isnan(got[128:192]).all()
        x = k[:128].double()
        step = x.reshape(4, -1).abs().max(1).values.repeat_interleave(32)[:, None, None] / 127
        lost = 2.0 ** -81 if dtype == torch.bfloat16 else 0.0
        assert torch.all((got[:128].double() - x).abs() <= 0.5001 * step + U[dtype] * x.abs() + U[dtype] * step + lost + 2.0 ** -25)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv,hd", [(8, 8, 64), (32, 8, 64), (6, 2, 128), (20, 1, 64), (16, 1, 128)])
def test_attention_of_single_tokens(heads, kv, hd, dtype):
    say("case: single tokens", heads, kv, hd, dtype)
    c = Case([1, 2, 31, 32, 33, 64, 95, 511, 512, 513, 1100], heads, kv, hd, dtype, 5)
    c.write(c.lens, c.lens)
    one = np.ones_like(c.lens)
    out = c.cache.attend(c.batch(c.lens, one, single=True), c.rows("q", c.lens, one))
    c.check_attend(c.lens, one, out)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv,hd", [(8, 8, 64), (24, 8, 128), (8, 1, 64)])
def test_attention_of_several_tokens(heads, kv, hd, dtype):
    say("case: several tokens", heads, kv, hd, dtype)
    c = Case([1, 5, 33, 64, 130, 0, 200, 620], heads, kv, hd, dtype, 6)
    new = np.array([1, 5, 2, 64, 17, 0, 33, 40])
    c.write(c.lens, c.lens)
    out = c.cache.attend(c.batch(c.lens, new), c.rows("q", c.lens, new))
    c.check_attend(c.lens, new, out)


@pytest.mark.parametrize("out_dtype", [torch.float16, torch.bfloat16])
def test_attention_output_type(out_dtype):
    say("case: output type", out_dtype)
    c = Case([40, 7], 4, 2, 64, torch.float16, 7)
    c.write(c.lens, c.lens)
    new = np.array([1, 1])
    out = c.cache.attend(c.batch(c.lens, new), c.rows("q", c.lens, new), out_dtype=out_dtype)
    assert out.dtype == out_dtype
    c.check_attend(c.lens, new, out, out_dtype)


def test_empty_slots_and_rows_behind_the_last():
    say("case: empty slots")
    c = Case([40, 0, 64, 0], 4, 2, 64, torch.float16, 8)
    one = np.ones(4, np.int64)
    c.write(c.lens, c.lens)
    before = [t.clone() for t in (c.cache.k, c.cache.tail)]
    q = torch.randn(4, 4, 64, device="cuda").half()
    q[0], q[2] = c.q[0][39], c.q[2][63]
    out = torch.full((6, 4, 64), 5.0, dtype=torch.float16, device="cuda")
    c.cache.attend(c.batch(c.lens, one, single=True), q, out=out[:4])
    assert torch.all(out[1] == 0) and torch.all(out[3] == 0) and torch.all(out[4:] == 5.0)
    c.check_attend(c.lens, [1, 0, 1, 0], out[[0, 2]])
    # an empty slot writes nothing; no sequence, no row: nothing at all
    c.cache.write(c.batch([0, 0, 0, 0], one, single=True), q[:, :2], q[:, :2])
    c.cache.write(c.batch([0, 0, 0, 0], [0, 0, 0, 0]), q[:0, :2], q[:0, :2])
    for a, b in zip(before, (c.cache.k, c.cache.tail)):
        assert torch.equal(a, b)
    none = DeviceKvCache(0, 0, 2, 64)
    b = none.batch(i32([]), i32([0]), 0)
    assert none.attend(b, q[:0]).shape == (0, 4, 64) and none.read(b)[0].shape == (0, 2, 64)
    c.ok()


def test_long_sequence_alone_and_among_others_gives_the_same_bits():
    """Split between workgroups where it is alone, walked by one among 1,100 others."""
    say("case: long sequence alone and in a batch")
    n = 1100
    lens = np.full(n, 3)
    lens[7] = 3000
    c = Case(lens, 3, 1, 64, torch.float16, 9)
    c.write(lens, lens)
    one = np.ones(n, np.int64)
    b = c.batch(lens, one, single=True)
    assert B.aiq_kv_attend_workspace_size(c.cache.struct, b.struct, 3) == 0
    many = c.cache.attend(b, c.rows("q", lens, one))
    s, e = c.start[7], c.start[8]
    alone = c.cache.batch(i32([3000]), i32([0, e - s]), 3000, blk_ids=c.blk_ids[s:e].contiguous(),
                          tail_ids=c.tail_ids[7:8].contiguous())
    assert B.aiq_kv_attend_workspace_size(c.cache.struct, alone.struct, 3) > 0
    out = c.cache.attend(alone, c.q[7][-1:].cuda())
    assert torch.equal(out[0], many[7])
    want, top = R.attend(c.q[7][-1:].float().numpy(), *c.held(7), [2999])
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= (2.0 ** -11 + 2.0 ** -14) * top[:, :, None] + 2.0 ** -11 * np.abs(want))
    c.ok()


def test_infinity_and_nan_behind_a_query_stay_there():
    """Later tokens of the batch hold NaN and infinities: in a later block, and in the tail."""
    say("case: NaN behind")
    for where in (70, 100):   # in a full block; in the tail
        c = Case([110], 4, 2, 64, torch.float16, 10, paged=False)
        c.k[0][where:, :, 3], c.v[0][where:, :, 5] = float("nan"), float("inf")
        c.write([110], [110])
        out = c.cache.attend(c.batch([110], [110]), c.rows("q", [110], [110]))
        first = where // 32 * 32 if where < 96 else where   # a block's poison is the whole block's
        c.check_attend([first], [first], out[:first])
        assert torch.isnan(out[where + 1:]).all()


def test_scores_far_apart():
    """One key takes all the weight, late or early; keys of very different blocks."""
    say("case: scores far apart")
    for at in (0, 40, 599):
        c = Case([600], 2, 1, 64, torch.float16, 11, paged=False)
        c.q[0] *= 0.5
        c.k[0][at] = c.q[0][599][:1] * 40
        c.v[0][32:64] *= 2.0 ** -9
        c.write([600], [600])
        out = c.cache.attend(c.batch([600], [1]), c.rows("q", [600], [1]))
        c.check_attend([600], [1], out)


def test_shared_blocks():
    """Two sequences with the first 64 tokens in the same blocks."""
    say("case: shared prefix blocks")
    c = Case([64, 90, 75], 4, 2, 64, torch.bfloat16, 12, paged=False)
    for x in (c.k, c.v):
        x[1][:64], x[2][:64] = x[0], x[0]
    c.write([64, 0, 0], [64, 0, 0])
    # sequences 1 and 2: the two shared blocks, then one of their own
    b = lambda new: c.cache.batch(i32([90, 75]), i32([0, 3, 6]), 90, cu=i32(starts(new)), blk_ids=i32([0, 1, 2, 0, 1, 5]),   # noqa: E731
                                  tail_ids=i32([2, 0]))
    c.cache.write(b([26, 11]), *(torch.cat((x[1][64:], x[2][64:75])).cuda() for x in (c.k, c.v)))
    out = c.cache.attend(b([1, 2]), torch.cat((c.q[1][89:], c.q[2][73:75])).cuda())
    c.check_attend([0, 90, 75], [0, 1, 2], out)


def test_cache_beyond_32_bit_offsets():
    """Blocks above 2 GiB of bytes (and 2^31 elements) from the start."""
    say("case: 70,000 blocks of 8 heads of 128")
    cache = DeviceKvCache(70000, 1, 8, 128)
    c = Case([100], 8, 8, 128, torch.float16, 13, paged=False)
    b = lambda new: cache.batch(i32([100]), i32([0, 4]), 100, cu=i32([0, new]), blk_ids=i32([69999, 3, 69998, 69000]))   # noqa: E731
    cache.write(b(100), c.k[0].cuda(), c.v[0].cuda())
    k, v = cache.read(b(100))
    for got, want in zip((k, v), c.held(0)):
        assert torch.equal(got.cpu(), torch.from_numpy(want).float().half())
    c.check_attend([100], [1], cache.attend(b(1), c.q[0][99:].cuda()))


def test_numbers_out_of_bounds_are_flagged_and_left_out():
    """Every one is kept from the memory by the kernels' own checks."""
    say("case: bad batches")
    c = Case([70, 40], 2, 2, 64, torch.float16, 14, paged=False)
    c.write(c.lens, c.lens)
    want = c.cache.attend(c.batch(c.lens, [1, 1]), c.rows("q", c.lens, [1, 1]))
    q = c.rows("q", c.lens, [1, 1])
    bad = [dict(length=[200, 40]), dict(length=[-1, 40]), dict(length=[0, 40], cu=[0, 1, 2]), dict(blk_ids=[0, 99, 2, 3, 4]),
           dict(blk_ids=[0, -5, 2, 3, 4]), dict(tail_ids=[7, 1]), dict(tail_ids=[-1, 1]), dict(blk_start=[0, 1, 5]),
           dict(blk_start=[-3, 3, 5], start0=True)]
    for d in bad:
        say("  ", d)
        kv = (c.cache.k.clone(), c.cache.v.clone(), c.cache.tail.clone())
        b = c.cache.batch(i32(d.get("length", [70, 40])), i32(d.get("blk_start", [0, 3, 5])), 128,
                          cu=i32(d.get("cu", [0, 1, 2])), blk_ids=i32(d["blk_ids"]) if "blk_ids" in d else None,
                          tail_ids=i32(d["tail_ids"]) if "tail_ids" in d else None)
        if "blk_start" in d and not d.get("start0"):
            want_1 = None    # sequence 1's blocks moved too
        else:
            want_1 = want[1]
        out = c.cache.attend(b, q)
        c.cache.read(b)
        assert int(c.cache.status.item()) == B.AIQ_DEV_KV_RANGE
        if want_1 is not None:
            assert torch.equal(out[1], want_1)   # the other sequence is not harmed
        c.cache.write(b, c.rows("k", c.lens, [1, 1]), c.rows("v", c.lens, [1, 1]))   # (its last row again)
        for x, y in zip(kv, (c.cache.k, c.cache.v, c.cache.tail)):
            assert torch.equal(x, y)
        c.cache.status.zero_()


def test_captured_steps_replay_as_eager_ones():
    """A step (write, attend) captured once and replayed as the sequences grow,
    with eager work between, on a stream of its own."""
    say("case: captured steps")
    lens = np.array([62, 600, 95, 31])
    c, e = (Case(lens + 40, 6, 2, 128, torch.bfloat16, 15) for _ in range(2))
    for x in (c, e):
        x.write(lens, lens)
    one = np.ones(4, np.int64)
    length = i32(lens)
    b = c.cache.batch(length, c.blk_start, 700, blk_ids=c.blk_ids, tail_ids=c.tail_ids)
    k, v, q = (torch.zeros(4, h, 128, dtype=torch.bfloat16, device="cuda") for h in (2, 2, 6))
    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.cache.attend(b, q, out=out)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        length.add_(1)
        c.cache.write(b, k, v)
        c.cache.attend(b, q, out=out)
    for step in range(1, 40):
        at = lens + step
        for t, what in ((k, "k"), (v, "v"), (q, "q")):
            t.copy_(c.rows(what, at, one))
        g.replay()
        e.write(at, one, single=True)
        want = e.cache.attend(e.batch(at, one, single=True), e.rows("q", at, one))
        torch.cuda.synchronize()
        assert torch.equal(out, want), step
    c.check_read(lens + 39)


def test_a_stream_of_its_own():
    say("case: side stream")
    c = Case([50, 700], 4, 2, 64, torch.float16, 16)
    one = np.ones(2, np.int64)
    k, v, q = (c.rows(w, c.lens, c.lens) for w in "kvq")
    ball, bone = c.batch(c.lens, c.lens), c.batch(c.lens, one, single=True)
    q1 = c.rows("q", c.lens, one)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    c.cache.write(ball, k, v, stream=s)
    out = c.cache.attend(bone, q1, stream=s)
    s.synchronize()
    c.check_attend(c.lens, one, out)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv,hd", [(24, 8, 128), (8, 8, 64), (20, 4, 64), (8, 1, 128)])
def test_attention_of_many_tokens(heads, kv, hd, dtype):
    """Long prompts on kept ones: ragged, whole, one token among them, none."""
    say("case: many tokens", heads, kv, hd, dtype)
    lens = np.array([130, 33, 1, 0, 257, 64, 700, 90, 128, 31] * 4)
    new = np.minimum(lens, np.array([130, 1, 1, 0, 129, 33, 200, 90, 127, 30] * 4))
    c = Case(lens, heads, kv, hd, dtype, 21)
    c.write(lens, lens)
    out = c.cache.attend(c.batch(lens, new), c.rows("q", lens, new))
    keep = np.zeros_like(new)
    keep[:10] = new[:10]
    c.check_attend(lens, keep, out[:keep.sum()])
    one = c.cache.attend(c.batch(lens, np.minimum(new, 1)), c.rows("q", lens, np.minimum(new, 1)))   # the last rows by the other kernel
    at = np.cumsum(new) - 1
    last = out[torch.as_tensor(at[new > 0]).cuda()]
    scale = max(float(x.abs().max()) for x in c.v if x.numel())
    assert float((last.float() - one.float()).abs().max()) <= (2 * U[dtype] + 2.0 ** -13) * scale + 2 * U[dtype] * float(one.float().abs().max())


def test_infinity_and_nan_behind_many_queries_stay_there():
    say("case: NaN behind many queries")
    for where in (70, 100):
        c = Case([110] * 40, 4, 2, 64, torch.bfloat16, 22, paged=False)
        for i in range(0, 40, 2):
            c.k[i][where:, :, 3], c.v[i][where:, :, 5] = float("nan"), float("inf")
        lens = np.full(40, 110)
        c.write(lens, lens)
        out = c.cache.attend(c.batch(lens, lens), c.rows("q", lens, lens))
        first = where // 32 * 32 if where < 96 else where
        sel = np.zeros(40, np.int64)
        sel[:4] = first
        c.check_attend(sel, sel, torch.cat([out[i * 110:i * 110 + first] for i in range(4)]))
        assert torch.isnan(out[where + 1:110]).all() and not torch.isnan(out[110:220]).any()


def test_zero_queries_and_keys():
    """Scores of nothing but zeros: the mean of the values."""
    say("case: zero queries and keys")
    for dtype in (torch.float16, torch.bfloat16):
        for n_seq, new in ((1, 1), (1, 40), (40, 90)):
            c = Case([90] * n_seq, 4, 2, 64, dtype, 23)
            for i in range(n_seq):
                c.k[i][:] = 0
                c.q[i][:] = 0
            lens, news = np.full(n_seq, 90), np.full(n_seq, new)
            c.write(lens, lens)
            out = c.cache.attend(c.batch(lens, news), c.rows("q", lens, news))
            sel = np.zeros(n_seq, np.int64)
            sel[0] = new
            c.check_attend(lens, sel, out[:new])


@pytest.mark.parametrize("lead", [1, 40, 300])
@pytest.mark.parametrize("lens,new", [([70, 200, 33], [3, 40, 1]), ([300] * 40, [90] * 40)])
def test_rows_before_the_first_sequence_are_left_alone(lens, new, lead):
    # the call's rows start at cu[0] > 0: what lies before belongs to nobody, in the cache and in the outputs
    say("lead", lead, len(lens))
    c = Case(lens, 8, 8, 64, torch.float16, 31)
    old = [L - m for L, m in zip(lens, new)]
    c.write(old, old)
    at = starts(new) + lead
    n = int(at[-1])

    def behind(x):
        y = torch.full((n,) + x.shape[1:], 3.0, dtype=x.dtype, device="cuda")
        y[lead:] = x
        return y

    b = c.cache.batch(i32(lens), c.blk_start, max(lens), cu=i32(at), blk_ids=c.blk_ids, tail_ids=c.tail_ids)
    c.cache.write(b, behind(c.rows("k", lens, new)), behind(c.rows("v", lens, new)))
    c.check_read(lens)
    out = torch.full((n, 8, 64), 5.0, dtype=torch.float16, device="cuda")
    c.cache.attend(b, behind(c.rows("q", lens, new)), out=out)
    assert bool((out[:lead] == 5.0).all())
    c.check_attend(lens, new, out[lead:])
    k = torch.full((n, 8, 64), 5.0, dtype=torch.float16, device="cuda")
    v = k.clone()
    B.aiq_kv_read(c.cache.struct, b.struct, k.data_ptr(), 512, v.data_ptr(), 512, torch.cuda.current_stream().cuda_stream)
    for got, what in ((k, 0), (v, 1)):
        assert bool((got[:lead] == 5.0).all())
        for i, (L, m) in enumerate(zip(lens, new)):
            want = torch.from_numpy(c.held(i, L)[what][L - m:]).to(torch.float32).half()
            assert torch.equal(got[at[i]:at[i + 1]].cpu(), want)
    c.ok()


def test_two_streams_and_two_graphs_at_once():
    # long sequences of one cache, split between workgroups: each call has a workspace of its own
    say("two streams")
    a, b = Case([9000, 5000, 700], 8, 8, 64, torch.float16, 41), Case([4000, 20000], 24, 8, 128, torch.bfloat16, 42)
    calls = []
    for c in (a, b):
        lens, ones = list(c.lens), [1] * len(c.lens)
        c.write(lens, lens)
        calls.append((c.cache, c.batch(lens, ones, single=True), c.rows("q", lens, ones)))
    want = [cache.attend(batch, q) for cache, batch, q in calls]
    for c, w in zip((a, b), want):
        c.check_attend(list(c.lens), [1] * len(c.lens), w)
    assert all(batch.ws_bytes[q.shape[1]] > 0 for _, batch, q in calls)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        got = [cache.attend(batch, q, stream=s) for (cache, batch, q), s in zip(calls, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    say("two graphs")
    graphs, outs = [], []
    for (cache, batch, q), s in zip(calls, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(cache.attend(batch, q))
        graphs.append(g)
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = calls[0][0].attend(*calls[0][1:])
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want)) and torch.equal(eager, want[0])


@pytest.mark.parametrize("n", [70, 300])
def test_many_rows_of_sequences_of_many_lengths(n):
    # lengths far apart, sequences without rows between; then one whose numbers do not fit
    say("many lengths", n)
    r = np.random.default_rng(51)
    lens = np.minimum(np.exp(r.normal(5.0, 0.9, n)).astype(np.int64) + 1, 3000)
    new = np.where(r.random(n) < 0.2, 0, np.minimum(lens, r.integers(60, 200, n)))
    c = Case(lens, 8, 4, 64, torch.float16, 52)
    c.write(lens, lens)
    q = c.rows("q", lens, new)
    out = c.cache.attend(c.batch(lens, new), q)
    c.check_attend(lens, new, out)
    bad = int(np.flatnonzero(new)[3])
    over = lens.copy()
    over[bad] = 4000
    at = starts(new)
    b = c.cache.batch(i32(over), c.blk_start, 3000, cu=i32(at), blk_ids=c.blk_ids, tail_ids=c.tail_ids)
    again = c.cache.attend(b, q)
    assert int(c.cache.status.item()) == B.AIQ_DEV_KV_RANGE
    keep = np.ones(int(at[-1]), bool)
    keep[at[bad]:at[bad + 1]] = False
    keep = torch.from_numpy(keep).cuda()
    assert torch.equal(again[keep], out[keep])


def test_single_rows_read_back_and_sequences_without_blocks():
    say("single rows")
    lens = [1, 31, 32, 33, 0, 64, 300]
    c = Case(lens, 4, 2, 64, torch.bfloat16, 61)
    c.write(lens, lens)
    k, v = c.cache.read(c.batch(lens, [1] * len(lens), single=True))
    for got, what in ((k, 0), (v, 1)):
        for i, L in enumerate(lens):
            if L:
                want = torch.from_numpy(c.held(i, L)[what][-1]).to(torch.float32).bfloat16()
                assert torch.equal(got[i].cpu(), want), L
    say("tails alone")
    lens = np.array([1, 17, 31, 0])
    c = Case(lens, 4, 2, 64, torch.float16, 62, paged=False)
    c.cache = DeviceKvCache(0, 4, 2, 64, torch.float16)
    c.write(lens, lens)
    c.check_read(lens)
    one = (lens > 0).astype(np.int64)
    q = torch.zeros(4, 4, 64, dtype=torch.float16, device="cuda")
    q[torch.from_numpy(lens > 0).cuda()] = c.rows("q", lens, one)
    out = c.cache.attend(c.batch(lens, one, single=True), q)
    c.check_attend(lens, np.ones(4, np.int64) * one, out[:3])
    assert not bool(out[3].any())


@pytest.mark.parametrize("n,hd", [(1, 64), (300, 128), (2100, 64)])
def test_single_rows_complete_blocks_in_any_group(n, hd):
    # steps of one row per sequence across a block's end, sequences at different places: what the calls with all rows hold
    say("steps", n, hd)
    r = np.random.default_rng(63)
    lens = r.integers(28, 70, n)
    c, d = (Case(lens + 6, 3, 3, hd, torch.float16, 64) for _ in range(2))
    c.write(lens, lens)
    for s in range(1, 7):
        c.write(lens + s, np.ones(n, np.int64), single=True)
    d.write(lens + 6, lens + 6)
    for name in ("k", "v", "k_scale", "v_scale"):
        x, y = getattr(c.cache, name), getattr(d.cache, name)
        full = torch.zeros(x.shape[0], dtype=torch.bool, device="cuda")   # (the last block, where it is not full, is not written)
        at = (c.blk_ids.long().cpu().numpy())
        for i in range(n):
            full[torch.from_numpy(at[c.start[i]:c.start[i] + (lens[i] + 6) // BLOCK]).cuda()] = True
        assert torch.equal(x[full], y[full]), name
    for p, q in zip(c.cache.read(c.batch(lens + 6, lens + 6)), d.cache.read(d.batch(lens + 6, lens + 6))):
        assert torch.equal(p, q)
    c.ok()


# (sequences, new rows of each or None for one by `cu` NULL, heads, K/V heads, head_dim): a workgroup per item, segments in
# workgroups of their own, waves alone, tiles of 16 rows, tiles of 128
FORMS = [([40, 100, 96], None, 6, 2, 64), ([3000], None, 8, 2, 128), ([50] * 1100, None, 4, 2, 64),
         ([40, 100, 96], 9, 6, 2, 64), ([90] * 60, 33, 8, 2, 128)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens,new,heads,kv,hd", FORMS, ids=lambda x: str(x)[:12])
def test_a_query_whose_scores_are_all_minus_infinity(lens, new, heads, kv, hd, dtype):
    """Its softmax is not a number, as by the formula; the other queries are as without it."""
    say("case: infinite query", len(lens), new, heads, kv, hd, dtype)
    c = Case(lens, heads, kv, hd, dtype, 71)
    for k in c.k:
        k[:, :, 0] = -1.0
    lens, ones = np.array(lens), np.full(len(lens), new or 1)
    c.write(lens, lens)
    b, q = c.batch(lens, ones, single=new is None), c.rows("q", lens, ones)
    want = c.cache.attend(b, q)
    poisoned = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    poisoned[::2, 1] = True
    poisoned[-1, -1] = True
    q = q.clone()
    q[..., 0] = torch.where(poisoned, torch.inf, q[..., 0])
    out = c.cache.attend(b, q)
    assert torch.isnan(out[poisoned]).all()
    top = max(float(v.abs().max()) for v in c.v)   # (a tile's rows share when their references move: two results within their bounds)
    tol = 2 * ((U[dtype] + 2.0 ** -14) * top + U[dtype] * want.double().abs() + 1e-7)
    assert bool(((out.double() - want.double()).abs() <= tol)[~poisoned].all())
    c.ok()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens,new,heads,kv,hd", FORMS, ids=lambda x: str(x)[:12])
def test_blocks_that_were_never_written_hold_zeros(lens, new, heads, kv, hd, dtype):
    say("case: nothing written", len(lens), new, heads, kv, hd, dtype)
    c = Case(lens, heads, kv, hd, dtype, 75)
    ones = np.full(len(lens), new or 1)
    for x in c.cache.read(c.batch(lens, lens)):
        assert bool((x == 0).all())
    assert bool((c.cache.attend(c.batch(lens, ones, single=new is None), c.rows("q", lens, ones)) == 0).all())
    c.ok()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,new", [(3, None), (3, 5), (60, 40)])
def test_an_infinite_value_of_a_seen_token_without_weight(n, new, dtype):
    """A token of the tail whose weight is 0 in 32 bits: 0 times its infinite value is not a number, in every form."""
    say("case: infinite value without weight", n, new, dtype)
    lens, ones, at = np.full(n, 90), np.full(n, new or 1), 86
    c = Case(lens, 8, 2, 64, dtype, 74)
    for q, k, v in zip(c.q, c.k, c.v):
        q[:], k[:] = 20.0, 0.0
        k[at] = -20.0        # a score of -3,200
        v[at, 1, 7] = float("inf")
    c.write(lens, lens)
    out = c.cache.attend(c.batch(lens, ones, single=new is None), c.rows("q", lens, ones)).view(n, -1, 8, 64)
    seen = 90 - at if new else 1
    assert torch.isnan(out[:, -seen:, 4:, 7]).all()
    assert torch.isfinite(out[:, -seen:, :4]).all() and torch.isfinite(out[:, :-seen]).all()


@pytest.mark.parametrize("heads,kv,hd", [(4, 4, 64), (12, 4, 64), (12, 4, 128), (20, 4, 64), (72, 4, 64)])
def test_waves_alone_over_several_segments(heads, kv, hd):
    """Groups of 1, 3, 5 and 18 (two tiles) heads, sequences of up to three segments of 512 tokens: within the bound, and the bits of the
    sequence by itself (a workgroup's four waves)."""
    say("case: waves alone, several segments", heads, kv, hd)
    n = 2400
    lens = np.full(n, 2)
    lens[[3, 700, 2399]] = 1400, 513, 1030
    c = Case(lens, heads, kv, hd, torch.float16, 76, paged=False)
    c.write(lens, lens)
    ones = np.ones(n, np.int64)
    q = c.rows("q", lens, ones)
    out = c.cache.attend(c.batch(lens, ones, single=True), q)
    for i in (3, 700, 2399):
        alone = c.cache.batch(i32(lens[i:i + 1]), i32(c.start[i:i + 2]), 1024 if lens[i] < 1024 else 1400, tail_ids=i32([i]))
        assert torch.equal(c.cache.attend(alone, q[i:i + 1])[0], out[i])
        want, top = R.attend(c.q[i][-1:].float().numpy(), *c.held(i), [lens[i] - 1])
        tol = (2.0 ** -11 + 2.0 ** -14) * top[:, :, None] + 2.0 ** -11 * np.abs(want) + 1e-7
        assert np.all(np.abs(out[i:i + 1].double().cpu().numpy() - want) <= tol)
    c.ok()


@pytest.mark.parametrize("n", [150, 400])
def test_one_row_per_sequence_and_many_heads_does_not_depend_on_the_others(n):
    """64 query heads on one K/V head, the rows given by cu: the bits of a sequence by itself."""
    say("case: 64 heads on one", n)
    lens = np.random.default_rng(72).integers(1, 500, n)
    lens[5] = 480
    c = Case(lens, 64, 1, 64, torch.float16, 73)
    c.write(lens, lens)
    ones = np.ones(n, np.int64)
    q = c.rows("q", lens, ones)
    many = c.cache.attend(c.batch(lens, ones), q)
    assert torch.equal(many, c.cache.attend(c.batch(lens, ones, single=True), q))
    for i in (0, 5, n - 1):
        s, e = c.start[i], c.start[i + 1]
        alone = c.cache.batch(i32([lens[i]]), i32([0, e - s]), 500, cu=i32([0, 1]), blk_ids=c.blk_ids[s:e].contiguous(),
                              tail_ids=c.tail_ids[i:i + 1].contiguous())
        assert torch.equal(c.cache.attend(alone, q[i:i + 1])[0], many[i])
    c.ok()


def test_blocks_past_the_end_of_the_list_are_flagged_and_left_out():
    say("case: short lists of blocks")
    lens, ones = np.array([70, 40]), np.ones(2, np.int64)
    c = Case(lens, 2, 2, 64, torch.float16, 77, paged=False)
    c.write(lens, lens)
    q = c.rows("q", lens, ones)
    want = c.cache.attend(c.batch(lens, ones), q)
    # sequence 1's full block is entry 3, sequence 0's are entries 0 and 1; the tails' entries are not read
    for ids, good in (([0, 1, 2, 3], [0, 1]), ([0, 1, 2], [0]), ([0, 1], [0]), ([0], []), ([], [])):
        for cu in (None, i32([0, 1, 2])):
            say("  ", ids, cu is None)
            kv = [t.clone() for t in (c.cache.k, c.cache.v, c.cache.k_scale, c.cache.v_scale, c.cache.tail)]
            b = c.cache.batch(i32(lens), i32([0, 3, 5]), 70, cu=cu, blk_ids=i32(ids))
            out = c.cache.attend(b, q)
            for i in good:
                assert torch.equal(out[i], want[i])
            assert int(c.cache.status.item()) == (0 if len(good) == 2 else B.AIQ_DEV_KV_RANGE)
            c.cache.read(b)
            c.cache.write(b, c.rows("k", lens, ones), c.rows("v", lens, ones))   # (its last row again)
            for x, y in zip(kv, (c.cache.k, c.cache.v, c.cache.k_scale, c.cache.v_scale, c.cache.tail)):
                assert torch.equal(x, y)
            assert int(c.cache.status.item()) == (0 if len(good) == 2 else B.AIQ_DEV_KV_RANGE)
            c.cache.status.zero_()


def test_a_batch_on_two_caches():
    """Caches of other heads and head sizes behind one batch: each call's workspace, and flags in the status of its cache."""
    say("case: a batch on two caches")
    lens = [6000, 37]
    c, d = Case(lens, 8, 1, 64, torch.float16, 78, paged=False), Case(lens, 8, 8, 128, torch.float16, 79, paged=False)
    b, one = c.batch(lens, lens), c.batch(lens, [1, 1], single=True)
    for x in (c, d, c):
        x.cache.write(b, x.rows("k", lens, lens), x.rows("v", lens, lens))
        x.check_attend(lens, [1, 1], x.cache.attend(one, x.rows("q", lens, [1, 1])))
    bad = c.cache.batch(i32([7000, 37]), c.blk_start, 7000)
    d.cache.attend(bad, d.rows("q", lens, [1, 1]))
    assert int(c.cache.status.item()) == 0 and int(d.cache.status.item()) == B.AIQ_DEV_KV_RANGE


@pytest.mark.parametrize("hd", [64, 128])
def test_rows_written_again(hd):
    """From a block's first token on, inside a block that is not full, or by the call that filled one: the same bytes and tails."""
    say("case: rows written again", hd)
    #  sequence:        0   1   2   3   4   5   6
    lens = np.array([  50, 50, 64, 32, 40, 33, 20])
    c = Case(lens, 2, 2, hd, torch.bfloat16, 80)
    first = np.array([ 10, 50, 45, 10,  0, 32,  5])   # tokens of a first call, the others come in a second
    c.write(first, first)
    c.write(lens, lens - first)
    names = ("k", "v", "k_scale", "v_scale", "tail")
    before = [getattr(c.cache, x).clone() for x in names]
    # the end of a tail; from a block's start over its end; the filling call; the filling call; a tail's one row; the same; all
    again = np.array([ 3, 50, 19, 22,  1,  1, 20])
    c.write(lens, again)
    # whole blocks in the middle, the later tokens left as they are
    c.write(np.array([32, 32, 32, 32, 32, 32, 0]), np.array([32, 32, 32, 32, 32, 32, 0]))
    for x, y in zip(names, before):
        assert torch.equal(getattr(c.cache, x), y), x
    c.write(lens, np.array([1, 1, 0, 0, 1, 1, 1]))
    one = lens % BLOCK != 0
    c.write(np.where(one, lens, 0), np.ones(7, np.int64) * one, single=False)
    for x, y in zip(names, before):
        assert torch.equal(getattr(c.cache, x), y), x
    c.check_read(lens)


@pytest.mark.parametrize("new", [None, 5, 40])
def test_values_of_blocks_scales_apart(new):
    """Blocks of zeros (the least scale), of tiny and of large values, 2^96 apart: every one weighs what its scores say."""
    say("case: scales of values apart", new)
    n = 3 if new != 40 else 60
    lens, ones = np.full(n, 150), np.full(n, new or 1)
    c = Case(lens, 8, 2, 64, torch.bfloat16, 81)
    for q, v in zip(c.q, c.v):
        q *= 0.25
        v[:32] = 0
        v[32:64] *= 2.0 ** -70
        v[64:96] *= 2.0 ** 16 / float(v[64:96].abs().max())
    c.write(lens, lens)
    out = c.cache.attend(c.batch(lens, ones, single=new is None), c.rows("q", lens, ones))
    sel = np.zeros(n, np.int64)
    sel[:3] = ones[:3]
    c.check_attend(lens, sel, out[:3 * (new or 1)])
