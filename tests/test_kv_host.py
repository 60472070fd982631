"""The refusals of the 8-bit cache's and the sampling's entry points, without
a device: a bad call returns its status before anything is enqueued (fake
addresses are never read)."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

from paper_2608_10139_amd import binding as B
from paper_2608_10139_amd.device import DeviceKvCache, sample
from tests.test_abi_host import model, query, table

FAKE = 0x10000


def cache(**kw):
    c = B.aiq_kv_cache()
    c.k = c.v = c.k_scale = c.v_scale = c.tail = FAKE
    c.n_blocks, c.n_tails, c.n_kv_heads, c.head_dim, c.dtype = 10, 2, 2, 64, B.AIQ_F16
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def batch(**kw):
    b = B.aiq_kv_batch()
    b.n_seq, b.max_len, b.n_rows = 2, 100, 5
    b.len = b.cu = b.blk_start = FAKE
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def write(c, b, k=FAKE, k_ld=128, v=FAKE, v_ld=128, read=False):
    f = B.load().aiq_kv_read if read else B.load().aiq_kv_write
    return f(C.byref(c) if c else None, C.byref(b) if b else None, k, k_ld, v, v_ld, None)


def attend(c, b, q=FAKE, q_ld=512, heads=8, out=FAKE, out_ld=512, dtype=B.AIQ_F16, ws=FAKE, ws_bytes=1 << 40):
    return B.load().aiq_kv_attend(C.byref(c), C.byref(b), q, q_ld, heads, out, out_ld, dtype, ws, ws_bytes, None)


BAD_CACHE = [(dict(dtype=B.AIQ_F32), B.AIQ_EUNSUPPORTED), (dict(dtype=B.AIQ_I8), B.AIQ_EUNSUPPORTED),
             (dict(head_dim=32), B.AIQ_EINVAL), (dict(head_dim=96), B.AIQ_EINVAL), (dict(n_kv_heads=0), B.AIQ_EINVAL),
             (dict(n_blocks=-1), B.AIQ_EINVAL), (dict(n_tails=-1), B.AIQ_EINVAL), (dict(k=0), B.AIQ_EINVAL),
             (dict(v=0), B.AIQ_EINVAL), (dict(k_scale=0), B.AIQ_EINVAL), (dict(v_scale=0), B.AIQ_EINVAL),
             (dict(tail=0), B.AIQ_EINVAL), (dict(k=FAKE + 8), B.AIQ_EINVAL), (dict(tail=FAKE + 2), B.AIQ_EINVAL),
             (dict(v_scale=FAKE + 2), B.AIQ_EINVAL)]
BAD_BATCH = [dict(n_seq=-1), dict(n_rows=-1), dict(n_rows=1 << 31), dict(max_len=-1), dict(len=0), dict(blk_start=0),
             dict(cu=0), dict(status=FAKE + 4)]


@pytest.mark.parametrize("kw,code", BAD_CACHE, ids=str)
def test_bad_caches(kw, code):
    n = C.c_size_t()
    assert write(cache(**kw), batch()) == write(cache(**kw), batch(), read=True) == attend(cache(**kw), batch()) == code
    assert B.load().aiq_kv_attend_workspace_size(C.byref(cache(**kw)), C.byref(batch()), 8, C.byref(n)) == code


@pytest.mark.parametrize("kw", BAD_BATCH, ids=str)
def test_bad_batches(kw):
    assert write(cache(), batch(**kw)) == write(cache(), batch(**kw), read=True) == attend(cache(), batch(**kw)) == B.AIQ_EINVAL


def test_counts_past_32_bits_are_refused():
    n = C.c_size_t()
    size = B.load().aiq_kv_attend_workspace_size
    for c, b, heads in ((cache(n_kv_heads=(1 << 16) + 1), batch(), (1 << 16) + 1), (cache(), batch(max_len=(1 << 30) + 1), 8),
                        (cache(), batch(n_seq=(1 << 26) + 1), 8)):
        ld = 1 << 30
        assert write(c, b, k_ld=ld, v_ld=ld) == write(c, b, k_ld=ld, v_ld=ld, read=True) == B.AIQ_EUNSUPPORTED
        assert attend(c, b, q_ld=ld, out_ld=ld, heads=heads) == B.AIQ_EUNSUPPORTED
        assert size(C.byref(c), C.byref(b), heads, C.byref(n)) == B.AIQ_EUNSUPPORTED
    assert attend(cache(), batch(), q_ld=1 << 30, out_ld=1 << 30, heads=(1 << 16) + 2) == B.AIQ_EUNSUPPORTED
    assert size(C.byref(cache()), C.byref(batch()), (1 << 16) + 2, C.byref(n)) == B.AIQ_EUNSUPPORTED
    assert size(C.byref(cache()), C.byref(batch(max_len=1 << 30)), 1 << 16, C.byref(n)) == B.AIQ_OK


@pytest.mark.parametrize("kw", [dict(k=0), dict(v=0), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(k_ld=127), dict(v_ld=120),
                                dict(k_ld=132), dict(v_ld=-128)], ids=str)
def test_bad_rows(kw):
    assert write(cache(), batch(), **kw) == write(cache(), batch(), read=True, **kw) == B.AIQ_EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(q=0), B.AIQ_EINVAL), (dict(out=0), B.AIQ_EINVAL), (dict(q=FAKE + 4), B.AIQ_EINVAL), (dict(q_ld=511), B.AIQ_EINVAL),
    (dict(out_ld=516), B.AIQ_EINVAL), (dict(heads=0), B.AIQ_EINVAL), (dict(heads=7), B.AIQ_EINVAL),
    (dict(dtype=B.AIQ_F32), B.AIQ_EUNSUPPORTED), (dict(dtype=0), B.AIQ_EUNSUPPORTED)], ids=str)
def test_bad_attention(kw, code):
    assert attend(cache(), batch(), **kw) == code


def test_attention_workspace():
    c, b, n = cache(n_blocks=1 << 20), batch(n_seq=1, n_rows=1, cu=0, max_len=100000), C.c_size_t()
    size = B.load().aiq_kv_attend_workspace_size
    assert size(C.byref(c), C.byref(b), 8, C.byref(n)) == B.AIQ_OK and n.value > 0
    assert attend(c, b, ws_bytes=n.value - 1) == B.AIQ_ENOSPC
    assert attend(c, b, ws=0, ws_bytes=n.value) == attend(c, b, ws=FAKE + 16, ws_bytes=n.value) == B.AIQ_EINVAL
    assert size(C.byref(c), C.byref(b), 7, C.byref(n)) == size(C.byref(c), C.byref(b), 8, None) == B.AIQ_EINVAL
    assert size(None, C.byref(b), 8, C.byref(n)) == size(C.byref(c), None, 8, C.byref(n)) == B.AIQ_EINVAL
    # short sequences need none
    b = batch(n_seq=1, n_rows=1, cu=0, max_len=100)
    assert size(C.byref(c), C.byref(b), 8, C.byref(n)) == B.AIQ_OK and n.value == 0


def test_empty_batches_enqueue_nothing():
    b = batch(n_seq=0, n_rows=0, len=0, cu=0, blk_start=0)
    for c in (cache(), cache(n_blocks=0, n_tails=0, k=0, v=0, k_scale=0, v_scale=0, tail=0)):
        assert write(c, b, k=0, v=0) == write(c, b, k=0, v=0, read=True) == B.AIQ_OK
        assert attend(c, b, q=0, out=0, ws=0, ws_bytes=0) == B.AIQ_OK


def draw(logits=FAKE, dtype=B.AIQ_F32, ld=100, vocab=100, rows=3, u=FAKE, token=FAKE, null=False, **kw):
    p = B.aiq_sampling()
    p.temperature, p.top_p = 1.0, 1.0
    for k, v in kw.items():
        setattr(p, k, v)
    return B.load().aiq_sample(logits, dtype, ld, vocab, rows, None if null else C.byref(p), u, token, None)


@pytest.mark.parametrize("kw,code", [
    (dict(null=True), B.AIQ_EINVAL), (dict(logits=0), B.AIQ_EINVAL), (dict(u=0), B.AIQ_EINVAL), (dict(token=0), B.AIQ_EINVAL),
    (dict(logits=FAKE + 2), B.AIQ_EINVAL), (dict(logits=FAKE + 1, dtype=B.AIQ_F16), B.AIQ_EINVAL), (dict(ld=99), B.AIQ_EINVAL),
    (dict(vocab=0), B.AIQ_EINVAL), (dict(vocab=(1 << 24) + 1, ld=1 << 25), B.AIQ_EINVAL), (dict(rows=-1), B.AIQ_EINVAL),
    (dict(dtype=B.AIQ_I8), B.AIQ_EUNSUPPORTED), (dict(temperature=-1.0), B.AIQ_EINVAL),
    (dict(temperature=float("nan")), B.AIQ_EINVAL), (dict(temperature=float("inf")), B.AIQ_EINVAL),
    (dict(top_p=0.0), B.AIQ_EINVAL), (dict(top_p=1.5), B.AIQ_EINVAL), (dict(top_p=float("nan")), B.AIQ_EINVAL),
    (dict(min_p=-0.1), B.AIQ_EINVAL), (dict(min_p=1.1), B.AIQ_EINVAL), (dict(top_k=-1), B.AIQ_EINVAL)], ids=str)
def test_bad_sampling(kw, code):
    assert draw(**kw) == code


def test_no_rows_to_sample():
    assert draw(rows=0, logits=0, u=0, token=0) == B.AIQ_OK


def test_wrapper_refusals():
    with pytest.raises(ValueError):
        DeviceKvCache(1, 1, 1, 64, torch.float32, "cpu")
    c = DeviceKvCache(4, 2, 2, 64, device="cpu")   # never launched: the checks come first
    i = lambda *x: torch.tensor(x, dtype=torch.int32)   # noqa: E731
    for kw in (dict(length=torch.tensor([1, 2])), dict(blk_start=i(0, 2)), dict(cu=i(0, 1)), dict(tail_ids=i(0)),
               dict(blk_ids=i(0, 1, 2, 3)[::2])):
        with pytest.raises(ValueError):
            c.batch(**{**dict(length=i(5, 6), blk_start=i(0, 2, 4), max_len=64), **kw})
    b = c.batch(i(5, 6), i(0, 2, 4), 64)
    good = torch.zeros(2, 2, 64, dtype=torch.float16)
    for bad in (good.bfloat16(), good[:1], good[:, :1], torch.zeros(2, 2, 128, dtype=torch.float16)[:, :, ::2],
                torch.zeros(2, 4, 64, dtype=torch.float16)[:, ::2]):
        with pytest.raises(ValueError):
            c.write(b, bad, good)
        with pytest.raises(ValueError):
            c.write(b, good, bad)
    for bad in (good.bfloat16(), good[:1], torch.zeros(2, 2, 32, dtype=torch.float16)):
        with pytest.raises(ValueError):
            c.attend(b, bad)
    with pytest.raises(ValueError):
        c.attend(b, good, out=good.float())
    with pytest.raises(ValueError):
        c.attend(b, good, out_dtype=torch.float32)
    x = torch.zeros(2, 10)
    for args in ((x, x[:, 0]), (x[0], x[0]), (x.double(), x[:, 0])):
        with pytest.raises(ValueError):
            sample(*args)


def test_wrapper_refuses_other_devices():
    c = DeviceKvCache(4, 2, 2, 64, device="cpu")
    i = lambda *x: torch.tensor(x, dtype=torch.int32)   # noqa: E731
    b, rows = c.batch(i(5, 6), i(0, 2, 4), 64), torch.zeros(2, 2, 64, dtype=torch.float16)
    other = SimpleNamespace(device=torch.device("cuda", 1))
    for call in (lambda s: c.write(b, rows, rows, stream=s), lambda s: c.read(b, stream=s), lambda s: c.attend(b, rows, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call(other)
    b.device = torch.device("cuda", 1)
    for call in (lambda: c.write(b, rows, rows), lambda: c.read(b), lambda: c.attend(b, rows)):
        with pytest.raises(ValueError, match="batch"):
            call()


def gen_query(**kw):
    q = query(gen_tokens=4, eos_id=-1)
    for k, v in kw.items():
        if k in ("temperature", "top_k", "top_p", "min_p"):
            setattr(q.sampling, k, v)
        else:
            setattr(q, k, v)
    return q


def plan(q, **opts):
    o = B.aiq_plan_opts()
    for k, v in opts.items():
        setattr(o, k, v)
    return B.aiq_plan_create_status(model(), table(), None, q, o)


GOOD = dict(sample=1, temperature=1.0, top_p=1.0, sample_u=FAKE)


@pytest.mark.parametrize("kw,code", [
    (dict(), B.AIQ_OK), (dict(temperature=0.0, sample_u=0), B.AIQ_OK), (dict(top_k=5, top_p=0.5, min_p=0.5), B.AIQ_OK),
    (dict(sample=2), B.AIQ_EINVAL), (dict(sample_u=0), B.AIQ_EINVAL), (dict(sample_u=FAKE + 2), B.AIQ_EINVAL),
    (dict(temperature=-1.0), B.AIQ_EINVAL), (dict(top_p=0.0), B.AIQ_EINVAL), (dict(min_p=2.0), B.AIQ_EINVAL),
    (dict(top_k=-1), B.AIQ_EINVAL), (dict(gen_tokens=0), B.AIQ_EINVAL)], ids=str)
def test_sampling_queries(kw, code):
    assert plan(gen_query(**{**GOOD, **kw})) == code


def test_cache_types_of_a_plan():
    assert plan(gen_query(), kv_dtype=B.AIQ_I8) == plan(gen_query(), kv_dtype=B.AIQ_F16) == plan(gen_query()) == B.AIQ_OK
    assert plan(gen_query(), kv_dtype=B.AIQ_BF16) == plan(gen_query(), kv_dtype=-1) == B.AIQ_EINVAL
    assert plan(query(), kv_dtype=B.AIQ_I8) == B.AIQ_EINVAL   # nothing is generated
    assert plan(query(), kv_dtype=B.AIQ_F16) == B.AIQ_OK


def test_8_bit_plans_out_of_range():
    def status(q=None, t=None, **m):
        o = B.aiq_plan_opts()
        o.kv_dtype = B.AIQ_I8
        return B.aiq_plan_create_status(model(**m), t or table(), None, q or gen_query(), o)

    assert status() == B.AIQ_OK
    assert status(d_model=256) != B.AIQ_OK   # heads of 32
    t = table()
    t.max_list_len = (1 << 31) - 2           # lengths and generated tokens pass 32 bits
    assert status(t=t) == B.AIQ_EUNSUPPORTED


def test_entries_of_the_block_list():
    n = C.c_size_t()
    for bad in (-1, -(1 << 40)):
        b = batch(blk_ids=FAKE, n_blk_ids=bad)
        assert write(cache(), b) == write(cache(), b, read=True) == attend(cache(), b) == B.AIQ_EINVAL
        assert B.load().aiq_kv_attend_workspace_size(C.byref(cache()), C.byref(b), 8, C.byref(n)) == B.AIQ_EINVAL
    c = DeviceKvCache(4, 2, 2, 64, device="cpu")
    i = lambda *x: torch.tensor(x, dtype=torch.int32)   # noqa: E731
    assert c.batch(i(5, 6), i(0, 2, 4), 64).struct.n_blk_ids == 0
    assert c.batch(i(5, 6), i(0, 2, 4), 64, blk_ids=i(3, 2, 1)).struct.n_blk_ids == 3
    b = c.batch(i(5, 6), i(0, 2, 4), 64, blk_ids=i())   # a list without entries is not the numbers themselves
    assert b.struct.blk_ids and b.struct.n_blk_ids == 1


def test_a_batch_on_caches_of_other_shapes(monkeypatch):
    """Workspace by the cache's shape, flags in its own status word, which the batch keeps."""
    from paper_2608_10139_amd import device as D

    class On:
        def __init__(self, device, stream):
            pass

        def __enter__(self):
            return 0

        def __exit__(self, *e):
            pass

    calls = []
    monkeypatch.setattr(D, "_on", On)
    for f in ("aiq_kv_write", "aiq_kv_read"):
        monkeypatch.setattr(B, f, lambda c, b, *a: calls.append((c, b.status, 0, 0)))
    monkeypatch.setattr(B, "aiq_kv_attend", lambda c, b, q, qs, heads, o, os, dt, ws, n, s: calls.append((c, b.status, n, heads)))
    i = lambda *x: torch.tensor(x, dtype=torch.int32)   # noqa: E731
    one, two, three = (DeviceKvCache(256, 1, kv, hd, device="cpu") for kv, hd in ((2, 64), (8, 128), (2, 64)))
    b = one.batch(i(8000), i(0, 256), 8192)
    needs = []
    for c in (one, two, three, one):
        kv = torch.zeros(1, c.n_kv_heads, c.head_dim, dtype=torch.float16)
        c.write(b, kv, kv)
        c.read(b)
        c.attend(b, torch.zeros(1, 8, c.head_dim, dtype=torch.float16))
        want = B.aiq_kv_attend_workspace_size(c.struct, b.struct, 8)
        assert calls[-1][2:] == (want, 8)
        assert [x[1] for x in calls[-3:]] == [c.status.data_ptr()] * 3
        needs.append(want)
    assert needs[0] == needs[2] == needs[3] < needs[1]
    assert any(t is one.status for t in b.keep)
