"""AI_TRANSFORM with keys and values in 8 bits, and by sampling, through the
query path.

8 bits: as in the 16-bit tests, every token is within the tolerance of its
step's largest logit, with the logits of a plain form in 64 bits (teacher
forcing) whose generation steps attend over the cache as it stands at that
step: 8-bit blocks that are full, the last one in full precision."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle.generate import generated_length, like_tokens
from oracle.query import relational
from oracle.transformer import Weights64, rmsnorm
from paper_2608_10139_amd import binding as B
from paper_2608_10139_amd.device import DeviceModel, DevicePrefill, DeviceQuery, sample
from synth.gen import make_model
from tests import _kv_ref as R
from tests._parity import TOL_BF16, random_gains
from tests.test_gpu_generate import MODELS, check_valid_tokens, model, query, run, tables

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def rope(x, pos, theta):
    """x [T, heads, hd], rotate-half pairs."""
    half = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[:, None] * theta ** (-np.arange(half) * 2.0 / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def step_logits(m, prompt, gen):
    """Logits that choose gen[0], gen[1], ..: the prompt's last position, then each generated token's."""
    spec, w = m["spec"], Weights64.w
    H, KV, hd = spec.n_heads, spec.n_kv_heads, spec.head_dim
    seq = np.concatenate([prompt, gen[:-1]]).astype(np.int64)
    P, T = len(prompt), len(seq)
    x = w(m["emb"])[seq]
    pos = np.arange(T)
    for L in m["layers"]:
        h = rmsnorm(x, w(L["attn_norm"]), spec.norm_eps)
        q = rope((h @ w(L["wq"]).T).reshape(T, H, hd), pos, spec.rope_theta)
        k = rope((h @ w(L["wk"]).T).reshape(T, KV, hd), pos, spec.rope_theta)
        v = (h @ w(L["wv"]).T).reshape(T, KV, hd)
        out = np.zeros((T, H, hd))
        out[:P] = R.attend(q[:P], k[:P], v[:P], pos[:P])[0]
        for t in range(P, T):   # the step that reads tokens 0 .. t
            kt, vt = (R.held(y[:t + 1].astype(np.float32)) for y in (k, v))
            out[t] = R.attend(q[t:t + 1], kt, vt, [t])[0][0]
        x = x + out.reshape(T, H * hd) @ w(L["wo"]).T
        h = rmsnorm(x, w(L["ffn_norm"]), spec.norm_eps)
        a = h @ w(L["w_gate"]).T
        x = x + ((a / (1 + np.exp(-a))) * (h @ w(L["w_up"]).T)) @ w(L["w_down"]).T
    return rmsnorm(x[P - 1:], w(m["final_norm"]), spec.norm_eps) @ w(m["lm_head"]).T


@pytest.mark.parametrize("mname,npre", [("hd64", 0), ("hd128", 33), ("hd64", 32)])
def test_tokens_are_greedy_over_8_bit_keys_and_values(mname, npre):
    say("case: 8-bit generation", mname, npre)
    m, dm = model(mname)
    t = tables(120, 61, max_len=80)
    q = query(12, npre=npre)
    r = run(t, m, dm, q, kv_dtype="i8")
    assert r["status"] == 0
    rows, _ = relational(t, q)
    np.testing.assert_array_equal(r["sel_ids"], rows)
    off, tok = t["probe"]["offsets"], t["probe"]["tokens"]
    exact = total = 0
    for i in range(0, len(rows), 6):
        prompt = np.concatenate([t["prefix"][:npre].astype(np.int64), tok[off[rows[i]]:off[rows[i] + 1]]])
        gen = r["gen"][i]
        lg = step_logits(m, prompt, gen)
        gap = lg.max(axis=1) - lg[np.arange(len(gen)), gen]
        assert gap.max() <= TOL_BF16, (i, int(gap.argmax()), gap.max())
        exact += int(np.sum(lg.argmax(axis=1) == gen))
        total += len(gen)
    say(f"  {exact}/{total} tokens equal the plain form's own argmax")
    assert exact >= 0.9 * total


def test_8_bit_tokens_do_not_depend_on_the_batch():
    """2,600 rows in one chunk and in several, their first 60 alone, a prefix shared and per row."""
    say("case: 8-bit tokens of 2,600 rows and of their first 60")
    m = random_gains(make_model(replace(MODELS["hd64"], n_heads=4, n_kv_heads=2)))
    dm = DeviceModel(m)
    t = tables(5200, 54)
    n = 0
    while np.sum(t["probe"]["c"][:n] < 500) < 60:
        n += 1
    few = {**t, "probe": {k: v[:n + 1] if k == "offsets" else v[:n] for k, v in t["probe"].items() if k != "tokens"}}
    few["probe"]["tokens"] = t["probe"]["tokens"][:few["probe"]["offsets"][-1]]
    q = query(12, npre=5)
    a = run(t, m, dm, q, kv_dtype="i8")
    assert a["status"] == 0 and a["n_selected"] > 2000
    for b in (run(few, m, dm, q, kv_dtype="i8"), run(t, m, dm, q, kv_dtype="i8", chunk_tokens=9000),
              run(t, m, dm, q, kv_dtype="i8"), run(few, m, dm, q, kv_dtype="i8", share_prefix=False)):
        assert b["status"] == 0
        np.testing.assert_array_equal(a["gen"][:len(b["gen"])], b["gen"])
    np.testing.assert_array_equal(a["gen"][:, 0], run(t, m, dm, q)["gen"][:, 0])   # prefill attends in 16 bits


def test_8_bit_generation_with_empty_rows_and_prefix():
    """Rows without tokens: behind a shared prefix, and with nothing at all."""
    say("case: 8-bit generation, empty rows")
    m, dm = model("hd64")
    t = tables(60, 71)
    lens = t["probe"]["len"].copy()
    lens[::3] = 0
    off = np.zeros(61, np.int64)
    off[1:] = np.cumsum(lens)
    t["probe"].update(len=lens, offsets=off, tokens=t["probe"]["tokens"][:off[-1]])
    for npre in (0, 9, 32):
        q = query(40, npre=npre)
        a, b = run(t, m, dm, q, kv_dtype="i8"), run(t, m, dm, q)
        assert a["status"] == 0 and b["status"] == 0
        np.testing.assert_array_equal(a["gen"][:, 0], b["gen"][:, 0])
        if npre:
            one = run(t, m, dm, q, kv_dtype="i8", share_prefix=False)
            np.testing.assert_array_equal(a["gen"], one["gen"])


def test_8_bit_plan_needs_less_workspace():
    m, dm = model("hd64")
    t = tables(400, 43)
    sizes = []
    for kv in ("f16", "i8"):
        d = DeviceQuery(t, m, query(64), dmodel=dm, kv_dtype=kv)
        sizes.append(d.ws_bytes)
        d.close()
    assert sizes[1] < sizes[0]


def u_for(t, G, seed=5):
    return np.random.default_rng(seed).random((len(t["probe"]["len"]), G), dtype=np.float32)


def sampled(q, T, k=0, p=1.0, mp=0.0):
    return replace(q, sampling=(T, k, p, mp))


@pytest.mark.parametrize("kv", ["f16", "i8"])
def test_sampling_from_one_token_is_greedy(kv):
    say("case: sampling, top_k 1 and temperature 0", kv)
    m, dm = model("hd64")
    t = tables(300, 41)
    q = query(12, npre=3)
    want = run(t, m, dm, q, kv_dtype=kv)
    for s in (sampled(q, 1.3, k=1), sampled(q, 0.7, p=1e-9), sampled(q, 0.0)):
        r = run(t, m, dm, s, kv_dtype=kv, sample_u=u_for(t, 12))
        assert r["status"] == 0
        np.testing.assert_array_equal(r["gen"], want["gen"])
    r = run(t, m, dm, sampled(q, 0.0), kv_dtype=kv)   # no random numbers needed
    np.testing.assert_array_equal(r["gen"], want["gen"])


def test_sampled_tokens_are_those_of_the_logits():
    """The first token of each row from the full-vocabulary logits and the
    row's own random number; every later one among the likely tokens."""
    say("case: sampled tokens")
    m, dm = model("hd64")
    t = tables(200, 59)
    u = u_for(t, 6)
    q = sampled(query(6), 0.9, 30, 0.95, 0.01)
    r = run(t, m, dm, q, sample_u=u)
    assert r["status"] == 0
    rows, _ = relational(t, q)
    off, tok = t["probe"]["offsets"], t["probe"]["tokens"]
    seqs = [tok[off[x]:off[x + 1]] for x in rows]
    cu = np.zeros(len(seqs) + 1, dtype=np.int32)
    cu[1:] = np.cumsum([len(s) for s in seqs])
    pf = DevicePrefill(m, max_tokens=int(cu[-1]), dmodel=dm)
    lg = pf.run(torch.from_numpy(np.concatenate(seqs).astype(np.int32)).cuda(), torch.from_numpy(cu).cuda(), full_vocab=True)
    want = sample(lg, torch.from_numpy(u[rows, 0]).cuda(), 0.9, 30, 0.95, 0.01)
    torch.cuda.synchronize()
    pf.close()
    np.testing.assert_array_equal(r["gen"][:, 0], want.cpu().numpy())
    # all tokens: within the filters' reach of the maximum: w >= min_p, so x >= max + T ln(min_p)
    check_valid_tokens(m, t, q, r, np.arange(0, len(rows), 7), tol=0.9 * np.log(100.0) + TOL_BF16)
    assert np.mean(r["gen"] != run(t, m, dm, query(6))["gen"]) > 0.2


def test_sampled_8_bit_generation_with_end_token_and_like():
    """All together: several chunks, an end token, LIKE; a row's tokens depend on its own numbers only."""
    say("case: sampling over an 8-bit cache, end token, LIKE")
    m, dm = model("hd128")
    t = tables(400, 43)
    u = u_for(t, 20)
    base = sampled(query(20, npre=4), 1.0, 5)
    free = run(t, m, dm, base, kv_dtype="i8", sample_u=u)
    vals, cnts = np.unique(free["gen"][:, 1:], return_counts=True)
    eos = int(vals[np.argmax(cnts)])
    i0 = next(i for i in range(len(free["gen"])) if generated_length(free["gen"][i], eos) >= 4)
    pat = tuple(int(x) for x in free["gen"][i0, 2:4])
    q = replace(base, eos_id=eos, pad_id=1023, like=pat)
    r = run(t, m, dm, q, kv_dtype="i8", sample_u=u, chunk_tokens=3000)
    assert r["status"] == 0
    rows, _ = relational(t, q)
    for i in range(len(rows)):
        n = generated_length(free["gen"][i], eos)
        np.testing.assert_array_equal(r["gen"][i, :n], free["gen"][i, :n])
        assert np.all(r["gen"][i, n:] == 1023)
    flags = np.array([like_tokens(r["gen"][i], pat, eos) for i in range(len(rows))])
    assert flags.any()
    np.testing.assert_array_equal(r["kept_ids"], rows[flags])
    other = u.copy()
    other[rows[1::2]] = u_for(t, 20, 6)[rows[1::2]]
    o = run(t, m, dm, base, kv_dtype="i8", sample_u=other)
    np.testing.assert_array_equal(o["gen"][::2], free["gen"][::2])
    assert np.any(o["gen"][1::2] != free["gen"][1::2])


def test_one_generated_token_needs_no_step():
    say("case: one token")
    m, dm = model("hd64")
    t = tables(50, 72)
    a, b = (run(t, m, dm, query(1, npre=5), kv_dtype=kv) for kv in ("i8", "f16"))
    assert a["status"] == 0 and a["n_selected"] > 0
    np.testing.assert_array_equal(a["gen"], b["gen"])
