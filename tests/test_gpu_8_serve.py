"""Generation from a paged cache (serve.py: router, Top-K, paged append and
attention, read back, sampling together) against the oracle's sparse_prefill /
decode_step, sequence by sequence.

The GPU's kept sets and decisions are given to the oracle, and each decision must equal the
oracle's own wherever its score is more than 1e-3 away from the threshold. An 8-bit cache
adds an error of 1/254 of a vector's largest value to keys and values, twice the
type's own rounding of bf16 (2^-8), so its bounds are twice those."""
import numpy as np
import pytest
import torch

from oracle import adadsf_oracle as O
from paper_2607_21291_gb300 import synth as S
from tests import helpers as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2607_21291_gb300 import adadsf
    adadsf.lib()
    return adadsf


QWEN_SMALL = S.QWEN25_1_5B.replace(d=1024, n_heads=8, n_kv_heads=2, ffn=1536, n_layers=3, vocab=512)
NEOX_SMALL = S.PYTHIA_160M.replace(n_layers=3, vocab=512)
NEOX_F32 = S.PYTHIA_70M.replace(n_layers=3, vocab=512)
LENS = [70, 1, 33, 16]
RATIOS = [1.0, 0.45, 0.0]


def make(A, shape, store, page, n_pages=64, max_len=100):
    from paper_2607_21291_gb300 import serve
    td = H.tdtype(shape)
    host = [H.host_layer(shape, 31, l) for l in range(shape.n_layers)]
    extra = H.host_extra(shape, 31)
    ex = A.to_device(extra, td)
    srv = serve.Server(A.make_cfg(shape), [A.to_device(w, td) for w in host], ex, ex["embed"], len(LENS), max_len, n_pages,
                       page, A.KV_I8 if store == "i8" else A.KV_SAME)
    return srv, [H.f64(w) for w in host], H.f64(extra)


def prompts_of(shape, seed=32):
    ids = S.token_ids(seed, len(LENS), max(LENS) + 40, shape.vocab)
    return ids, [torch.from_numpy(ids[b, :n].astype(np.int64)) for b, n in enumerate(LENS)]


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("shape", [QWEN_SMALL, NEOX_SMALL, NEOX_F32], ids=["qwen", "neox", "neox-f32"])
def test_prefill_and_steps(A, shape, store):
    """Ragged prompts and 18 single tokens over pages of 16, against the
    definition; pages are taken as the layers' sequences grow and no more."""
    srv, W, E = make(A, shape, store, 16)
    ids, prompts = prompts_of(shape)
    p = O.params_of(shape)
    tol = (H.tol(shape) if store == "same" else 2 * H.BF16_TOL)
    etol = None if store == "same" else 2 * H.BF16_ELEM_TOL
    kept = []
    got = H.to_np(srv.prefill(prompts, RATIOS, kept))
    states = []
    for b, n in enumerate(LENS):
        force = [k[b].cpu().numpy()[None] for k in kept]
        assert [f.shape[1] for f in force] == [int(np.floor(r * n)) for r in RATIOS]
        ref, st = O.sparse_prefill(ids[b:b + 1, :n], E, W, p, [f.shape[1] for f in force], idx_force=force)
        H.assert_close(got[b], ref[0, -1], tol, f"prompt {b}", etol)
        states.append(st)
    checked = 0
    for step in range(18):
        tok = np.array([ids[b, n + step] for b, n in enumerate(LENS)])
        flags = torch.empty(shape.n_layers, len(LENS), dtype=torch.bool, device="cuda")
        got = H.to_np(srv.step(torch.from_numpy(tok.astype(np.int32)).cuda(), flags))
        flags = flags.cpu().numpy()
        for b in range(len(LENS)):
            thr = np.array(states[b]["thr"])
            ref, own, score = O.decode_step(tok[b:b + 1], E, W, p, states[b], kept_force=flags[:, b:b + 1])
            with np.errstate(invalid="ignore"):
                clear = np.abs(score - thr) > 1e-3 * np.maximum(1.0, np.abs(thr))
            if store == "same":
                assert (flags[:, b:b + 1][clear] == own[clear]).all()
            checked += int(clear.sum())
            H.assert_close(got[b], ref[0], tol, f"step {step} of {b}", etol)
    srv.check()
    assert checked > 0
    lens = srv.lens.cpu().numpy()
    assert lens.tolist() == [[len(st["rows"][l][0]) for st in states] for l in range(shape.n_layers)]
    assert (lens[2] == 0).all() and (srv.pool.held[2] <= 1).all()   # a layer that keeps nothing: a page at most
    assert (srv.pool.held <= lens // 16 + 2).all()
    # the first layer's cached rows are the definition's keys and values (its inputs are embeddings)
    hd, q, kv = shape.head_dim, shape.q_dim, shape.kv_dim
    for b, (k, v) in enumerate(srv.cached(0)):
        rows, pos = np.array(states[b]["rows"][0][0]), np.array(states[b]["pos"][0][0])
        a = (O.layer_norm(rows, W[0]["ln1_w"], W[0]["ln1_b"], p["norm_eps"]) if shape.arch == S.NEOX
             else O.rms_norm(rows, W[0]["ln1_w"], p["norm_eps"]))
        qkv = a @ W[0]["w_qkv"].T + W[0]["b_qkv"]
        keys = np.concatenate([O.rope(qkv[:, q + h * hd:q + (h + 1) * hd], pos, shape.rotary_dim, shape.rope_theta)
                               for h in range(shape.n_kv_heads)], axis=1)
        H.assert_close(H.to_np(k), keys, tol, f"keys of {b}", etol)
        H.assert_close(H.to_np(v), qkv[:, q + kv:], tol, f"values of {b}", etol)


def test_generate(A):
    """Greedy tokens are those of a step-by-step run with an argmax; with a nucleus, the same
    random numbers give the same tokens from another pool and after pages went
    back to it, and log-probabilities are finite."""
    shape = NEOX_SMALL
    ids, prompts = prompts_of(shape)
    srv, _, _ = make(A, shape, "same", 16)
    free = len(srv.pool.free)
    n = 12
    u = torch.rand(n, len(LENS), generator=torch.Generator().manual_seed(5)).cuda()
    cold = torch.zeros(len(LENS), device="cuda")
    tokens, logprob = srv.generate(prompts, RATIOS, n, u, temperature=cold)
    assert (logprob == 0).all()
    other, _, _ = make(A, shape, "same", 64)
    hidden = other.prefill(prompts, RATIOS)
    for i in range(n):
        logits = hidden.float() @ other.head.float().T
        best = logits.topk(2, -1)
        sure = (best.values[:, 0] - best.values[:, 1]) > 2.0 ** -6 * best.values[:, 0].abs()   # logits are bf16
        assert (tokens[i] == best.indices[:, 0])[sure].all()
        if i + 1 < n:
            hidden = other.step(tokens[i])
    other.check()
    for b in range(len(LENS)):
        srv.release(b)
    assert len(srv.pool.free) == free and (srv.lens == 0).all()
    top_p = torch.full((len(LENS),), 0.9, device="cuda")
    first = srv.generate(prompts, RATIOS, n, u, top_p=top_p)
    for b in range(len(LENS)):
        srv.release(b)
    srv.pool.free.reverse()
    again = srv.generate(prompts, RATIOS, n, u, top_p=top_p)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert torch.isfinite(first[1]).all() and (first[1] <= 0).all()


def test_refusals(A):
    shape = NEOX_F32
    srv, _, _ = make(A, shape, "same", 16, n_pages=8, max_len=80)
    _, prompts = prompts_of(shape)
    with pytest.raises(MemoryError, match="free"):
        srv.prefill(prompts, RATIOS)
    with pytest.raises(ValueError, match="prompts"):
        srv.prefill(prompts[:2], RATIOS)
    with pytest.raises(ValueError, match="prompts"):
        srv.prefill([p[:0] for p in prompts], RATIOS)
    with pytest.raises(ValueError, match="flags"):
        from paper_2607_21291_gb300 import serve
        serve.Server(A.make_cfg(shape, A.FLAG_GATE_SIGMOID), [], {}, srv.head, 1, 16, 1)


def test_a_released_sequence_stays_released(A):
    """A sequence that is released between steps takes no page again, nor does a layer that keeps nothing; the others go on
    with the pages that it gave back, past the length where it would have had to stop, and answer as without the release."""
    shape = NEOX_SMALL
    ids, prompts = prompts_of(shape)
    srv, _, _ = make(A, shape, "same", 16, n_pages=14, max_len=75)     # the prompts fill the pool
    other, _, _ = make(A, shape, "same", 16)
    assert torch.equal(srv.prefill(prompts, RATIOS), other.prefill(prompts, RATIOS))
    assert not srv.pool.free
    srv.release(0)
    free = len(srv.pool.free)
    assert free == 7
    for step in range(12):
        tok = torch.tensor([int(ids[b, n + step]) for b, n in enumerate(LENS)], dtype=torch.int32, device="cuda")
        flags = [torch.empty(shape.n_layers, len(LENS), dtype=torch.bool, device="cuda") for _ in range(2)]
        got, want = srv.step(tok, flags[0]), other.step(tok, flags[1])
        assert torch.equal(flags[0][:, 1:], flags[1][:, 1:]) and not flags[0][:, 0].any()
        H.assert_close(H.to_np(got[1:]), H.to_np(want[1:]), H.tol(shape), f"step {step}")
        assert (srv.pool.held[:, 0] == 0).all() and (srv.pool.held[2] == 0).all() and (other.pool.held[2] == 0).all()
        assert (srv.lens[:, 0] == 0).all()
    srv.check()
    assert len(srv.pool.free) < free                                   # taken by the others
    # everything released: steps need no page and meet no end
    for b in range(1, len(LENS)):
        srv.release(b)
    for step in range(80):
        srv.step(tok)
    srv.check()
    assert len(srv.pool.free) == 14
    # the pool and the slots serve the next prompts
    assert torch.equal(srv.prefill(prompts, RATIOS), other.prefill(prompts, RATIOS))
    srv.release(3)                                                     # the next step needs a page
    for step in range(5):
        srv.step(tok)
    with pytest.raises(ValueError, match="longer"):                    # 75 tokens
        srv.step(tok)
    srv.release(0)
    srv.step(tok)
    srv.check()


def test_kept_numbers_are_the_librarys(A):
    """Layers keep the numbers that the retention allocation gives, also where r T falls a rounding short of a whole
    number (0.29 x 100, 0.58 x 50) or r a rounding above 1."""
    ids = S.token_ids(32, len(LENS), 100, NEOX_SMALL.vocab)
    lens = [100, 50, 1, 100]
    srv, _, _ = make(A, NEOX_SMALL, "same", 16)
    ratios = [0.29, 0.58, 1.0 + 1e-12]
    kept = []
    srv.prefill([torch.from_numpy(ids[b, :n].astype(np.int64)) for b, n in enumerate(lens)], ratios, kept)
    srv.check()
    want = [[int(O.kept_counts(r, n)) for n in lens] for r in ratios]
    assert want == [[29, 14, 0, 29], [58, 29, 0, 58], [100, 50, 1, 100]]
    assert [[len(k) for k in row] for row in kept] == want == srv.lens.tolist()
    # and no fewer than none, no more than all
    assert [int(O.kept_counts(r, 10)) for r in (-0.5, 2.0)] == [0, 10]
    srv.prefill([torch.from_numpy(ids[b, :10].astype(np.int64)) for b in range(4)], [-0.5, 2.0, 0.5])
    assert srv.lens.tolist() == [[0] * 4, [10] * 4, [5] * 4]


def _slope(x, W):
    """|gradient| of the router's score at rows x, times their rms."""
    h = x @ W["router_w1"].T + W["router_b1"]
    s = 1 / (1 + np.exp(-h))
    g = (W["router_w2"] * s * (1 + h * (1 - s))) @ W["router_w1"]
    return np.linalg.norm(g, axis=-1) * np.sqrt((x * x).mean(-1))


@pytest.mark.parametrize("shape", [QWEN_SMALL, NEOX_SMALL, NEOX_F32], ids=["qwen", "neox", "neox-f32"])
def test_decisions_with_an_8_bit_cache(A, shape):
    """Keep decisions over an 8-bit cache, wherever the score is clear of the threshold. The first layer's scores are of
    embeddings, which no cache changes: 1e-3, as with a cache in the model's type. A later layer's inputs are off by about 2^-7 of
    their rms in bf16, 2^-6 with 8 bits; six standard deviations of that along the router's gradient, for the score and for the
    threshold, come on top. At least half of a layer's decisions have to be clear."""
    srv, W, E = make(A, shape, "i8", 16)
    ids, prompts = prompts_of(shape)
    p = O.params_of(shape)
    kept, states = [], []
    srv.prefill(prompts, RATIOS, kept)
    for b, n in enumerate(LENS):
        force = [k[b].cpu().numpy()[None] for k in kept]
        states.append(O.sparse_prefill(ids[b:b + 1, :n], E, W, p, [f.shape[1] for f in force], idx_force=force)[1])
    clear, all_of = np.zeros(2, dtype=int), np.zeros(2, dtype=int)
    for step in range(18):
        tok = np.array([ids[b, n + step] for b, n in enumerate(LENS)])
        flags = torch.empty(shape.n_layers, len(LENS), dtype=torch.bool, device="cuda")
        srv.step(torch.from_numpy(tok.astype(np.int32)).cuda(), flags)
        flags = flags.cpu().numpy()
        for b in range(len(LENS)):
            thr = [states[b]["thr"][l][0] for l in range(2)]
            _, own, score = O.decode_step(tok[b:b + 1], E, W, p, states[b], kept_force=flags[:, b:b + 1])
            for l in range(2):
                if not np.isfinite(thr[l]):
                    assert not flags[l, b]
                    continue
                margin = 1e-3 + (12 * 2.0 ** -6 * _slope(np.array(states[b]["rows"][l][0]), W[l]).max() if l else 0.0)
                all_of[l] += 1
                if abs(score[l, 0] - thr[l]) > margin:
                    clear[l] += 1
                    assert flags[l, b] == own[l, 0], (step, b, l)
    srv.check()
    assert (2 * clear >= all_of).all() and (all_of > 0).all(), (clear, all_of)


def test_greedy_tokens_that_are_compared(A):
    """Greedy generation against an argmax of the logits in 32 bits, where the two largest are further apart than bf16's
    rounding of both: that has to be so for half of the tokens at least."""
    shape = NEOX_SMALL
    ids, prompts = prompts_of(shape)
    srv, other = make(A, shape, "same", 16)[0], make(A, shape, "same", 64)[0]
    n = 12
    tokens, _ = srv.generate(prompts, RATIOS, n, torch.zeros(n, len(LENS), device="cuda"), temperature=torch.zeros(len(LENS), device="cuda"))
    hidden, compared = other.prefill(prompts, RATIOS), 0
    for i in range(n):
        best = (hidden.float() @ other.head.float().T).topk(2, -1)
        sure = (best.values[:, 0] - best.values[:, 1]) > 2.0 ** -6 * best.values[:, 0].abs()
        assert (tokens[i] == best.indices[:, 0])[sure].all()
        compared += int(sure.sum())
        if i + 1 < n:
            hidden = other.step(tokens[i])
    other.check()
    assert 2 * compared >= n * len(LENS), compared


def test_ratios_are_checked(A):
    """A ratio that is no number, or not one for each layer, is refused and changes nothing."""
    srv, _, _ = make(A, NEOX_SMALL, "same", 16)
    _, prompts = prompts_of(NEOX_SMALL)
    srv.prefill(prompts, RATIOS)
    lens, held = srv.lens.clone(), srv.pool.held.copy()
    for ratios in ([1.0, 0.5], [1.0] * 4, [1.0, float("nan"), 0.5], [1.0, float("inf"), 0.5], []):
        with pytest.raises(ValueError, match="ratio"):
            srv.prefill(prompts, ratios)
    assert torch.equal(srv.lens, lens) and (srv.pool.held == held).all()
    srv.step(torch.zeros(len(LENS), dtype=torch.int32, device="cuda"))
    srv.check()
