"""Pins of the oracles of the operators around the verification step (page plans, rotary positions, token log probabilities) and the
host function that makes rotary frequencies: hand-worked cases, conservation laws, library functions in float64, differences."""
import math

import numpy as np
import pytest
import torch

from oracle.operators_oracle import cache_plan, rope_turn, token_logprobs, token_logprobs_backward


# ---- page plans -------------------------------------------------------------------------------------------------------
def test_a_hand_worked_plan():
    """Pages of 4.  Request 0 holds 6 tokens (pages 9, 2) and wants 9; 1 holds 8 (5, 7) and keeps 3; 2 ends (page 1); 3 begins with 5.
    Free: 3, 8 (8 on top).  Given back: 7, then 1; taken: 1 for request 0, then 7 and 8 for request 3."""
    table = np.array([[9, 2, -1], [5, 7, -1], [1, -1, -1], [-1, -1, -1]], np.int32)
    free = np.array([3, 8, -1, -1, -1, -1, -1, -1, -1, -1], np.int32)
    r = cache_plan([6, 8, 2, 0], [9, 3, 0, 5], table, free, 2, 4, 10)
    assert r["table"].tolist() == [[9, 2, 1], [5, 7, -1], [1, -1, -1], [7, 8, -1]]
    assert r["count"] == 1 and r["free"][0] == 3
    assert r["seq_lens"].tolist() == [9, 3, 0, 5] and r["row_start"].tolist() == [0, 3, 3, 3, 8]
    assert r["positions"].tolist() == [6, 7, 8, 0, 1, 2, 3, 4, 0, 0]
    assert r["slots"].tolist() == [10, 11, 4, 28, 29, 30, 31, 32, -1, -1]
    assert r["info"].tolist() == [8, 3, 2, 0]


def test_refusals_of_a_plan():
    table = np.full((4, 2), -1, np.int32)
    free = np.arange(3, dtype=np.int32)
    # request 1 does not fit its row of the table: refused alone.  Request 2 finds one page left of two: it and request 3 are refused.
    r = cache_plan([0, 0, 0, 0], [8, 9, 8, 1], table, free, 3, 4, 100)
    assert r["seq_lens"].tolist() == [8, 0, 0, 0] and r["info"].tolist() == [8, 2, 0, 3] and r["count"] == 1
    # the rows run out at request 2
    r = cache_plan([0, 0, 0, 0], [4, 0, 4, 1], table, free, 3, 4, 7)
    assert r["seq_lens"].tolist() == [4, 0, 0, 0] and r["info"].tolist() == [4, 1, 0, 2]


def test_no_page_is_lost_or_owned_twice():
    rng = np.random.default_rng(3)
    for _ in range(30):
        B, page, width = int(rng.integers(1, 40)), int(rng.choice([1, 4, 16])), 12
        pages = lambda n: -(-n // page)
        held = rng.integers(0, page * width + 1, B)
        ids = rng.permutation(B * width + 30)
        table = np.full((B, width), -1, np.int32)
        at = 0
        for b in range(B):
            table[b, :pages(held[b])] = ids[at:at + pages(held[b])]
            at += pages(held[b])
        n = int(rng.integers(0, len(ids) - at + 1))
        free = np.full(len(ids), -1, np.int32)
        free[:n] = ids[at:at + n]
        r = cache_plan(held, rng.integers(0, page * width + 1, B), table, free, n, page, 10 ** 6)
        owned = [r["table"][b, i] for b in range(B) for i in range(pages(r["seq_lens"][b]))] + list(r["free"][:r["count"]])
        assert sorted(owned) == sorted(ids[:at + n])
        live = r["slots"][:r["info"][0]]
        assert len(set(live.tolist())) == len(live)


# ---- rotary positions ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("interleaved", [False, True])
def test_turns_keep_norms_and_see_only_distances(interleaved):
    rng = np.random.default_rng(4)
    f = 10000.0 ** (-np.arange(8) / 8)
    q, k = rng.standard_normal((2, 1, 1, 20))
    turn = lambda x, t: rope_turn(x, [t], f, 16, interleaved)
    assert np.allclose(np.linalg.norm(turn(q, 77)), np.linalg.norm(q))
    assert np.allclose((turn(q, 100) * turn(k, 93)).sum(), (turn(q, 7) * turn(k, 0)).sum())
    assert np.array_equal(turn(q, 5)[..., 16:], q[..., 16:]) and np.array_equal(turn(q, 0), q)
    assert np.allclose(rope_turn(turn(q, 9), [9], f, 16, interleaved, back=True), q)
    # the transpose: <R q, k> = <q, R^T k>
    assert np.allclose((rope_turn(q, [9], f, 16, interleaved, 1.3) * k).sum(), (q * rope_turn(k, [9], f, 16, interleaved, 1.3, back=True)).sum())


def test_a_quarter_turn_by_hand():
    f = [math.pi / 2, math.pi]
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    assert np.allclose(rope_turn(x, [1], f, 4, False), [[[-3, -2, 1, -4]]])   # pairs (1, 3) and (2, 4)
    assert np.allclose(rope_turn(x, [1], f, 4, True), [[[-2, 1, -3, -4]]])    # pairs (1, 2) and (3, 4)


def test_frequencies_of_the_host_function():
    import paper_2602_06932_amd as av
    R, base, ctx = 128, 10000.0, 4096.0
    plain = base ** (-2.0 * np.arange(R // 2) / R)
    make = lambda kind, **kw: av.aurora_rope_frequencies(av.aurora_rope_scaling(rotary_dim=R, kind=kind, base=base, **kw))
    f, m = make(av.AURORA_ROPE_PLAIN)
    assert np.allclose(f, plain, rtol=1e-14) and m == 1.0
    f, _ = make(av.AURORA_ROPE_LINEAR, factor=8.0)
    assert np.allclose(f, plain / 8, rtol=1e-14)
    f, _ = make(av.AURORA_ROPE_BASE, factor=8.0)
    assert f[0] == 1.0 and np.isclose(f[-1], plain[-1] / 8, rtol=1e-12) and np.all(np.diff(f) < 0)
    f, m = make(av.AURORA_ROPE_BANDS, factor=8.0, trained_context=ctx, low=1.0, high=4.0)
    turns = ctx * plain / (2 * np.pi)
    for i in range(R // 2):
        want = plain[i] if turns[i] >= 4 else plain[i] / 8 if turns[i] <= 1 else \
            (turns[i] - 1) / 3 * plain[i] + (4 - turns[i]) / 3 * plain[i] / 8
        assert np.isclose(f[i], want, rtol=1e-12)
    assert m == 1.0
    f, m = make(av.AURORA_ROPE_RAMP, factor=8.0, trained_context=ctx, low=1.0, high=32.0)
    lo = max(0, int(np.sum(turns > 32)) - 1)     # the last pair that makes more turns than that, and the first that makes fewer
    hi = int(np.sum(turns >= 1))
    assert np.allclose(f[:lo + 1], plain[:lo + 1], rtol=1e-12) and np.allclose(f[hi:], plain[hi:] / 8, rtol=1e-12)
    mid = np.arange(lo, hi + 1)
    keep = 1 - (mid - lo) / (hi - lo)
    assert np.allclose(np.array(f)[mid], keep * plain[mid] + (1 - keep) * plain[mid] / 8, rtol=1e-12)
    assert np.isclose(m, 0.1 * math.log(8.0) + 1, rtol=1e-6)
    for bad in (dict(kind=9, factor=2.0), dict(kind=av.AURORA_ROPE_LINEAR, factor=0.5),
                dict(kind=av.AURORA_ROPE_BANDS, factor=2.0, trained_context=ctx, low=4.0, high=4.0),
                dict(kind=av.AURORA_ROPE_RAMP, factor=2.0, trained_context=0.0, low=1.0, high=4.0)):
        with pytest.raises(av.AuroraError) as e:
            make(**bad)
        assert e.value.status == av.AURORA_ERR_INVALID_ARG
    for R2, b2 in ((0, 10.0), (7, 10.0), (4, 1.0), (4, float("nan"))):
        with pytest.raises(av.AuroraError):
            av.aurora_rope_frequencies(av.aurora_rope_scaling(rotary_dim=R2, kind=0, base=b2))


# ---- token log probabilities -------------------------------------------------------------------------------------------------
def _logits(rng, M, V):
    z = rng.standard_normal((M, V)) * 3
    z[:, rng.integers(0, V, max(1, V // 10))] = -np.inf
    z[:, 0] = 1.0
    return z


def test_log_probabilities_against_the_library():
    rng = np.random.default_rng(5)
    z, tok, T = _logits(rng, 9, 41), rng.integers(0, 41, 9), 0.7
    r = token_logprobs(z, tok, T, n_top=6)
    lp = torch.log_softmax(torch.tensor(z) / T, -1)
    assert np.allclose(r["logprob"], lp[torch.arange(9), torch.tensor(tok)].numpy(), rtol=1e-12, atol=0)
    assert np.allclose(r["entropy"], torch.distributions.Categorical(logits=torch.tensor(z).clamp(min=-1e9) / T).entropy().numpy(), rtol=1e-10)
    v, i = torch.tensor(z).topk(6)
    assert np.array_equal(r["top_ids"], i.numpy()) and np.allclose(r["top_logprobs"], lp.gather(1, i).numpy())


def test_ties_masks_and_rows_without_a_token():
    z = np.array([[1.0, 2.0, 2.0, -0.0, 0.0], [-np.inf] * 5, [-np.inf, -np.inf, 3.0, -np.inf, -np.inf]])
    r = token_logprobs(z, [7, 2, -1], 1.0, n_top=7)
    assert r["top_ids"].tolist() == [[1, 2, 0, 3, 4, -1, -1], [0, 1, 2, 3, 4, -1, -1], [2, 0, 1, 3, 4, -1, -1]]
    assert r["logprob"].tolist() == [0.0, -np.inf, 0.0] and r["lse"][1] == -np.inf and r["entropy"][1] == 0 and r["entropy"][2] == 0
    assert r["lse"][2] == 3.0 and r["top_logprobs"][2].tolist() == [0.0] + [-np.inf] * 6


def test_gradient_against_reverse_mode_differentiation_and_differences():
    rng = np.random.default_rng(6)
    M, V, T = 5, 23, 1.3
    z, tok = rng.standard_normal((M, V)) * 2, np.array([3, -1, 22, 0, 9])
    gl, gh = rng.standard_normal((2, M))
    g = token_logprobs_backward(z, tok, T, gl, gh)
    x = torch.tensor(z, requires_grad=True)
    lp = torch.log_softmax(x / T, -1)
    known = torch.tensor(tok >= 0)
    picked = torch.where(known, lp[torch.arange(M), torch.tensor(tok).clamp(min=0)], torch.zeros(M, dtype=torch.float64))
    ((picked * torch.tensor(gl)).sum() - (lp.exp() * lp).sum(1) @ torch.tensor(gh)).backward()
    assert np.allclose(g, x.grad.numpy(), rtol=1e-10, atol=1e-13)

    def loss(z):
        r = token_logprobs(z, tok, T)
        return r["logprob"] @ gl + r["entropy"] @ gh
    for m, v in ((0, 3), (0, 4), (1, 7), (2, 22), (4, 1)):
        zp, zm = z.copy(), z.copy()
        zp[m, v] += 1e-5
        zm[m, v] -= 1e-5
        assert abs((loss(zp) - loss(zm)) / 2e-5 - g[m, v]) < 1e-8
