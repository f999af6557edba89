"""Token log probabilities, entropies, alternatives and the gradient against the float64 oracle.

Tolerances, per row, with x = z / T, m = max x, p the probabilities and u = 2^-24 (half a step of fp32):
  log2(e) / T is rounded twice: all x are off by the same factor 1 +- 2u;
  an exponent d = (x - m) log2 e is one fused product, off by u |d|, its exponential by 2u more, the sums of at most 32 values by 10 u:
  a weight p is off by e = u (2 |x - m| + 16), relative.
  lse      2u max|x| + sum p e + u |lse|          (the common factor moves lse by at most max |x| times itself)
  logprob  2u |x_t - E x| + sum p e + u |logprob|
  entropy  2u Var x + sum p e (|log p + H| + 1) + 16 u sum p |x - m| + u H
  dz       p off by u (2 |x| + 2 |lse| + 2 |log p| + 16): the logsumexp is handed over in fp32; log p + H by u (2 |x| + 2 |lse| + 2 H + 8);
           half a step of the result on top (bfloat16: 2^-8)."""
import numpy as np
import pytest
import torch

from oracle.operators_oracle import token_logprobs, token_logprobs_backward

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def _logits(seed, M, V, dtype, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(M, V, generator=g) * 2.5
    if kind == "peaked":
        z[torch.arange(M), torch.randint(0, V, (M,), generator=g)] += 15
    if kind == "masked":          # minus infinity, the lowest finite value, a row with nothing left, rows with less than the alternatives
        z[:, torch.rand(V, generator=g) < 0.3] = -float("inf")
        z[:, torch.rand(V, generator=g) < 0.1] = torch.finfo(DT[dtype]).min
        z[0] = -float("inf")
        if M > 2:
            z[1, 2:] = -float("inf")
            z[1, :2] = 1.0
            z[2] = torch.finfo(DT[dtype]).min
    if kind == "equal":
        z[:] = 0.25
        z[M // 2:] = torch.randint(0, 2, (M - M // 2, V), generator=g).float()
        z[0] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    if kind == "rising":          # the largest ones side by side
        z = torch.linspace(-8, 8, V).expand(M, V).clone()
        z[M // 2:] = z[M // 2:].flip(1)
    return z.to(DT[dtype])


def _place(z, stride, shift):
    """z on the GPU with rows `stride` apart, starting `shift` elements past an aligned address; and the whole buffer."""
    M, V = z.shape
    buf = torch.full((shift + M * stride + 8,), 3.0, dtype=z.dtype, device="cuda")
    view = torch.as_strided(buf, (M, V), (stride, 1), shift)
    view.copy_(z)
    return view, buf


def _run(av, z, tokens, T, n_top, stride=0, shift=0, temps=None):
    M, V = z.shape
    view, buf = _place(z, stride or V, shift)
    d = av.aurora_logprob_desc(rows=M, vocab=V, dtype=av.AURORA_F32 if z.dtype == torch.float32 else av.AURORA_BF16, n_top=n_top,
                               row_stride=stride, temperature=T, temperatures=None if temps is None else temps.data_ptr())
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    o = dict(logprob=nan(M), entropy=nan(M), lse=nan(M), top_ids=torch.full((M, n_top), -7, dtype=torch.int32, device="cuda") if n_top else None,
             top_logprobs=nan(M, n_top) if n_top else None)
    ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    tok = torch.from_numpy(np.asarray(tokens, np.int32)).cuda()
    av.aurora_token_logprobs(d, view, tok, o["logprob"], o["entropy"], o["lse"], o["top_ids"], o["top_logprobs"], ws)
    torch.cuda.synchronize()
    return {k: None if v is None else v.cpu().numpy() for k, v in o.items()}, (d, view, buf, tok, o)


def _inf_close(got, ref, tol):
    # the results are float32: the lowest value, -(2 - 2^-23) 2^127, is at T = 0.8 1.25 times that, which rounds to minus infinity
    ref = np.where(ref <= -(2.0 - 2.0 ** -24) * 2.0 ** 127, -np.inf, ref)
    same = np.isneginf(ref)
    assert np.array_equal(np.isneginf(got), same)
    with np.errstate(invalid="ignore"):
        off = np.abs(got - ref)
    assert np.isfinite(got[~same]).all() and (off[~same] <= tol[~same]).all(), (off[~same] - tol[~same]).max()


def _check(av, z, tokens, T=1.0, n_top=0, temps=None, grad=True, seed=0, **kw):
    M, V = z.shape
    print(f"[case] {M} x {V} {z.dtype} n_top={n_top} T={T} {kw}", flush=True)
    got, (d, view, buf, tok, o) = _run(av, z, tokens, T, n_top, temps=temps, **kw)
    Tr = np.full(M, T) if temps is None else np.where(temps.cpu().numpy() > 0, temps.cpu().numpy(), 1.0)
    zz = z.double().numpy()
    ref = token_logprobs(zz, tokens, Tr, n_top)
    x = zz / Tr[:, None]
    fin = np.where(np.isfinite(x), x, 0.0)
    lse0 = np.where(np.isneginf(ref["lse"]), 0.0, ref["lse"])
    lp = np.where(np.isfinite(x), x - lse0[:, None], 0.0)
    p = np.where(np.isfinite(x), np.exp(x - lse0[:, None]), 0.0)
    dist = np.where(p > 0, np.abs(fin - np.where(p > 0, fin, -np.inf).max(1, initial=-np.inf, keepdims=True)), 0.0)
    e = U * (2 * dist + 16)
    pe = (p * e).sum(1)
    mean = (p * fin).sum(1)
    top = np.where(p > 0, np.abs(fin), 0.0).max(1)     # (values without weight do not move the sums)
    x_t = fin[np.arange(M), np.clip(tokens, 0, V - 1)]
    _inf_close(got["lse"], ref["lse"], 2 * U * top + pe + U * np.abs(lse0))
    _inf_close(got["logprob"], ref["logprob"], 2 * U * np.abs(x_t - mean) + pe + U * np.where(np.isfinite(ref["logprob"]), np.abs(ref["logprob"]), 0))
    H = ref["entropy"]
    var = (p * (fin - mean[:, None]) ** 2).sum(1)
    tol_h = 2 * U * var + (p * e * (np.abs(lp + H[:, None]) + 1)).sum(1) + 16 * U * (p * dist).sum(1) + U * H
    _inf_close(got["entropy"], H, tol_h)
    if n_top:
        assert np.array_equal(got["top_ids"], ref["top_ids"])
        picked = np.take_along_axis(fin, np.clip(ref["top_ids"], 0, None), 1)
        tl = np.where(np.isfinite(ref["top_logprobs"]), np.abs(ref["top_logprobs"]), 0)
        _inf_close(got["top_logprobs"], ref["top_logprobs"], 2 * U * np.abs(picked - mean[:, None]) + pe[:, None] + U * tl)
    if not grad:
        return
    rng = np.random.default_rng(seed)
    gl, gh = rng.standard_normal((2, M)).astype(np.float32)
    gref = token_logprobs_backward(zz, tokens, Tr, gl.astype(np.float64), gh.astype(np.float64))
    tolp = U * (2 * np.abs(fin) + 2 * np.abs(lse0)[:, None] + 2 * np.abs(lp) + 16)
    tol = p * (np.abs(gl)[:, None] * tolp + np.abs(gh)[:, None] * (np.abs(lp + H[:, None]) * tolp + U * (2 * np.abs(fin) + 2 * np.abs(lse0)[:, None] + 2 * H[:, None] + 8) + tol_h[:, None]))
    tol = tol / Tr[:, None] + 4 * U * np.abs(gl)[:, None] / Tr[:, None] + (2.0 ** -8 if z.dtype == torch.bfloat16 else 4 * U) * np.abs(gref) + 1e-38
    dl, de = torch.from_numpy(gl).cuda(), torch.from_numpy(gh).cuda()
    before = buf.clone()
    # where the logits' rows lie, and elsewhere within 16 bytes
    for out in (torch.full_like(buf, 9.0), torch.full((buf.numel() + 1,), 9.0, dtype=buf.dtype, device="cuda")[1:]):
        gview = torch.as_strided(out, view.shape, view.stride(), view.storage_offset() + out.storage_offset())
        av.aurora_token_logprobs_backward(d, view, tok, o["entropy"], o["lse"], dl, de, gview)
        torch.cuda.synchronize()
        g = gview.double().cpu().numpy()
        assert np.isfinite(g).all() and (np.abs(g - gref) <= tol).all(), (np.abs(g - gref) - tol).max()
        rest = torch.ones_like(out, dtype=torch.bool)
        torch.as_strided(rest, view.shape, view.stride(), view.storage_offset()).fill_(False)
        assert (out[rest] == 9.0).all()                    # between the rows, and around them
    assert torch.equal(buf.view(torch.uint8), before.view(torch.uint8))
    av.aurora_token_logprobs_backward(d, view, tok, o["entropy"], o["lse"], dl, de, view)  # in place
    torch.cuda.synchronize()
    assert torch.equal(view, torch.as_strided(out, view.shape, view.stride(), view.storage_offset() + out.storage_offset()))


def _tokens(seed, M, V):
    t = np.random.default_rng(seed).integers(0, V, M)
    if M > 3:
        t[1], t[3] = -1, V
    return t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 31, 100, 777, 2049, 16001, 32003])
def test_vocabularies_short_and_odd(gpu_lib, vocab, dtype):
    for M, n_top, T in ((1, 5, 1.0), (6, 32, 0.7), (6, 1, 1.5)):
        _check(gpu_lib, _logits(vocab + M, M, vocab, dtype), _tokens(vocab, M, vocab), T, n_top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["peaked", "masked", "equal", "rising"])
def test_rows_that_are_masked_equal_or_sorted(gpu_lib, kind, dtype):
    for M, V, n_top in ((6, 50, 8), (6, 5003, 32), (7, 70001, 20)):
        _check(gpu_lib, _logits(V, M, V, dtype, kind), _tokens(V, M, V), 1.0, n_top, grad=V < 60000)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_full_vocabularies_and_many_rows(gpu_lib, dtype):
    _check(gpu_lib, _logits(1, 5, 128256, dtype, "peaked"), _tokens(1, 5, 128256), 1.0, 5)
    _check(gpu_lib, _logits(2, 40, 128257, dtype), _tokens(2, 40, 128257), 0.7, 20, grad=False)
    _check(gpu_lib, _logits(3, 700, 4099, dtype), _tokens(3, 700, 4099), 1.0, 3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,kind", [(1, "rising"), (2, "masked"), (9, "equal"), (33, "masked"), (64, "rising"), (65, "equal"), (100, "masked")])
def test_rows_in_parts_of_every_size(gpu_lib, M, kind, dtype):
    """From one step of a row to a part's four, in as many parts as the number of rows makes of it."""
    _check(gpu_lib, _logits(40 + M, M, 65541, dtype, kind), _tokens(M, M, 65541), 0.8, 32, grad=False)
    _check(gpu_lib, _logits(41 + M, M, 65541, dtype), _tokens(M, M, 65541), 1.0, 0, grad=False)


@pytest.mark.parametrize("kind", ["masked", "equal", "rising"])
def test_one_workgroup_a_row(gpu_lib, kind):
    """So many rows that none is split: the selection's rare paths write the results themselves."""
    for dtype in ("f32", "bf16"):
        z = _logits(5, 520, 9001, dtype, kind)
        _check(gpu_lib, z, _tokens(5, 520, 9001), 1.0, 32, grad=False)


def test_rows_longer_than_a_workgroup_takes(gpu_lib):
    _check(gpu_lib, _logits(6, 520, 300001, "f32")[:520], _tokens(6, 520, 300001), 1.0, 4, grad=False)
    z = _logits(7, 1, 1 << 24, "bf16")
    _check(gpu_lib, z, [12345678], 1.0, 32, grad=False)


def test_more_rows_than_a_launch_counts_in_one_dimension(gpu_lib):
    av = gpu_lib
    M, V = (1 << 22) + 5, 3
    z = torch.randn(M, V, device="cuda")
    tok = torch.randint(0, V, (M,), device="cuda", dtype=torch.int32)
    d = av.aurora_logprob_desc(rows=M, vocab=V, dtype=av.AURORA_F32, n_top=1)
    ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    lp, H, lse, tl = (torch.full((M,), 7.0, device="cuda") for _ in range(4))
    ti, g = torch.full((M,), -7, dtype=torch.int32, device="cuda"), torch.zeros_like(z)
    av.aurora_token_logprobs(d, z.view(1, M, V), tok, lp, H, lse, ti, tl, ws)
    av.aurora_token_logprobs_backward(d, z, tok, None, lse, torch.ones(M, device="cuda"), None, g)
    torch.cuda.synchronize()
    ref = torch.log_softmax(z.double(), -1)
    # three values: every sum within a few ulp of numbers below 16
    assert (lp - ref.gather(1, tok.long()[:, None])[:, 0]).abs().max() < 4e-6
    assert (H + (ref.exp() * ref).sum(1)).abs().max() < 4e-6 and torch.equal(ti, z.argmax(1).to(torch.int32))
    want = torch.nn.functional.one_hot(tok.long(), V) - ref.exp()
    assert (g - want).abs().max() < 4e-6


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_rows_apart_and_not_aligned(gpu_lib, shift, dtype):
    for V, stride in ((1000, 1024), (1003, 1111), (5, 9)):
        _check(gpu_lib, _logits(V, 9, V, dtype), _tokens(V, 9, V), 0.9, 6, stride=stride, shift=shift)


@pytest.mark.parametrize("dtype,M", [("f32", 700), ("bf16", 1400)])
def test_large_calls_and_calls_that_leave_results_out(gpu_lib, dtype, M):
    """Logits that are read past the caches and ones that are not: equal bits, forward with and without lse, back whole and in pieces."""
    av = gpu_lib
    V, step = 20003, 100
    z = _logits(39, M, V, dtype).cuda()
    tok = torch.from_numpy(_tokens(39, M, V).astype(np.int32)).cuda()
    code = av.AURORA_F32 if dtype == "f32" else av.AURORA_BF16
    new = lambda: torch.full((M,), float("nan"), device="cuda")
    lp, H, lse, lp2, H2 = (new() for _ in range(5))
    d = av.aurora_logprob_desc(rows=M, vocab=V, dtype=code)
    ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    av.aurora_token_logprobs(d, z, tok, lp, H, lse, None, None, ws)
    av.aurora_token_logprobs(d, z, tok, lp2, H2, None, None, None, ws)
    g, pieces = torch.zeros_like(z), torch.zeros_like(z)
    av.aurora_token_logprobs_backward(d, z, tok, H, lse, lp, H, g)
    for o in range(0, M, step):
        s = slice(o, o + step)
        av.aurora_token_logprobs_backward(av.aurora_logprob_desc(rows=step, vocab=V, dtype=code), z[s], tok[s], H[s], lse[s], lp[s], H[s], pieces[s])
    torch.cuda.synchronize()
    assert torch.equal(lp, lp2) and torch.equal(H, H2) and torch.equal(g, pieces)
    # fp32: a log probability of about -13, its sums off by 2^-20 at most
    ref = torch.log_softmax(z.double(), -1)
    known = (tok >= 0) & (tok < V)
    want = ref.gather(1, tok.clamp(0, V - 1).long()[:, None])[:, 0] * known
    assert (lp - want).abs().max() < 8e-6 and (H + (ref.exp() * ref).sum(1)).abs().max() < 8e-6


def test_rows_past_32_bits(gpu_lib):
    """Rows of logits 2^31 elements apart, and their gradient in place: what the same rows side by side give."""
    av = gpu_lib
    M, V, far = 3, 5003, 2 ** 31 + 8
    near = _logits(12, M, V, "f32").cuda()
    wide = torch.zeros((M - 1) * far + V, device="cuda")
    z = wide.as_strided((M, V), (far, 1))
    z.copy_(near)
    tok = torch.tensor([4, 5002, 77], dtype=torch.int32, device="cuda")
    got = []
    for x, stride in ((z, far), (near.clone(), 0)):
        d = av.aurora_logprob_desc(rows=M, vocab=V, dtype=av.AURORA_F32, n_top=4, row_stride=stride)
        ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        o = [torch.zeros(M, device="cuda") for _ in range(3)] + [torch.zeros((M, 4), dtype=torch.int32, device="cuda"), torch.zeros((M, 4), device="cuda")]
        av.aurora_token_logprobs(d, x, tok, *o, ws)
        av.aurora_token_logprobs_backward(d, x, tok, o[1], o[2], o[0], o[1], x)
        got.append(o + [x.clone()])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(got[1][0].cpu(), got[0][0].cpu()) and not bool(wide[V:far].any()) and not bool(wide[far + V:2 * far].any())


def test_a_temperature_for_every_row(gpu_lib):
    temps = torch.tensor([0.5, 0.0, 1.0, 2.0, 0.0, 0.1, 3.0], device="cuda")
    _check(gpu_lib, _logits(9, 7, 3001, "f32"), _tokens(9, 7, 3001), 1.0, 7, temps=temps)


@pytest.mark.parametrize("vocab", [301, 50001])
def test_rows_that_share_a_temperature(gpu_lib, vocab):
    """Rows in threes, the last ones a part of their three: what as many entries give."""
    av = gpu_lib
    M, z = 8, _logits(38, 8, vocab, "f32").cuda()
    tok = torch.arange(M, dtype=torch.int32, device="cuda")
    temps = torch.tensor([0.6, 0.0, 1.9], device="cuda")
    each = temps.repeat_interleave(3)[:M].contiguous()
    got = []
    for t, share in ((temps, 3), (each, 0)):
        d = av.aurora_logprob_desc(rows=M, vocab=vocab, dtype=av.AURORA_F32, n_top=4, temperatures=t.data_ptr(), temperature_rows=share)
        lp, H, lse, tl, ti = *(torch.zeros(M, device="cuda") for _ in range(3)), torch.zeros(M, 4, device="cuda"), torch.zeros(M, 4, dtype=torch.int32, device="cuda")
        ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        g = torch.zeros_like(z)
        av.aurora_token_logprobs(d, z, tok, lp, H, lse, ti, tl, ws)
        av.aurora_token_logprobs_backward(d, z, tok, H, lse, lp, H, g)
        got.append((lp, H, lse, ti, tl, g))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_temperatures_far_from_one(gpu_lib, dtype):
    """Masked rows where a scaled limit of the type overflows, in all the ways a row is dealt out; logits past each other's range."""
    for T in (5.9, 50.0, 3e4, 1e38):
        _check(gpu_lib, _logits(31, 6, 5003, dtype, "masked"), _tokens(31, 6, 5003), T, 8)
    for M, V in ((700, 5003), (1100, 777)):
        _check(gpu_lib, _logits(32, M, V, dtype, "masked"), _tokens(32, M, V), 8.0, 4, grad=False)
    z = _logits(33, 6, 5003, dtype)
    z[:, ::3] = -float("inf")
    _check(gpu_lib, z, _tokens(33, 6, 5003), 1e-30, 8)
    _check(gpu_lib, z, _tokens(33, 6, 5003), 1e-35, 8)          # (a gradient of 10^35: times a logarithm's limit it is finite)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_large_values(gpu_lib, dtype):
    """Nothing left but a mask's value, of any size; or large values next to each other, whose exponents are larger than their steps."""
    for M, n_top in ((9, 5), (660, 5)):
        z = torch.empty(M, 1500)
        for m in range(M):
            z[m] = [-1e5, -1e6, -3e7, -1e9, -1e10, -1e15, -1e30, 1e10, 2e37][m % 9]
        z[:, 7::50] = -float("inf")
        for T in (1.0, 0.37, 5.9):
            _check(gpu_lib, z.to(DT[dtype]), _tokens(35, M, 1500), T, n_top, grad=False)
    z = _logits(36, 12, 1500, "f32")
    z[:] = z.to(DT[dtype])
    big = torch.tensor([2.0 ** e for e in (10, 16, 19, 20, 21, 22)]).repeat(2)[:, None]
    z = (z.clamp(-3, 3) + torch.cat([big[:6], -big[6:]])).to(DT[dtype])
    for T in (1.0, 3.0):
        _check(gpu_lib, z, _tokens(37, 12, 1500), T, 5, grad=False)


def test_temperatures_past_the_normal_numbers(gpu_lib):
    """Those below 2^-126 count as that, infinity as the largest finite one."""
    z = _logits(34, 4, 3001, "f32", "masked")
    tok = _tokens(34, 4, 3001)
    big = float(torch.finfo(torch.float32).max)
    for odd, like in ((1e-42, 2.0 ** -126), (float("inf"), big)):
        got, want = (_run(gpu_lib, z, tok, 1.0, 4, temps=torch.full((4,), T, device="cuda"))[0] for T in (odd, like))
        for name in got:
            assert np.array_equal(got[name], want[name]), (odd, name)
            assert not np.isnan(got[name].astype(np.float64)).any(), (odd, name)
    assert np.array_equal(_run(gpu_lib, z, tok, 1e-42, 4)[0]["top_logprobs"], _run(gpu_lib, z, tok, 2.0 ** -126, 4)[0]["top_logprobs"])


def test_nan_and_infinity_reach_the_results_of_their_row_alone(gpu_lib):
    z = _logits(10, 6, 5000, "f32")
    z[1, 77], z[2, 4999], z[4] = float("nan"), float("inf"), float("nan")
    tok = np.full(6, 5)
    got, (d, view, buf, t, o) = _run(gpu_lib, z, tok, 1.0, 8)
    ref = token_logprobs(z[[0, 3, 5]].double().numpy(), tok[[0, 3, 5]], 1.0, 8)
    for k in ("lse", "entropy", "logprob"):
        assert np.isnan(got[k][[1, 2, 4]]).all(), k
        assert np.allclose(got[k][[0, 3, 5]], ref[k], rtol=1e-5, atol=1e-6)
    assert np.array_equal(got["top_ids"][[0, 3, 5]], ref["top_ids"])
    assert ((got["top_ids"] >= -1) & (got["top_ids"] < 5000)).all()
    g = torch.zeros_like(view)
    ones = torch.ones(6, device="cuda")
    gpu_lib.aurora_token_logprobs_backward(d, view, t, o["entropy"], o["lse"], ones, ones, g)
    torch.cuda.synchronize()
    assert torch.isnan(g[[1, 2, 4]]).any(1).all() and torch.isfinite(g[[0, 3, 5]]).all()


def test_parts_of_the_results_and_either_gradient(gpu_lib):
    av = gpu_lib
    z = _logits(11, 4, 3000, "f32").cuda()
    tok = torch.tensor([5, -1, 2999, 0], dtype=torch.int32, device="cuda")
    d = av.aurora_logprob_desc(rows=4, vocab=3000, dtype=av.AURORA_F32)
    ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    e = lambda: torch.zeros(4, device="cuda")
    lp, H, lse, H2, lse2 = e(), e(), e(), e(), e()
    av.aurora_token_logprobs(d, z, tok, lp, H, lse, None, None, ws)
    av.aurora_token_logprobs(d, z, None, None, None, lse2, None, None, ws)
    av.aurora_token_logprobs(d, z, None, None, H2, None, None, None, ws)
    assert torch.equal(lse, lse2) and torch.equal(H, H2)
    gl, gh = torch.randn(4, device="cuda"), torch.randn(4, device="cuda")
    a, b, both = (torch.zeros_like(z) for _ in range(3))
    av.aurora_token_logprobs_backward(d, z, tok, None, lse, gl, None, a)
    av.aurora_token_logprobs_backward(d, z, None, H, lse, None, gh, b)
    av.aurora_token_logprobs_backward(d, z, tok, H, lse, gl, gh, both)
    torch.cuda.synchronize()
    ref = token_logprobs_backward(z.double().cpu().numpy(), tok.cpu().numpy(), 1.0, gl.double().cpu().numpy(), None)
    assert np.allclose(a.cpu().numpy(), ref, rtol=1e-5, atol=1e-7)
    assert torch.allclose(a + b, both, rtol=1e-5, atol=1e-7)


def test_two_graphs_and_a_stream_of_its_own(gpu_lib):
    """Captured calls on new logits; the workspace's contents do not matter from one call to the next."""
    av = gpu_lib
    M, V, n = 12, 40000, 6
    z = _logits(12, M, V, "f32").cuda()
    tok = torch.arange(M, dtype=torch.int32, device="cuda") * 3
    d = av.aurora_logprob_desc(rows=M, vocab=V, dtype=av.AURORA_F32, n_top=n)
    ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    new = lambda: [torch.zeros(M, device="cuda") for _ in range(3)] + [torch.zeros((M, n), dtype=torch.int32, device="cuda"), torch.zeros((M, n), device="cuda")]
    a, b, ref = new(), new(), new()
    g = torch.zeros_like(z)
    torch.cuda.synchronize()

    def step(o):
        av.aurora_token_logprobs(d, z, tok, *o, ws)
        av.aurora_token_logprobs_backward(d, z, tok, o[1], o[2], o[0], o[1], g)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(a)
    side.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        step(a)
    with torch.cuda.graph(g2):
        step(b)
    for k in range(3):
        z.copy_(torch.randn_like(z) * 3)
        ws.fill_(0xff)
        g1.replay()
        g2.replay()
        torch.cuda.synchronize()
        gg = g.clone()
        step(ref)
        torch.cuda.synchronize()
        for x, y, r in zip(a, b, ref):
            assert torch.equal(x, r) and torch.equal(y, r)
        assert torch.equal(gg, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(6, 300), (6, 5000), (6, 70001), (700, 5000), (1100, 777)])
def test_a_masked_token_does_not_hide_what_is_not_a_number(gpu_lib, M, V, dtype):
    """NaN or +inf somewhere in the row and the token at -inf, in all the ways a row is dealt out; beside rows where -inf is right."""
    z = _logits(50, M, V, dtype)
    tok = np.random.default_rng(50).integers(0, V, M)
    z[torch.arange(M), torch.from_numpy(tok)] = -float("inf")
    z[0, (tok[0] + 1) % V], z[1, (tok[1] + V // 2) % V], z[2, (tok[2] - 1) % V] = float("nan"), float("inf"), float("nan")
    z[4] = -float("inf")
    z[5, :] = -float("inf")
    z[5, (tok[5] + 1) % V] = float("nan")                   # nothing else left
    for T, n_top in ((1.0, 0), (0.7, 3)):
        got, _ = _run(gpu_lib, z, tok, T, n_top)
        for k in ("lse", "entropy", "logprob"):
            assert np.isnan(got[k][[0, 1, 2, 5]]).all(), k
        rest = [m for m in range(M) if m not in (0, 1, 2, 5)]
        assert np.isneginf(got["logprob"][rest]).all()
        assert not np.isnan(got["lse"][rest]).any() and not np.isnan(got["entropy"][rest]).any()


def _check_gradient(av, z, tokens, T, seed, exact=True):
    """The gradient alone, against the formula twice.  With the lse and entropy that the call is given, L and H, and i = fp32(1 / T):
      l = x i - L is one fused product, off by u |l|, and held between -256 and 0; l log2 e is off by 2u |l| more, the exponential by 2u:
      p = e^l is off by u (3 |l| + 3), relative, and by 2^-126 where it is less than that; g_l i, g_H i and the sum with H by 4u:
      dz off by p i (|g_l + g_H (l + H)| u (3 |l| + 6) + |g_H| u |l| + 4u (|g_l| + |g_H| (|l| + H))), and half a step of the result.
    And with exact ones: the given lse is off by u |lse|, the common factor's 2u max|x| and the sums' e (see above), x i by u |x|, so that l
    is off by
      y = u (2 max|x| + 2 |lse| + |x| + 16) + sum p e,   p by e^y - 1, relative, and log p + H by y and by what H is off."""
    M, V = z.shape
    T = float(np.float32(T))
    print(f"[case] gradient {M} x {V} {z.dtype} T={T}", flush=True)
    got, (d, view, buf, tok, o) = _run(av, z, tokens, T, 0)
    rng = np.random.default_rng(seed)
    gl, gh = rng.standard_normal((2, M)).astype(np.float32)
    g = torch.full_like(view, 9.0)
    av.aurora_token_logprobs_backward(d, view, tok, o["entropy"], o["lse"], torch.from_numpy(gl).cuda(), torch.from_numpy(gh).cuda(), g)
    torch.cuda.synchronize()
    g, zz = g.double().cpu().numpy(), z.double().numpy()
    half = 2.0 ** -8 if z.dtype == torch.bfloat16 else U
    hit = np.arange(V)[None] == np.asarray(tokens)[:, None]
    gl, gh = np.where(hit.any(1), gl, 0.0).astype(np.float64)[:, None], gh.astype(np.float64)[:, None]

    L, H = (got[k].astype(np.float64)[:, None] for k in ("lse", "entropy"))
    assert np.isfinite(L).all() and np.isfinite(H).all()
    i = float(np.float32(1.0) / np.float32(T))
    l = np.clip(zz * i - L, -256.0, 0.0)
    p, inner = np.exp(l), gl + gh * (l + H)
    ref = (hit * gl - p * inner) * i
    off = p * i * (np.abs(inner) * U * (3 * np.abs(l) + 6) + np.abs(gh) * U * np.abs(l) + 4 * U * (np.abs(gl) + np.abs(gh) * (np.abs(l) + H)))
    off += 2.0 ** -126 * i * np.abs(inner) + 2 * U * i * hit * np.abs(gl)
    off += half * (np.abs(ref) + off) + 2.0 ** -126
    assert np.isfinite(g).all() and (np.abs(g - ref) <= off).all(), (np.abs(g - ref) - off).max()
    if not exact:
        return
    x, f = zz / T, token_logprobs(zz, tokens, T)
    ref = token_logprobs_backward(zz, tokens, T, gl[:, 0], gh[:, 0])
    lse, H = f["lse"][:, None], f["entropy"][:, None]
    lp = x - lse
    p, dist, mean = np.exp(lp), np.abs(x - x.max(1, keepdims=True)), (np.exp(lp) * x).sum(1, keepdims=True)
    e = U * (2 * dist + 16)
    pe = (p * e).sum(1, keepdims=True)
    y = U * (2 * np.abs(x).max(1, keepdims=True) + 2 * np.abs(lse) + np.abs(x) + 16) + pe
    off_h = 2 * U * (p * (x - mean) ** 2).sum(1, keepdims=True) + (p * e * (np.abs(lp + H) + 1)).sum(1, keepdims=True) + 16 * U * (p * dist).sum(1, keepdims=True) + U * H
    inner = gl + gh * (lp + H)
    off = p / T * (np.abs(inner) * (np.expm1(y) + U * (3 * np.abs(lp) + 6)) + np.abs(gh) * np.exp(y) * (y + off_h) + 4 * U * (np.abs(gl) + np.abs(gh) * (np.abs(lp) + H)))
    off += 2.0 ** -126 / T * np.abs(inner) + 2 * U / T * hit * np.abs(gl)
    off += half * (np.abs(ref) + off) + 2.0 ** -126
    assert (np.abs(g - ref) <= off).all(), (np.abs(g - ref) - off).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_rows_with_an_offset(gpu_lib, dtype):
    """A common offset, or a low temperature, takes digits from p: the logsumexp is handed over in fp32."""
    rng = np.random.default_rng(51)
    for bits in (0, 10, 13, 16):
        for V, T in ((777, 1.0), (5003, 0.7), (5003, 3.0)):
            z = _logits(60 + bits, 8, V, "f32") + torch.tensor([1.0, -1.0]).repeat(4)[:, None] * (2.0 ** bits if bits else 0.0)
            _check_gradient(gpu_lib, z.to(DT[dtype]), rng.integers(0, V, 8), T, bits)
    for T in (0.1, 0.01):
        _check_gradient(gpu_lib, _logits(61, 8, 5003, dtype), rng.integers(0, 5003, 8), T, 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_at_temperatures_far_from_one(gpu_lib, dtype):
    """Far below one a float32 logsumexp says no more than which entry is the largest, if that: the formula holds with the one given."""
    for T in (1e-3, 1e-6, 1e-12, 1e-30, 1e-35, 50.0, 1e6):
        z, tok = _logits(62, 6, 5003, dtype), _tokens(62, 6, 5003)
        tok[0] = int(z[0].float().argmax())
        _check_gradient(gpu_lib, z, tok, T, 8, exact=T >= 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_of_requests_cut_from_a_padded_vocabulary(gpu_lib, dtype):
    """[B, Nq, V] out of [B, Nq, Vpad], forward and gradient: what the rows side by side give, and nothing in the padding."""
    av = gpu_lib
    B, Nq, V, Vpad = 3, 5, 3001, 3008
    code = av.AURORA_F32 if dtype == "f32" else av.AURORA_BF16
    wide = torch.full((B, Nq, Vpad), 100.0, dtype=DT[dtype], device="cuda")
    cut = wide[..., :V]
    cut.copy_(_logits(63, B * Nq, V, dtype).view(B, Nq, V))
    tok = torch.from_numpy(np.random.default_rng(63).integers(0, V, (B, Nq)).astype(np.int32)).cuda()
    got = []
    for z, stride in ((cut, Vpad), (cut.contiguous(), 0)):
        d = av.aurora_logprob_desc(rows=B * Nq, vocab=V, dtype=code, n_top=3, row_stride=stride)
        ws = torch.empty(av.aurora_token_logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        lp, H, lse = (torch.zeros(B, Nq, device="cuda") for _ in range(3))
        ti, tl = torch.zeros((B, Nq, 3), dtype=torch.int32, device="cuda"), torch.zeros((B, Nq, 3), device="cuda")
        g = torch.full_like(wide, 9.0)[..., :V] if stride else torch.zeros_like(z)
        av.aurora_token_logprobs(d, z, tok, lp, H, lse, ti, tl, ws)
        av.aurora_token_logprobs_backward(d, z, tok, H, lse, lp, H, g)
        torch.cuda.synchronize()
        if stride:
            assert bool((g._base[..., V:] == 9.0).all()) and bool((wide[..., V:] == 100.0).all())
        got.append((lp, H, lse, ti, tl, g))
    assert torch.equal(got[0][3], got[1][3])
    # Rows that start elsewhere within 16 bytes are summed in another order.  |x| below 13, distances below 25: by the bounds above each
    # result is off by less than 2u 13 + u (2 25 + 16) + u 13 = 105 u, the entropy (below 8.1) by less than ten times that, p by 118 u.  No
    # p above 0.6: the gradient is off by 105 u + 25 p 118 u, by 8.1 p (10 118 + 1050 + 118) u and by 1050 p 10 u, 20 000 u together, and
    # by half a step of its type
    for a, b in zip(got[0][:3] + got[0][4:5], got[1][:3] + got[1][4:5]):
        assert (a - b).abs().max() <= 2 * 1050 * U
    assert got[0][4].max() < np.log(0.6)
    a, b = (x[5].double() for x in got)
    assert ((a - b).abs() <= 2 * 20000 * U + 2 * (2.0 ** -8 if dtype == "bf16" else U) * torch.maximum(a.abs(), b.abs())).all()
