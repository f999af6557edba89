"""Host checks of the calls around the verification step: descriptors, pointers, alignments and workspaces are looked at before any device
is touched (no address below is ever read)."""
import pytest
import torch

import paper_2602_06932_amd as av

P = 4096
BAD, NOT, WS = av.AURORA_ERR_INVALID_ARG, av.AURORA_ERR_UNSUPPORTED, av.AURORA_ERR_WORKSPACE


def _ws(n, short=0):
    t = torch.empty(n + 256, dtype=torch.uint8)
    return t[(-t.data_ptr()) % 256:][:n - short]


def _desc(kind, base, **kw):
    return kind(**{**base, **kw})


PLAN = dict(batch=3, page_size=16, max_pages_per_seq=8, num_pages=50, max_rows=20)
PLAN_ARGS = dict(held=P, want=P, table=P, free=P, count=P, count_out=P, lens=P, start=P, positions=P, slots=P, info=P)


def _plan(desc={}, ws=None, **kw):
    d = _desc(av.aurora_cache_plan_desc, PLAN, **desc)
    return av.aurora_cache_plan(d, *{**PLAN_ARGS, **kw}.values(), ws if ws is not None else _ws(65536), stream=0, check=False)


@pytest.mark.parametrize("desc,want", [(dict(batch=-1), BAD), (dict(page_size=0), BAD), (dict(max_pages_per_seq=0), BAD), (dict(num_pages=0), BAD),
                                       (dict(max_rows=-1), BAD), (dict(num_pages=2 ** 27), NOT), (dict(max_pages_per_seq=2 ** 27), NOT),
                                       (dict(batch=2 ** 20, max_pages_per_seq=2 ** 12), NOT)])
def test_plan_descriptors(desc, want):
    assert _plan(desc) == want
    with pytest.raises(av.AuroraError):
        av.aurora_cache_plan_workspace_bytes(_desc(av.aurora_cache_plan_desc, PLAN, **desc))


def test_plan_arguments():
    for name in ("want", "table", "free", "count", "count_out", "lens", "positions", "slots"):
        assert _plan(**{name: None}) == BAD, name
    for name in PLAN_ARGS:
        assert _plan(**{name: P + 2}) == BAD, name
    n = av.aurora_cache_plan_workspace_bytes(_desc(av.aurora_cache_plan_desc, PLAN))
    assert _plan(ws=_ws(n, short=1)) == WS and _plan(ws=_ws(n + 8)[8:]) == WS
    assert av.load().aurora_cache_plan(None, *([None] * 12), 0, None) == BAD


ROPE = dict(rows=4, num_q_heads=8, num_kv_heads=2, head_dim=64, rotary_dim=64, page_size=16, num_pages=9, dtype=av.AURORA_BF16)
ROPE_ARGS = dict(q=P, k=P, v=P, positions=P, slots=P, frequencies=P, q_out=P, kp=P, vp=P)


def _rope(desc={}, back=False, **kw):
    d = _desc(av.aurora_rope_desc, ROPE, **desc)
    a = {**ROPE_ARGS, **kw}
    if back:
        return av.aurora_rope_append_backward(d, a["q_out"], a["kp"], a["vp"], a["positions"], a["slots"], a["frequencies"], a["q"], a["k"], a["v"],
                                              stream=0, check=False)
    return av.aurora_rope_append(d, *a.values(), stream=0, check=False)


@pytest.mark.parametrize("desc,want", [(dict(rows=-1), BAD), (dict(num_q_heads=-1), BAD), (dict(num_q_heads=0, num_kv_heads=0), BAD), (dict(head_dim=0), BAD),
                                       (dict(rotary_dim=66), BAD), (dict(rotary_dim=63), BAD), (dict(rotary_dim=-2), BAD), (dict(interleaved=2), BAD),
                                       (dict(page_size=0), BAD), (dict(num_pages=0), BAD), (dict(dtype=av.AURORA_FP8_E4M3), BAD), (dict(dtype=7), BAD),
                                       (dict(kv_fp8=1), BAD), (dict(kv_fp8=2), BAD), (dict(magnitude=-1.0), BAD), (dict(magnitude=float("nan")), BAD),
                                       (dict(magnitude=float("inf")), BAD), (dict(q_stride=511), BAD), (dict(q_out_stride=511), BAD), (dict(k_stride=127), BAD),
                                       (dict(v_stride=-128), BAD), (dict(head_dim=512), NOT), (dict(rows=2 ** 22 + 1), NOT), (dict(num_pages=2 ** 28), NOT)])
def test_rope_descriptors(desc, want):
    assert _rope(desc) == want and _rope(desc, back=True) == want


def test_rope_arguments():
    for back in (False, True):
        for name in ROPE_ARGS:
            assert _rope(back=back, **{name: None}) == BAD, name
        for name in ROPE_ARGS:
            assert _rope(back=back, **{name: P + 1}) == BAD, name
        assert _rope(back=back, frequencies=P + 4) == BAD
        assert _rope(dict(rows=0), back=back, q=None) == av.AURORA_OK
    assert _rope(dict(dtype=av.AURORA_F32), q=P + 2) == BAD and _rope(back=True, kp=P + 2) == BAD
    assert _rope(dict(kv_fp8=1, k_scale=P, v_scale=P), back=True) == NOT


def test_rows_that_do_not_lie_as_the_descriptor_says():
    x = torch.zeros(4, 700)
    d = _desc(av.aurora_rope_desc, ROPE, q_stride=700)
    with pytest.raises(ValueError):
        av.aurora_rope_append(_desc(av.aurora_rope_desc, ROPE), x[:, :512], P, P, P, P, P, P, P, P, stream=0, check=False)
    with pytest.raises(ValueError):
        av.aurora_rope_append(d, torch.zeros(4, 512), P, P, P, P, P, P, P, P, stream=0, check=False)
    with pytest.raises(ValueError):
        av.aurora_rope_append(d, x[:, 0:512:2], P, P, P, P, P, P, P, P, stream=0, check=False)


def test_rows_that_are_one_row_expanded():
    """Rows 0 elements apart have the storage of one: the calls would go through as many."""
    one = torch.zeros(1, 8, 64, dtype=torch.bfloat16).expand(160, 8, 64)
    d = _desc(av.aurora_rope_desc, ROPE, rows=160)
    small = one[:, :2]
    for name, t in (("q", one), ("k", small), ("v", small), ("q_out", one)):
        a = {**ROPE_ARGS, name: t}
        with pytest.raises(ValueError):
            av.aurora_rope_append(d, *a.values(), stream=0, check=False)
        with pytest.raises(ValueError):
            av.aurora_rope_append_backward(d, a["q_out"], a["kp"], a["vp"], a["positions"], a["slots"], a["frequencies"], a["q"], a["k"], a["v"],
                                           stream=0, check=False)
    z = torch.zeros(1, 5, 1000).expand(4, 5, 1000)
    with pytest.raises(ValueError):
        _lp(dict(rows=20), logits=z)
    for name in ("logits", "dlogits"):
        with pytest.raises(ValueError):
            _lpb(dict(rows=20), **{name: z})
    for stride in (0, 700):  # a dimension of one is no such tensor, whatever its stride says
        assert _rope(dict(rows=0, q_stride=stride), q=one[:1]) == av.AURORA_OK


LP = dict(rows=4, vocab=1000, dtype=av.AURORA_F32, n_top=3)


def _lp(desc={}, ws=None, **kw):
    d = _desc(av.aurora_logprob_desc, LP, **desc)
    a = {**dict(logits=P, tokens=P, logprob=P, entropy=P, lse=P, ids=P, tops=P), **kw}
    return av.aurora_token_logprobs(d, *a.values(), ws if ws is not None else _ws(1 << 20), stream=0, check=False)


def _lpb(desc={}, **kw):
    d = _desc(av.aurora_logprob_desc, LP, **desc)
    a = {**dict(logits=P, tokens=P, entropy=P, lse=P, dlogprob=P, dentropy=P, dlogits=P), **kw}
    return av.aurora_token_logprobs_backward(d, *a.values(), stream=0, check=False)


@pytest.mark.parametrize("desc,want", [(dict(rows=-1), BAD), (dict(vocab=0), BAD), (dict(dtype=2), BAD), (dict(n_top=-1), BAD), (dict(row_stride=999), BAD),
                                       (dict(row_stride=-1), BAD), (dict(temperature_rows=-1), BAD), (dict(temperature=-0.5), BAD), (dict(temperature=float("nan")), BAD),
                                       (dict(temperature=float("inf")), BAD), (dict(n_top=33), NOT), (dict(vocab=2 ** 24 + 1), NOT)])
def test_logprob_descriptors(desc, want):
    assert _lp(desc) == want and _lpb(desc) == want
    with pytest.raises(av.AuroraError):
        av.aurora_token_logprobs_workspace_bytes(_desc(av.aurora_logprob_desc, LP, **desc))


def test_a_logprob_workspace_is_enough_for_fewer_rows():
    for dtype in (av.AURORA_F32, av.AURORA_BF16):
        for vocab in (777, 32000, 200064, 1 << 24):
            n = [av.aurora_token_logprobs_workspace_bytes(_desc(av.aurora_logprob_desc, LP, rows=r, vocab=vocab, dtype=dtype, n_top=32))
                 for r in (0, 1, 5, 7, 8, 9, 16, 17, 31, 63, 64, 65, 100, 119, 120, 121, 200, 201, 320, 321, 639, 640, 641, 1000, 1024, 5000, 100000)]
            assert n == sorted(n) and all(x % 256 == 0 and x for x in n)


def test_logprob_arguments():
    assert _lp(logits=None) == BAD and _lp(tokens=None) == BAD and _lp(logprob=None) == BAD and _lp(ids=None) == BAD and _lp(tops=None) == BAD
    assert _lp(dict(n_top=0), tokens=None, logprob=None, entropy=None, lse=None) == BAD     # nothing requested
    for name in ("logits", "tokens", "logprob", "entropy", "lse", "ids", "tops"):
        assert _lp(**{name: P + 2}) == BAD, name
    assert _lp(dict(dtype=av.AURORA_BF16), logits=P + 1) == BAD and _lp(dict(temperatures=P + 2)) == BAD
    n = av.aurora_token_logprobs_workspace_bytes(_desc(av.aurora_logprob_desc, LP, vocab=100000))
    assert _lp(dict(vocab=100000), ws=_ws(n, short=1)) == WS
    assert _lp(dict(rows=0), logits=None) == av.AURORA_OK
    assert _lpb(logits=None) == BAD and _lpb(lse=None) == BAD and _lpb(dlogits=None) == BAD and _lpb(dlogprob=None, dentropy=None) == BAD
    assert _lpb(tokens=None) == BAD and _lpb(entropy=None) == BAD
    for name in ("logits", "tokens", "entropy", "lse", "dlogprob", "dentropy", "dlogits"):
        assert _lpb(**{name: P + 2}) == BAD, name


def _device_verify(B=4, Nq=5, vocab=1000):
    """A DeviceVerify with what logprobs() looks at before anything is enqueued, and without a device."""
    from types import SimpleNamespace

    from paper_2602_06932_amd.device import DeviceVerify
    dv = object.__new__(DeviceVerify)
    dv.w = SimpleNamespace(batch=B, num_q=Nq, vocab=vocab, temperature=1.0)
    dv.temperatures = None
    return dv


def test_tokens_that_are_not_one_a_row():
    """The step's next_token has one entry a request, not one a row: the call would read past it."""
    on = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device="meta")
    for tokens, why in ((on(4), "4 entries"), (on(4, 1), "4 entries"), (on(4, 4), "16 entries"), (on(4, 6), "24 entries"), (on(0), "0 entries"),
                        (on(4, 5, dtype=torch.int64), "int64"), (on(20, dtype=torch.float32), "float32"),
                        (torch.zeros(4, 5, dtype=torch.int32), "device")):
        with pytest.raises(ValueError, match="tokens: .*" + why):
            _device_verify().logprobs(tokens)


def test_a_change_of_the_alternatives_leaves_the_buffers_of_other_calls(monkeypatch):
    """A captured call goes on writing to the buffers that it was captured with: they are there again, and not given to others in between."""
    empty, calls = torch.empty, []
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k))
    monkeypatch.setattr(av.binding, "aurora_verify_logits_ptr", lambda attn, accept, workspace: P if attn is None else 2 * P)
    monkeypatch.setattr(av.binding, "aurora_token_logprobs", lambda *a: calls.append(a))
    dv = _device_verify(B=1, vocab=128256)
    dv.attn_desc = dv.accept_desc = dv.workspace = 0
    for n_top, after in ((5, "verify"), (0, "verify"), (5, "accept"), (5, "verify"), (0, "verify"), (5, "accept")):
        dv.logprobs(P, n_top, after)
        mine = (dv.logprob_desc, 2 * P if after == "verify" else P, P, dv.logprob, dv.entropy, dv.lse, dv.top_ids, dv.top_logprobs)
        assert all(x is y or x == y for x, y in zip(calls[-1], mine)) and (dv.top_ids is None) == (n_top == 0)  # (the last call's are the results)
    buffers = [[x for x in c if isinstance(x, torch.Tensor)] for c in calls]
    for a, b in zip(buffers[:3], buffers[3:]):
        assert len(a) == len(b) and all(x is y for x, y in zip(a, b))
    first = [x for b in buffers[:3] for x in b]
    assert len({x.data_ptr() for x in first}) == len(first)


def test_rows_over_several_dimensions():
    """Rows that all lie as far apart as the descriptor says are taken in any shape; those that do not are not.  (No rows: the addresses
    are looked at and nothing is enqueued.)"""
    wide = torch.zeros(4, 5, 1024)
    cut, flat = wide[..., :1000], wide.view(20, 1024)[:, :1000]
    for z in (cut, flat, wide.view(2, 2, 5, 1024)[..., :1000], wide, cut[:1], cut[:, :, :1000]):
        assert _lp(dict(rows=0, row_stride=1024), logits=z) == av.AURORA_OK
        assert _lpb(dict(rows=0, row_stride=1024), logits=z, dlogits=z) == av.AURORA_OK
    for z, why in ((cut[:, :4], "requests of five rows, four of them"), (cut[::2], "every other request"), (cut.transpose(0, 1), "another order"),
                   (wide[..., ::2], "every other logit"), (wide[..., 0:1000:2], "every other logit"), (cut.unsqueeze(-1).expand(4, 5, 1000, 2), "twice each"),
                   (torch.zeros(4, 2, 1024)[..., :512], "rows shorter than the vocabulary")):
        with pytest.raises(ValueError):
            _lp(dict(rows=0, row_stride=1024), logits=z)
        with pytest.raises(ValueError):
            _lpb(dict(rows=0, row_stride=1024), logits=z)
    with pytest.raises(ValueError):
        _lp(dict(rows=0), logits=cut)                       # the descriptor says: side by side
    qkv = torch.zeros(3, 5, 12 * 64, dtype=torch.bfloat16)  # a projection's output for requests of five tokens
    q, k, v = (x.unflatten(-1, (-1, 64)) for x in qkv.split([512, 128, 128], -1))
    d = dict(rows=0, q_stride=768, k_stride=768, v_stride=768)
    for back in (False, True):
        assert _rope(d, back=back, q=q, k=k, v=v) == av.AURORA_OK
        assert _rope(d, back=back, q=q.flatten(0, 1), k=k.flatten(0, 1), v=v.flatten(0, 1)) == av.AURORA_OK
        for bad in (q[:, :4], q[:, :, ::2], q[..., ::2], q.transpose(1, 2)):
            with pytest.raises(ValueError):
                _rope(d, back=back, q=bad, k=k, v=v)
        with pytest.raises(ValueError):                     # heads as far apart as rows should be
            _rope(d, back=back, q=torch.zeros(3, 8, 768, dtype=torch.bfloat16)[..., :64], k=k, v=v)


def test_rope_rows_too_wide_for_so_many():
    """A launch has less than 2^32 threads: past that a block takes more rows, and their angles have to fit into its LDS."""
    for back in (False, True):
        for rotary in (2, 64, 256):
            assert _rope(dict(rows=2 ** 22, num_q_heads=65535, num_kv_heads=65535, head_dim=256, rotary_dim=rotary), back=back) == NOT
        assert _rope(dict(rows=2 ** 22, num_q_heads=65535, num_kv_heads=1, head_dim=256, rotary_dim=256), back=back) == NOT
