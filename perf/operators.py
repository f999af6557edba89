"""The operators on either side of the verification step whose speed is measured: block tables and slot maps from request lengths,
rotary positions on the way into the paged KV cache and back, log probabilities of given tokens with entropy and alternatives.

With `own` false run() computes them from elementary torch operations, with `own` true by the framework's calls; both take what
prepare() gives.  Sizes are those of the benchmark's workloads (32 query heads over 8 KV heads of 128, vocabularies of 128 256;
the stress shape 48/8/128 with 200 064; a 32K-entry draft vocabulary) and odd and ragged ones around them.  Every input is made
from the seed alone.
"""
import math
import random

import torch

own = False
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
TYPES = {"f32": F32, "bf16": BF16}


# ---------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------
def _pages(batch, lo, hi, chunk=5, page=16, grow=100, shrink=0, finish=0, start=0, short=False, seq_rows=0):
    """Of the requests `grow` percent take `chunk` tokens more, `shrink` percent give up to chunk - 1 back, `finish` percent end and
    `start` percent begin; the rest stay as they are.  short: the free pages do not last."""
    return {"kind": "pages", "batch": batch, "len_lo": lo, "len_hi": hi, "chunk": chunk, "page": page, "grow": grow, "shrink": shrink,
            "finish": finish, "start": start, "short": short, "spare_rows": seq_rows}


def _rope(kind, rows, hq=32, hkv=8, d=128, rotary=128, interleaved=False, dtype="bf16", kv8=False, fused=True, page=16, chunk=5,
          padded=0, far=32768, factor=1.0):
    """`rows` tokens in runs of `chunk` consecutive positions up to `far`, `padded` of them behind the last sequence."""
    return {"kind": kind, "rows": rows, "hq": hq, "hkv": hkv, "d": d, "rotary": rotary, "interleaved": interleaved, "dtype": dtype,
            "kv8": kv8, "fused": fused, "page": page, "chunk": chunk, "padded": padded, "far": far, "factor": factor}


def _logprobs(kind, rows, vocab, dtype="f32", n_top=0, temperature=1.0):
    return {"kind": kind, "rows": rows, "vocab": vocab, "dtype": dtype, "n_top": n_top, "temperature": temperature}


def listed():
    return [
        # before every verification step of a server: 32 requests take five tokens each
        {"name": "pages_decode_b32", **_pages(32, 1024, 4096)},
        # a full server between two steps: requests grow, give rejected tokens back, end, and new prompts come in
        {"name": "pages_mixed_b256", **_pages(256, 256, 8192, grow=45, shrink=30, finish=10, start=10, seq_rows=512)},
        # the largest plan: a batch of long prompts, a million token rows
        {"name": "pages_prefill_1m", **_pages(64, 2048, 30000, grow=0, start=100)},
        # one layer of a verification step: 32 requests of five positions
        {"name": "rope_decode_b32", **_rope("rope", 160)},
        # one layer of a prefill of long prompts
        {"name": "rope_prefill_16k", **_rope("rope", 16384, chunk=2048)},
        # a prefill into an 8-bit cache: half of each head rotated, neighbouring pairs, long-context frequencies, a padded batch
        {"name": "rope_prefill_8k_kv8", **_rope("rope", 8192, hq=48, rotary=64, interleaved=True, kv8=True, chunk=777, padded=100,
                                                far=262144, factor=8.0)},
        # the training side: from the attention's gradients to those of the projections
        {"name": "rope_backward_8k", **_rope("rope_backward", 8192, chunk=512)},
        # one user: what is returned with the tokens of one step
        {"name": "logprobs_one_request", **_logprobs("logprobs", 5, 128256, n_top=5)},
        # the same of a served batch, with twenty alternatives at a temperature
        {"name": "logprobs_b32", **_logprobs("logprobs", 160, 128256, n_top=20, temperature=0.7)},
        # the stress batch, from 16-bit logits
        {"name": "logprobs_b256_bf16", **_logprobs("logprobs", 1280, 200064, dtype="bf16", n_top=8)},
        # the training side: the drafter's log probabilities and entropies of a batch of trace rows, and the gradient
        {"name": "logprobs_train_4096", **_logprobs("logprobs_train", 4096, 32000)},
        # the gradient alone, of 16-bit logits over the whole vocabulary
        {"name": "logprobs_backward_1k_bf16", **_logprobs("logprobs_backward", 1024, 128256, dtype="bf16")},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pages", "pages", "rope", "rope", "rope_backward", "logprobs", "logprobs", "logprobs_train", "logprobs_backward"])
    if kind == "pages":
        batch = _log_int(rng, 1, 700)
        hi = min(_log_int(rng, 40, 30000), max(40, 900000 // batch))
        grow, shrink, finish, start = rng.choice([(100, 0, 0, 0), (50, 30, 5, 5), (0, 0, 0, 100), (30, 40, 20, 5), (60, 0, 0, 30)])
        return _pages(batch, max(12, hi // rng.randint(1, 20)), hi, chunk=rng.randint(1, 40), page=rng.choice([16, 16, 32, 64, 24, 1]),
                      grow=grow, shrink=shrink, finish=finish, start=start, short=rng.random() < 0.25, seq_rows=rng.choice([0, 100, 513]))
    if kind in ("rope", "rope_backward"):
        hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (48, 8, 128), (28, 4, 128), (8, 2, 64), (16, 16, 64), (9, 3, 80)])
        rows = _log_int(rng, 1, 9000)
        return _rope(kind, rows, hq, hkv, d, rotary=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.4,
                     dtype=rng.choice(["bf16", "bf16", "f32"]), kv8=kind == "rope" and rng.random() < 0.3, fused=rng.random() < 0.6,
                     page=rng.choice([16, 16, 64, 24]), chunk=_log_int(rng, 1, 3000), padded=rng.choice([0, 0, rows // 7]),
                     far=rng.choice([4096, 32768, 1000000]), factor=rng.choice([1.0, 1.0, 4.0, 8.0]))
    vocab = rng.choice([128256, 151936, 200064, 32000, 32003, 16001, 4096, 777, 128257])
    dtype = rng.choice(["f32", "f32", "bf16"])
    rows = _log_int(rng, 1, max(2, min(6000, 250_000_000 // vocab // (2 if kind != "logprobs" else 1))))
    return _logprobs(kind, rows, vocab, dtype, n_top=rng.choice([0, 1, 5, 20, 32]) if kind == "logprobs" else 0,
                     temperature=rng.choice([1.0, 1.0, 0.7, 1.3]))


# ---------------------------------------------------------------------------------------------------------------
# inputs, from the seed alone
# ---------------------------------------------------------------------------------------------------------------
def _dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def _normal(shape, dtype, g, std=1.0):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat, step = out.view(-1), 1 << 26
    for o in range(0, flat.numel(), step):
        n = min(step, flat.numel() - o)
        flat[o:o + n] = torch.randn(n, device=DEV, generator=g) * std
    return out


def _lengths(c, rnd):
    """(held, wanted) of every request.  The kinds of requests and their lengths do not depend on the seed, their order does."""
    n, lo, hi = c["batch"], c["len_lo"], c["len_hi"]
    kinds = []
    for name in ("grow", "shrink", "finish", "start"):
        kinds += [name] * round(n * c[name] / 100)
    kinds = (kinds + ["stay"] * n)[:n]
    got = []
    for i, k in enumerate(kinds):
        x = lo + (hi - lo) * ((i * 37) % n) // max(1, n - 1)
        held = 0 if k == "start" else x
        want = {"grow": x + c["chunk"], "shrink": x - 1 - i % max(1, min(c["chunk"] - 1, lo - 2)), "finish": 0, "start": x, "stay": x}[k]
        got.append((held, max(0, want)))
    rnd.shuffle(got)
    return [g[0] for g in got], [g[1] for g in got]


def _page_inputs(c, rnd, g):
    held, want = _lengths(c, rnd)
    per = lambda x: -(-x // c["page"])
    held_pages = [per(x) for x in held]
    need = sum(max(0, per(w) - per(h)) for h, w in zip(held, want))
    back = sum(max(0, per(h) - per(w)) for h, w in zip(held, want))
    n_free = max(0, need - back) + need // 10 + 3
    if c["short"]:
        n_free = max(0, (need * 3) // 4 - back)
    pool, width = sum(held_pages) + n_free + 5, max(max(per(h), per(w)) for h, w in zip(held, want)) + 1
    ids = torch.randperm(pool, device=DEV, generator=g).to(torch.int32)
    cols = torch.arange(width, device=DEV)[None]
    n_held = _dev(held_pages, torch.int64)[:, None]
    at = (n_held.cumsum(0) - n_held + cols).clamp(max=pool - 1)
    table = torch.where(cols < n_held, ids[at], -1).contiguous()
    free = torch.full((pool,), -1, dtype=torch.int32, device=DEV)
    free[:n_free] = ids[sum(held_pages):sum(held_pages) + n_free]
    rows = sum(max(0, w - h) for h, w in zip(held, want)) + c["spare_rows"]
    return {"held": _dev(held), "want": _dev(want), "table": table, "free": free, "count": _dev([n_free]), "max_rows": rows, "pool": pool}


def _frequencies(c):
    """Radians per position of every pair; past the factor 1 the slow ones are stretched, with a smooth passage between."""
    i = torch.arange(c["rotary"] // 2, dtype=torch.float64)
    f = 500000.0 ** (-2.0 * i / c["rotary"])
    if c["factor"] != 1.0:
        turns = 8192 * f / (2 * math.pi)  # of the context the model was trained on
        keep = ((turns - 1.0) / 3.0).clamp(0, 1)
        f = keep * f + (1 - keep) * f / c["factor"]
    return f.to(DEV)


def _rope_inputs(c, rnd, g):
    T, hq, hkv, d, page = c["rows"], c["hq"], c["hkv"], c["d"], c["page"]
    live = T - c["padded"]
    dt = TYPES[c["dtype"]]
    n_runs = -(-live // c["chunk"])
    per = -(-c["chunk"] // page) + 1
    pool = n_runs * per + n_runs * per // 8 + 1
    pages = torch.randperm(pool, device=DEV, generator=g)[:n_runs * per].view(n_runs, per)
    first = _dev([rnd.randrange(0, max(1, c["far"] - c["chunk"])) for _ in range(n_runs)], torch.int64)
    t = torch.arange(live, device=DEV)
    run_of, pos = t // c["chunk"], first[t // c["chunk"]] + t % c["chunk"]
    slot = pages[run_of, pos // page - first[run_of] // page] * page + pos % page
    pad = torch.zeros(c["padded"], dtype=torch.int64, device=DEV)
    s = {"positions": torch.cat([pos, pad]).to(torch.int32), "slots": torch.cat([slot, pad - 1]).to(torch.int32), "pool": pool,
         "frequencies": _frequencies(c), "k_scale": None, "v_scale": None, "magnitude": 1.0 if c["factor"] == 1.0 else 0.1 * math.log(c["factor"]) + 1.0}
    if c["kind"] == "rope_backward":
        s["dq_out"] = _normal((T, hq, d), F32, g)
        s["dk_pages"], s["dv_pages"] = (_normal((pool, hkv, page, d), F32, g) for _ in range(2))
        s["dq"], s["dk"], s["dv"] = (torch.zeros((T, h, d), dtype=dt, device=DEV) for h in (hq, hkv, hkv))
        return s
    if c["fused"]:  # one projection's output: a row holds the queries, the keys and the values
        qkv = _normal((T, (hq + 2 * hkv) * d), dt, g)
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
    else:
        s["q"], s["k"], s["v"] = (_normal((T, h, d), dt, g) for h in (hq, hkv, hkv))
    s["q_out"] = torch.zeros((T, hq, d), dtype=dt, device=DEV)
    if c["kv8"]:
        s["k_scale"] = (1 + torch.arange(hkv, device=DEV) % 3).float() * 0.009
        s["v_scale"] = (3 - torch.arange(hkv, device=DEV) % 3).float() * 0.008
        s["k_pages"], s["v_pages"] = (torch.randint(0, 120, (pool, hkv, page, d), device=DEV, generator=g, dtype=torch.uint8) for _ in range(2))
    else:
        s["k_pages"], s["v_pages"] = (_normal((pool, hkv, page, d), dt, g) for _ in range(2))
    return s


def _logprob_inputs(c, g):
    """Logits as a trained head gives them: a broad floor, the token in question raised in most rows, a tail of ids that no
    tokenizer has at minus infinity, and rows without a token among the training rows."""
    M, V = c["rows"], c["vocab"]
    z = _normal((M, V), TYPES[c["dtype"]], g, 2.5)
    tokens = torch.randint(0, V - V // 200, (M,), device=DEV, generator=g)
    raised = torch.rand(M, device=DEV, generator=g) < 0.7
    z[torch.arange(M, device=DEV), tokens] += (raised * (6 + 8 * torch.rand(M, device=DEV, generator=g))).to(z.dtype)
    z[:, V - V // 200:] = -math.inf
    if M > 64:
        tokens = torch.where(torch.rand(M, device=DEV, generator=g) < 0.05, -1, tokens)
    s = {"logits": z, "tokens": tokens.to(torch.int32)}
    if c["kind"] != "logprobs":
        s.update(dlogprob=torch.randn(M, device=DEV, generator=g) / M, dentropy=torch.randn(M, device=DEV, generator=g) * 0.01 / M)
    if c["kind"] == "logprobs_backward":
        lse, ent = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
        for o in range(0, M, 256):
            lp = torch.log_softmax(z[o:o + 256].double() / c["temperature"], -1)
            lse[o:o + 256] = torch.logsumexp(z[o:o + 256].double() / c["temperature"], -1)
            ent[o:o + 256] = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(1)
        s.update(lse=lse, entropy=ent)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = random.Random(seed)
    make = {"pages": lambda: _page_inputs(case, rnd, g), "rope": lambda: _rope_inputs(case, rnd, g),
            "rope_backward": lambda: _rope_inputs(case, rnd, g)}
    return {**make.get(case["kind"], lambda: _logprob_inputs(case, g))(), "case": case}


# ---------------------------------------------------------------------------------------------------------------
# one pass, by elementary operations
# ---------------------------------------------------------------------------------------------------------------
def _plain_pages(c, s):
    page, width = c["page"], s["table"].shape[1]
    held, want, n = s["held"].long(), s["want"].long(), s["count"].long()[0]
    hp, wp = (held + page - 1) // page, (want + page - 1) // page
    valid = (held >= 0) & (want >= 0) & (hp <= width) & (wp <= width)
    grow, shrink = valid & (want > held), valid & (want < held)
    back = torch.where(shrink, hp - wp, 0)
    freed = back.sum()
    need, rows = torch.where(grow, wp - hp, 0), torch.where(grow, want - held, 0)
    ok = grow & (need.cumsum(0) <= n + freed) & (rows.cumsum(0) <= s["max_rows"])
    need, rows = torch.where(ok, need, 0), torch.where(ok, rows, 0)
    new = torch.where(ok | shrink, want, held)
    taken, total = need.sum(), rows.sum()
    at = torch.arange(len(held), device=DEV)
    # the pages given back, in order, on top of the free ones
    b = at.repeat_interleave(back)
    back_start, need_start, row_start = back.cumsum(0) - back, need.cumsum(0) - need, rows.cumsum(0) - rows
    given = s["table"][b, wp[b] + torch.arange(len(b), device=DEV) - back_start[b]].clone()
    push = torch.arange(len(b), device=DEV)
    push = push[push < freed - taken]
    # the pages taken, from the top
    b = at.repeat_interleave(need)
    k = torch.arange(len(b), device=DEV)
    from_stack = s["free"][(n - 1 - (k - freed)).clamp(min=0)]
    got = torch.where(k < freed, given[(freed - 1 - k).clamp(min=0)] if len(given) else from_stack, from_stack)
    s["table"][b, hp[b] + k - need_start[b]] = got
    s["free"][n + push] = given[push]
    # the new tokens' positions and places
    b = at.repeat_interleave(rows)
    pos = held[b] + torch.arange(len(b), device=DEV) - row_start[b]
    slots = torch.full((s["max_rows"],), -1, dtype=torch.int32, device=DEV)
    positions = torch.zeros_like(slots)
    slots[:len(b)] = (s["table"][b, pos // page].long() * page + pos % page).to(torch.int32)
    positions[:len(b)] = pos.to(torch.int32)
    info = torch.stack([total, taken, freed, (~ok & (want != held) & ~shrink).sum()])
    start = torch.cat([row_start, total[None]])
    return {"table": s["table"], "free": s["free"], "count": (n + freed - taken).to(torch.int32)[None], "seq_lens": new.to(torch.int32),
            "row_start": start.to(torch.int32), "positions": positions, "slots": slots, "info": info.to(torch.int32)}


def _pair_index(c):
    """The elements of a head that are rotated: the first ones and the second ones of the pairs."""
    i = torch.arange(c["rotary"] // 2, device=DEV)
    return (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rotary"] // 2)


def _turn(c, s, x, sign):
    """x [rows, heads, d] in float32, every pair turned by its angle."""
    angle = s["positions"].double()[:, None] * s["frequencies"][None]
    cos, sin = (angle.cos() * s["magnitude"]).float()[:, None], (angle.sin() * (sign * s["magnitude"])).float()[:, None]
    first, second = _pair_index(c)
    x, y = x.float(), x.float().clone()
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def _plain_rope(c, s):
    live = s["slots"] >= 0
    slot = s["slots"].long()[live]
    page, off = slot // c["page"], slot % c["page"]
    s["q_out"][live] = _turn(c, s, s["q"], 1)[live].to(s["q_out"].dtype)
    k, v = _turn(c, s, s["k"], 1)[live], s["v"].float()[live]
    if c["kv8"]:
        k, v = (((x / s[n][None, :, None]).clamp(-448, 448)).to(torch.float8_e4m3fn).view(torch.uint8) for x, n in ((k, "k_scale"), (v, "v_scale")))
    s["k_pages"][page, :, off] = k.to(s["k_pages"].dtype)
    s["v_pages"][page, :, off] = v.to(s["v_pages"].dtype)


def _plain_rope_backward(c, s):
    dt = TYPES[c["dtype"]]
    live = s["slots"] >= 0
    slot = s["slots"].long().clamp(min=0)
    page, off = slot // c["page"], slot % c["page"]
    kept = live[:, None, None]
    return {"dq": torch.where(kept, _turn(c, s, s["dq_out"], -1), 0.0).to(dt),
            "dk": torch.where(kept, _turn(c, s, s["dk_pages"][page, :, off], -1), 0.0).to(dt),
            "dv": torch.where(kept, s["dv_pages"][page, :, off], 0.0).to(dt)}


def _plain_logprobs(c, s):
    V, n = c["vocab"], c["n_top"]
    z = s["logits"].float()
    x = z / c["temperature"]
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1)
    lse = m[:, 0] + total.log()
    known = s["tokens"] >= 0
    x_t = x.gather(1, s["tokens"].long().clamp(min=0)[:, None])[:, 0]
    got = {"logprob": torch.where(known, x_t - lse, 0.0), "lse": lse,
           "entropy": total.log() - torch.where(e > 0, e * (x - m), 0.0).sum(1) / total}
    if n:  # largest first, equal ones by their index: one whole number holds both
        bits = (z + 0.0).view(torch.int32)
        key = ((bits ^ ((bits >> 31) & 0x7fffffff)).long() << 32) + (V - 1 - torch.arange(V, device=DEV))
        ids = V - 1 - (key.topk(n, dim=1).values & 0xffffffff)
        got.update(top_ids=ids.to(torch.int32), top_logprobs=x.gather(1, ids) - lse[:, None])
    return got


def _plain_logprobs_backward(c, s):
    lp = s["logits"].float() / c["temperature"] - s["lse"][:, None]
    p = lp.exp()
    known = s["tokens"] >= 0
    gl = torch.where(known, s["dlogprob"], 0.0)[:, None]
    grad = -gl * p - s["dentropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    grad.scatter_add_(1, s["tokens"].long().clamp(min=0)[:, None], gl)
    return {"grad": (grad / c["temperature"]).to(s["logits"].dtype)}


def _plain_logprobs_train(c, s):
    got = _plain_logprobs(c, s)
    return {**got, **_plain_logprobs_backward(c, {**s, **got})}


# ---------------------------------------------------------------------------------------------------------------
# one pass, by the framework
# ---------------------------------------------------------------------------------------------------------------
def _keep(s):
    """What a program keeps from pass to pass: the descriptor, the workspace and the buffers of the results."""
    import paper_2602_06932_amd as av
    c = s["case"]
    code = {"f32": av.AURORA_F32, "bf16": av.AURORA_BF16}
    empty = lambda shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEV)
    i32 = torch.int32
    k = {"av": av}
    if c["kind"] == "pages":
        B = c["batch"]
        k["desc"] = av.aurora_cache_plan_desc(batch=B, page_size=c["page"], max_pages_per_seq=s["table"].shape[1], num_pages=s["pool"],
                                              max_rows=s["max_rows"])
        k["ws"] = empty(av.aurora_cache_plan_workspace_bytes(k["desc"]), torch.uint8)
        k.update(count=empty(1, i32), seq_lens=empty(B, i32), row_start=empty(B + 1, i32), positions=empty(s["max_rows"], i32),
                 slots=empty(s["max_rows"], i32), info=empty(4, i32))
    elif c["kind"] in ("rope", "rope_backward"):
        ptr = lambda t: None if t is None else t.data_ptr()
        stride = lambda n: s[n].stride(0) if n in s else 0
        k["desc"] = av.aurora_rope_desc(rows=c["rows"], num_q_heads=c["hq"], num_kv_heads=c["hkv"], head_dim=c["d"], rotary_dim=c["rotary"],
                                        interleaved=int(c["interleaved"]), page_size=c["page"], num_pages=s["pool"], dtype=code[c["dtype"]],
                                        kv_fp8=int(c["kv8"]), k_scale=ptr(s["k_scale"]), v_scale=ptr(s["v_scale"]), magnitude=s["magnitude"],
                                        q_stride=stride("q"), k_stride=stride("k"), v_stride=stride("v"))
    else:
        M, n = c["rows"], c["n_top"]
        k["desc"] = av.aurora_logprob_desc(rows=M, vocab=c["vocab"], dtype=code[c["dtype"]], n_top=n, temperature=c["temperature"])
        if c["kind"] != "logprobs_backward":
            k["ws"] = empty(av.aurora_token_logprobs_workspace_bytes(k["desc"]), torch.uint8)
            k.update(logprob=empty(M), entropy=empty(M), lse=empty(M))
            k.update(top_ids=empty((M, n), i32) if n else None, top_logprobs=empty((M, n)) if n else None)
        if c["kind"] != "logprobs":
            k["grad"] = torch.empty_like(s["logits"])
    return k


def _own(c, s):
    if "keep" not in s:
        s["keep"] = _keep(s)
    k = s["keep"]
    av = k["av"]
    if c["kind"] == "pages":
        av.aurora_cache_plan(k["desc"], s["held"], s["want"], s["table"], s["free"], s["count"], k["count"], k["seq_lens"], k["row_start"],
                             k["positions"], k["slots"], k["info"], k["ws"])
        return {"table": s["table"], "free": s["free"], **{n: k[n] for n in ("count", "seq_lens", "row_start", "positions", "slots", "info")}}
    if c["kind"] == "rope":
        av.aurora_rope_append(k["desc"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["frequencies"], s["q_out"], s["k_pages"],
                              s["v_pages"])
        return None
    if c["kind"] == "rope_backward":
        av.aurora_rope_append_backward(k["desc"], s["dq_out"], s["dk_pages"], s["dv_pages"], s["positions"], s["slots"], s["frequencies"],
                                       s["dq"], s["dk"], s["dv"])
        return {n: s[n] for n in ("dq", "dk", "dv")}
    got = {}
    if c["kind"] != "logprobs_backward":
        av.aurora_token_logprobs(k["desc"], s["logits"], s["tokens"], k["logprob"], k["entropy"], k["lse"], k["top_ids"], k["top_logprobs"],
                                 k["ws"])
        got = {n: k[n] for n in ("logprob", "entropy", "lse") + (("top_ids", "top_logprobs") if c["n_top"] else ())}
    if c["kind"] != "logprobs":
        saved = s if c["kind"] == "logprobs_backward" else k
        av.aurora_token_logprobs_backward(k["desc"], s["logits"], s["tokens"], saved["entropy"], saved["lse"], s["dlogprob"], s["dentropy"],
                                          k["grad"])
        got["grad"] = k["grad"]
    return got


def run(s):
    c = s["case"]
    if own:
        got = _own(c, s)
    else:
        plain = {"pages": _plain_pages, "rope": _plain_rope, "rope_backward": _plain_rope_backward, "logprobs": _plain_logprobs,
                 "logprobs_train": _plain_logprobs_train, "logprobs_backward": _plain_logprobs_backward}
        got = plain[c["kind"]](c, s)
    if c["kind"] == "rope":  # the caches are updated in place; codes are returned as the values that they stand for
        values = (lambda x: x.view(torch.float8_e4m3fn)) if c["kv8"] else (lambda x: x)
        got = {"q_out": s["q_out"], "k_pages": values(s["k_pages"]), "v_pages": values(s["v_pages"])}
    return got


# ---------------------------------------------------------------------------------------------------------------
# the work of one pass, and the results in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "pages":
        held, want = _lengths(c, random.Random(0))
        per = lambda x: -(-x // c["page"])
        rows = sum(max(0, w - h) for h, w in zip(held, want))
        moved = sum(abs(per(w) - per(h)) for h, w in zip(held, want))
        # lengths in and out, row starts, a position and a slot for every row, the pages taken and given back
        return {"bytes": 16 * c["batch"] + 8 * (rows + c["spare_rows"]) + 8 * moved + 24, "flops": 0}
    if c["kind"] in ("rope", "rope_backward"):
        e = 4 if c["dtype"] == "f32" else 2
        cache = 1 if c["kv8"] else e
        live, q, kv = c["rows"] - c["padded"], c["hq"] * c["d"], 2 * c["hkv"] * c["d"]
        each = q * 2 * e + kv * (e + cache) if c["kind"] == "rope" else (q + kv) * (4 + e)
        return {"bytes": live * each + 8 * c["rows"] + 4 * c["rotary"], "flops": 3 * live * (c["hq"] + c["hkv"]) * c["rotary"]}
    e = 4 if c["dtype"] == "f32" else 2
    n = c["rows"] * c["vocab"]
    if c["kind"] == "logprobs":
        return {"bytes": n * e + c["rows"] * (16 + 8 * c["n_top"]), "flops": 6 * n}
    train = c["kind"] == "logprobs_train"  # (the logits of both passes: once is enough to read them in principle)
    return {"bytes": 2 * n * e + (24 if train else 20) * c["rows"], "flops": (15 if train else 9) * n}


def _exact_pages(c, s):
    """The definition, request by request and page by page."""
    page, width = c["page"], s["table"].shape[1]
    held, want, n = s["held"].tolist(), s["want"].tolist(), s["count"].tolist()[0]
    table, free = s["table"].cpu(), s["free"].cpu()
    stack = free[:n].tolist()
    per = lambda x: -(-x // page)
    fits = [h >= 0 and w >= 0 and per(h) <= width and per(w) <= width for h, w in zip(held, want)]
    new, freed, refused, taken = list(held), 0, 0, 0
    for b, (h, w) in enumerate(zip(held, want)):
        if fits[b] and w < h:
            stack += table[b, per(w):per(h)].tolist()
            freed += per(h) - per(w)
            new[b] = w
    starts, pos, slots, full = [], [], [], False
    for b, (h, w) in enumerate(zip(held, want)):
        starts.append(len(pos))
        if w <= h and fits[b]:
            continue
        need = per(w) - per(h)
        if full or not fits[b] or need > len(stack) or len(pos) + w - h > s["max_rows"]:
            full = full or fits[b]
            refused += w != h
            continue
        if need:
            table[b, per(h):per(w)] = torch.tensor(stack[:-need - 1:-1], dtype=torch.int32)
            del stack[-need:]
        taken += need
        new[b] = w
        t = torch.arange(h, w)
        pos += t.tolist()
        slots += (table[b].long()[t // page] * page + t % page).tolist()
    free[n:max(n, len(stack))] = torch.tensor(stack[n:], dtype=torch.int32)
    pad = s["max_rows"] - len(pos)
    return {"table": table.to(DEV), "free": free.to(DEV), "count": _dev([len(stack)]), "seq_lens": _dev(new), "row_start": _dev(starts + [len(pos)]),
            "positions": _dev(pos + [0] * pad), "slots": _dev(slots + [-1] * pad), "info": _dev([len(pos), taken, freed, refused])}


def _exact_turn(c, s, x, sign):
    """Every pair as a complex number, multiplied by one on the circle."""
    x = x.double().clone()
    angle = s["positions"].double()[:, None] * s["frequencies"]
    unit = torch.polar(torch.full_like(angle, s["magnitude"]), sign * angle)[:, None]
    R = c["rotary"]
    part = x[..., :R].unflatten(-1, (R // 2, 2)) if c["interleaved"] else x[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(part.contiguous()) * unit)
    x[..., :R] = turned.flatten(-2) if c["interleaved"] else turned.transpose(-1, -2).flatten(-2)
    return x


def _exact_rope(c, s):
    live = (s["slots"] >= 0).nonzero()[:, 0]
    slot = s["slots"][live].long()
    if c["kind"] == "rope_backward":
        gather = lambda x: torch.zeros((c["rows"], c["hkv"], c["d"]), dtype=torch.float64, device=DEV).index_copy(
            0, live, x.double().transpose(1, 2).flatten(0, 1)[slot])
        dq = _exact_turn(c, s, s["dq_out"], -1)
        dq[s["slots"] < 0] = 0
        return {"dq": dq, "dk": _exact_turn(c, s, gather(s["dk_pages"]), -1), "dv": gather(s["dv_pages"])}
    got = {"q_out": s["q_out"].double()}
    got["q_out"][live] = _exact_turn(c, s, s["q"], 1)[live]
    for n, x in (("k", _exact_turn(c, s, s["k"], 1)), ("v", s["v"].double())):
        cache = s[n + "_pages"].view(torch.float8_e4m3fn).double() if c["kv8"] else s[n + "_pages"].double()
        if c["kv8"]:
            x = (x / s[n + "_scale"].double()[:, None]).clamp(-448, 448)
        flat = cache.transpose(1, 2).flatten(0, 1)
        flat[slot] = x[live]
        got[n + "_pages"] = flat.unflatten(0, (-1, c["page"])).transpose(1, 2).contiguous()
    return got


def _exact_logprobs(c, s):
    M, V, n = c["rows"], c["vocab"], c["n_top"]
    new = lambda *shape: torch.empty(shape, dtype=torch.float64, device=DEV)
    got = {}
    if c["kind"] != "logprobs_backward":
        got = {"logprob": new(M), "entropy": new(M), "lse": new(M)}
    if n:
        got.update(top_ids=torch.empty((M, n), dtype=torch.int32, device=DEV), top_logprobs=new(M, n))
    if c["kind"] != "logprobs":
        got["grad"] = new(M, V)
    for o in range(0, M, 64):
        e = slice(o, min(M, o + 64))
        z = s["logits"][e].double()
        lp = torch.log_softmax(z / c["temperature"], -1)
        p = lp.exp()
        tok = s["tokens"][e].long()
        known = tok >= 0
        if c["kind"] != "logprobs_backward":
            got["logprob"][e] = torch.where(known, lp.gather(1, tok.clamp(min=0)[:, None])[:, 0], 0.0)
            got["entropy"][e] = torch.special.entr(p).sum(1)
            got["lse"][e] = torch.logsumexp(z / c["temperature"], -1)
            if n:
                order = z.sort(dim=1, descending=True, stable=True).indices[:, :n]
                got["top_ids"][e] = order.to(torch.int32)
                got["top_logprobs"][e] = lp.gather(1, order)
        if c["kind"] == "logprobs":
            continue
        hit = torch.zeros_like(z)
        hit[known, tok[known]] = 1.0
        gl, gh = torch.where(known, s["dlogprob"][e], 0.0).double()[:, None], s["dentropy"][e].double()[:, None]
        H = torch.special.entr(p).sum(1, keepdim=True)
        got["grad"][e] = (gl * (hit - p) + gh * (torch.special.entr(p) - p * H)) / c["temperature"]
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "pages":
        return _exact_pages(case, s)
    if case["kind"] in ("rope", "rope_backward"):
        return _exact_rope(case, s)
    return _exact_logprobs(case, s)
