"""Rotary positions into the paged cache, and back, against the float64 oracle.

Tolerances.  A turned element is x c - y s in fp32.  Cosine and sine come from an angle reduced in 64 bits: at most 2 ulp of 1 each
(2 * 2^-24 on either side), times the magnitude (half an ulp more), and the two products and their sum round once or twice: within
8 * 2^-24 * m (|x| + |y|).  A bfloat16 result adds half a step, 2^-8 |r|; an E4M3 code of r / scale half a step, 2^-4 |r / scale|, or half of
its smallest, 2^-10.  What is not turned is equal bit for bit (8-bit: the code of the exactly rounded quotient)."""
import numpy as np
import pytest
import torch

from oracle.operators_oracle import rope_turn

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _host(t):
    return t.double().cpu().numpy()


def _turn_error(x, positions, freqs, R, inter, m):
    """8 * 2^-24 m (|x| + |y|) for every element, 0 for those that pass through."""
    half = R // 2
    e = np.zeros_like(x)
    a, b = (np.arange(0, R, 2), np.arange(1, R, 2)) if inter else (np.arange(half), np.arange(half) + half)
    s = (np.abs(x[..., a]) + np.abs(x[..., b])) * 8 * 2.0 ** -24 * m
    e[..., a] = s
    e[..., b] = s
    return e


class Case:
    def __init__(self, rows, hq, hkv, d, R, inter=False, dtype="bf16", kv8=False, fused=False, page=16, padded=0, far=5000, m=1.0, seed=1, shift=0):
        self.__dict__.update(locals())
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        rnd = lambda *s: torch.randn(*s, generator=g)
        self.pool = rows // page + 5
        n_slots = self.pool * page
        slots = torch.randperm(n_slots, generator=g)[:rows].to(torch.int32)
        if padded:
            slots[rows - padded:] = torch.tensor([-1, n_slots, 2 ** 31 - 1, -2 ** 31])[torch.arange(padded) % 4].to(torch.int32)
        self.slots = slots.cuda()
        self.live = ((slots >= 0) & (slots < n_slots)).numpy()
        self.positions = torch.randint(0, far, (rows,), generator=g, dtype=torch.int32).cuda()
        self.freqs = (10000.0 ** (-torch.arange(max(R // 2, 1), dtype=torch.float64) * 2 / max(R, 2))).cuda()
        width = (hq + 2 * hkv) * d
        if fused:
            buf = rnd(rows, width + 8).to(dt).cuda()
            cut = lambda o, h: buf[:, o:o + h * d].unflatten(1, (h, d)) if h else None
            self.q, self.k, self.v = cut(0, hq), cut(hq * d, hkv), cut((hq + hkv) * d, hkv)
        else:
            def alone(h):  # shift: the rows start `shift` elements past an aligned address
                return None if not h else rnd(rows * h * d + shift).to(dt).cuda()[shift:].view(rows, h, d)
            self.q, self.k, self.v = alone(hq), alone(hkv), alone(hkv)
        self.strides = dict(q_stride=width + 8, k_stride=width + 8, v_stride=width + 8) if fused else {}
        self.k_scale = (0.01 * (1 + torch.arange(max(hkv, 1)) % 3)).float().cuda()
        self.v_scale = (0.02 * (1 + torch.arange(max(hkv, 1)) % 2)).float().cuda()

    def desc(self, av):
        ptr = lambda t: t.data_ptr() if self.kv8 else None
        return av.aurora_rope_desc(rows=self.rows, num_q_heads=self.hq, num_kv_heads=self.hkv, head_dim=self.d, rotary_dim=self.R,
                                   interleaved=int(self.inter), page_size=self.page, num_pages=self.pool,
                                   dtype=av.AURORA_F32 if self.dtype == "f32" else av.AURORA_BF16, kv_fp8=int(self.kv8),
                                   k_scale=ptr(self.k_scale), v_scale=ptr(self.v_scale), magnitude=self.m, **self.strides)

    def pools(self):
        shape = (self.pool, self.hkv, self.page, self.d)
        if self.kv8:
            return [torch.full(shape, 0x31, dtype=torch.uint8, device="cuda") for _ in range(2)]
        return [torch.full(shape, 77.0, dtype=DT[self.dtype], device="cuda") for _ in range(2)]

    def at_slots(self, pool):
        flat = pool.transpose(1, 2).reshape(-1, self.hkv, self.d)
        return flat[self.slots[torch.from_numpy(self.live).cuda()].long()], flat


CASES = [
    dict(rows=1, hq=32, hkv=8, d=128, R=128), dict(rows=160, hq=32, hkv=8, d=128, R=128, fused=True),
    dict(rows=37, hq=48, hkv=8, d=128, R=64, inter=True, kv8=True, fused=True, padded=5, far=1000000, m=1.2),
    dict(rows=300, hq=8, hkv=2, d=64, R=64, dtype="f32", page=24), dict(rows=29, hq=9, hkv=3, d=80, R=40, page=7),
    dict(rows=29, hq=9, hkv=3, d=80, R=80, inter=True, kv8=True, page=1), dict(rows=12, hq=3, hkv=1, d=7, R=6, dtype="f32", padded=4),
    dict(rows=12, hq=3, hkv=1, d=7, R=6, inter=True, kv8=True), dict(rows=65, hq=4, hkv=4, d=256, R=256, far=2 ** 31 - 1, dtype="f32"),
    dict(rows=65, hq=4, hkv=4, d=96, R=64, kv8=True, dtype="f32"), dict(rows=40, hq=0, hkv=2, d=128, R=128), dict(rows=40, hq=4, hkv=2, d=128, R=0),
    dict(rows=40, hq=4, hkv=2, d=128, R=32, shift=1), dict(rows=40, hq=4, hkv=2, d=64, R=64, inter=True, shift=1, dtype="f32"),
    dict(rows=5000, hq=16, hkv=4, d=128, R=96, fused=True, padded=900),
]


@pytest.mark.parametrize("kw", CASES, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
def test_queries_turn_and_the_cache_is_filled(gpu_lib, kw):
    av = gpu_lib
    c = Case(**kw)
    print(f"[case] {kw}", flush=True)
    kp, vp = c.pools()
    before = kp.clone(), vp.clone()
    out = torch.full((c.rows, c.hq, c.d), 55.0, dtype=DT[c.dtype], device="cuda") if c.hq else None
    av.aurora_rope_append(c.desc(av), c.q, c.k, c.v, c.positions, c.slots, c.freqs, out, kp, vp)
    torch.cuda.synchronize()
    pos, f, live = c.positions.cpu().numpy(), c.freqs.cpu().numpy(), c.live
    if c.hq:
        x = _host(c.q)
        ref = rope_turn(x, pos, f, c.R, c.inter, c.m)
        tol = _turn_error(x, pos, f, c.R, c.inter, c.m) + STEP[c.dtype] * np.abs(ref) * (c.R > 0)
        got = _host(out)
        assert (np.abs(got - ref)[live] <= tol[live]).all(), np.abs(got - ref)[live].max()
        assert np.array_equal(got[live][..., c.R:], x[live][..., c.R:])
        assert (got[~live] == 55.0).all()                        # rows behind the last sequence
    for pool, old, src, scale, turned in ((kp, before[0], c.k, c.k_scale, True), (vp, before[1], c.v, c.v_scale, False)):
        at, flat = c.at_slots(pool)
        x = _host(src)
        ref = rope_turn(x, pos, f, c.R, c.inter, c.m) if turned else x
        err = _turn_error(x, pos, f, c.R, c.inter, c.m) if turned else np.zeros_like(x)
        if c.kv8:
            sc = scale.double().cpu().numpy()[None, :c.hkv, None]
            got = at.cpu().view(torch.float8_e4m3fn).double().numpy()
            r = np.clip(ref / sc, -448, 448)
            tol = err / sc + np.maximum(2.0 ** -4 * np.abs(r), 2.0 ** -10) * (1 + 2.0 ** -20)
            assert (np.abs(got - r[live]) <= tol[live]).all()
            if not turned:  # the same quotient in fp32, rounded once: equal codes
                want = (src.float().cpu() / scale.cpu()[None, :c.hkv, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                assert torch.equal(at.cpu(), want[torch.from_numpy(live)])
        else:
            got = _host(at)
            tol = err + STEP[c.dtype] * np.abs(ref) * turned
            assert (np.abs(got - ref[live]) <= tol[live]).all(), np.abs(got - ref[live]).max()
            assert np.array_equal(got[..., c.R:], ref[live][..., c.R:])
        rest = torch.ones(flat.shape[0], dtype=torch.bool, device="cuda")
        rest[c.slots[torch.from_numpy(live).cuda()].long()] = False
        assert torch.equal(flat[rest], old.transpose(1, 2).reshape(flat.shape)[rest])   # every other slot as it was


@pytest.mark.parametrize("kw", [k for k in CASES if not k.get("kv8")], ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
def test_gradients_turn_back(gpu_lib, kw):
    av = gpu_lib
    c = Case(**kw)
    print(f"[case] {kw}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    dqo = rnd(c.rows, c.hq, c.d) if c.hq else None
    dkp, dvp = rnd(c.pool, c.hkv, c.page, c.d), rnd(c.pool, c.hkv, c.page, c.d)
    dq, dk, dv = c.q, c.k, c.v                                    # written with the strides of the rows
    av.aurora_rope_append_backward(c.desc(av), dqo, dkp, dvp, c.positions, c.slots, c.freqs, dq, dk, dv)
    torch.cuda.synchronize()
    pos, f, live = c.positions.cpu().numpy(), c.freqs.cpu().numpy(), c.live
    idx = torch.from_numpy(live).cuda()
    for got, src, turned in ((dq, dqo, True), (dk, dkp, True), (dv, dvp, False)):
        if got is None:
            continue
        x = np.zeros(got.shape)
        x[live] = _host(src[idx]) if src is dqo else _host(c.at_slots(src)[0])
        ref = rope_turn(x, pos, f, c.R, c.inter, c.m, back=True) if turned else x
        tol = (_turn_error(x, pos, f, c.R, c.inter, c.m) if turned else 0) + STEP[c.dtype] * np.abs(ref)
        assert (np.abs(_host(got) - ref) <= tol).all(), np.abs(_host(got) - ref).max()
        assert (_host(got)[~live] == 0).all()


@pytest.mark.parametrize("kv8", [False, True])
def test_a_cache_and_rows_past_32_bits(gpu_lib, kv8):
    """Pools of more than 2^32 elements, the last slots of them; rows of queries 2^31 elements apart.  And the gradients' way back."""
    av = gpu_lib
    rows, hq, hkv, d, page, P, far = 5, 2, 8, 128, 16, 270000, 2 ** 31 + 64
    kp, vp = (torch.zeros((P, hkv, page, d), dtype=torch.uint8 if kv8 else torch.bfloat16, device="cuda") for _ in range(2))
    assert kp.numel() > 2 ** 32
    wide = torch.zeros((rows - 1) * far + hq * d, dtype=torch.bfloat16, device="cuda")
    q = wide.as_strided((rows, hq, d), (far, d, 1))
    q.copy_(torch.randn(rows, hq, d, device="cuda"))
    k, v = (torch.randn(rows, hkv, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    slots = torch.tensor([P * page - 1, 3, P * page - 33, 2 ** 22 - 1, P * page // 2], dtype=torch.int32, device="cuda")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 1000
    f = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)
    one = torch.ones(hkv, device="cuda")
    desc = av.aurora_rope_desc(rows=rows, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, rotary_dim=d, page_size=page, num_pages=P, dtype=av.AURORA_BF16,
                               kv_fp8=int(kv8), k_scale=one.data_ptr(), v_scale=one.data_ptr(), q_stride=far, q_out_stride=far)
    before = _host(q)
    av.aurora_rope_append(desc, q, k, v, pos, slots, f.cuda(), q, kp, vp)          # (in place)
    torch.cuda.synchronize()
    page_of, off = slots.long() // page, slots.long() % page
    p = pos.cpu().numpy()
    ref = rope_turn(before, p, f.numpy(), d, False)
    assert (np.abs(_host(q) - ref) <= _turn_error(before, p, f, d, False, 1.0) + STEP["bf16"] * np.abs(ref)).all()
    if kv8:
        assert torch.equal(vp[page_of, :, off], v.float().to(torch.float8_e4m3fn).view(torch.uint8))
    else:
        assert torch.equal(vp[page_of, :, off], v)
        ref = rope_turn(_host(k), p, f.numpy(), d, False)
        assert (np.abs(_host(kp[page_of, :, off]) - ref) <= _turn_error(_host(k), p, f, d, False, 1.0) + STEP["bf16"] * np.abs(ref)).all()
    at = kp[page_of, :, off].clone()
    kp[page_of, :, off] = 0                                       # nothing else was written
    vp[page_of, :, off] = 0
    assert all(not bool(x.any()) for pool in (kp, vp) for x in pool.split(10000))
    if kv8:
        return
    del vp
    dk = torch.zeros((P, hkv, page, d), device="cuda")
    dk[page_of, :, off] = at.float()
    desc.q_out_stride, desc.num_q_heads = 0, 0
    got, gv = torch.zeros_like(k), torch.zeros_like(v)
    av.aurora_rope_append_backward(desc, None, dk, dk, pos, slots, f.cuda(), None, got, gv)
    torch.cuda.synchronize()
    x = _host(at)
    ref = rope_turn(x, p, f.numpy(), d, False, back=True)
    assert (np.abs(_host(got) - ref) <= _turn_error(x, p, f, d, False, 1.0) + STEP["bf16"] * np.abs(ref)).all() and torch.equal(gv, at)


def test_in_place_queries_alone_and_without_slots(gpu_lib):
    av = gpu_lib
    for fused in (False, True):
        c = Case(rows=700, hq=8, hkv=2, d=128, R=128, fused=fused)
        x = _host(c.q)
        d = c.desc(av)
        d.num_kv_heads, d.q_out_stride = 0, d.q_stride
        rest = None if not fused else (c.k.clone(), c.v.clone())
        av.aurora_rope_append(d, c.q, None, None, c.positions, None, c.freqs, c.q, None, None)
        torch.cuda.synchronize()
        ref = rope_turn(x, c.positions.cpu().numpy(), c.freqs.cpu().numpy(), 128, False)
        tol = _turn_error(x, None, None, 128, False, 1.0) + STEP["bf16"] * np.abs(ref)
        assert (np.abs(_host(c.q) - ref) <= tol).all()
        if fused:
            assert torch.equal(c.k, rest[0]) and torch.equal(c.v, rest[1])


def test_values_that_do_not_fit_eight_bits(gpu_lib):
    """Beyond the largest code, ties between codes, the smallest ones, infinities and NaN."""
    av = gpu_lib
    vals = torch.tensor([448.0, 449, 1e30, -1e30, float("inf"), -float("inf"), float("nan"), 464, -480, 17, 19, 18, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10,
                         1.5 * 2.0 ** -10, 0.0, -0.0, 1.0625, 1.1875])
    x = torch.zeros(1, 1, 32)
    x[0, 0, :len(vals)] = vals
    one = torch.ones(1, device="cuda")
    xc = x.cuda()
    kp = torch.zeros(1, 1, 1, 32, dtype=torch.uint8, device="cuda")
    vp = kp.clone()
    d = av.aurora_rope_desc(rows=1, num_kv_heads=1, head_dim=32, page_size=1, num_pages=1, dtype=av.AURORA_F32, kv_fp8=1,
                            k_scale=one.data_ptr(), v_scale=one.data_ptr())
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    av.aurora_rope_append(d, None, xc, xc, zero, zero, None, None, kp, vp)
    torch.cuda.synchronize()
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).flatten()
    got = vp.cpu().flatten()
    nan = torch.isnan(x.flatten())
    assert torch.equal(got[~nan], want[~nan]) and ((got[nan] & 0x7f) == 0x7f).all() and torch.equal(got, kp.cpu().flatten())


def test_a_captured_call_follows_its_inputs(gpu_lib):
    av = gpu_lib
    c = Case(rows=160, hq=8, hkv=2, d=128, R=128)
    kp, vp = c.pools()
    out = torch.zeros_like(c.q)
    d = c.desc(av)
    call = lambda: av.aurora_rope_append(d, c.q, c.k, c.v, c.positions, c.slots, c.freqs, out, kp, vp)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for k in range(3):
        c.q.copy_(torch.randn_like(c.q))
        c.positions.add_(11)
        kp.fill_(1.0)
        g.replay()
        torch.cuda.synchronize()
        seen = out.clone(), kp.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(seen[0], out) and torch.equal(seen[1], kp)
