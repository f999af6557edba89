"""Block tables and slot maps against the oracle: whole numbers, equal everywhere, cells and entries that the call must leave alone
among them."""
import numpy as np
import pytest
import torch

from oracle.operators_oracle import cache_plan

pytestmark = pytest.mark.gpu


def _state(rng, B, page, width, free_share=1.0, grow=0.5, chunk=None, fresh=False):
    """A consistent state: distinct pages held, the rest of the pool (a share of it) on the stack, and wanted lengths."""
    pages = lambda n: -(-n // page)
    top = page * width
    held = np.zeros(B, np.int64) if fresh else rng.integers(0, top + 1, B)
    kind = rng.random(B)
    want = np.where(kind < grow, np.minimum(held + rng.integers(1, (chunk or top) + 1, B), top), rng.integers(0, np.maximum(held, 1) + 1, B))
    want = np.where(kind > 0.95, held, np.minimum(want, top))
    P = B * width + 7
    ids = rng.permutation(P).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :pages(held[b])] = ids[at:at + pages(held[b])]
        at += pages(held[b])
    n = int((P - at) * free_share)
    free = np.full(P, -5, np.int32)
    free[:n] = ids[at:at + n]
    return held.astype(np.int32), want.astype(np.int32), table, free, n


def _run(av, held, want, table, free, n, page, max_rows, in_place=False, optional=True, shift=0, stream=None):
    B, P = len(want), len(free)
    width = table.shape[1]
    i32 = torch.int32
    d = av.aurora_cache_plan_desc(batch=B, page_size=page, max_pages_per_seq=width, num_pages=P, max_rows=max_rows or 0)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    h = None if held is None else dev(held)
    w, t, f, c = dev(want), dev(table), dev(free), dev([n])
    rows = max_rows or 0
    out = dict(count=c if in_place else torch.full((1,), -9, dtype=i32, device="cuda"),
               seq_lens=(w if in_place else torch.full((max(B, 1),), -9, dtype=i32, device="cuda")),
               row_start=torch.full((B + 1,), -9, dtype=i32, device="cuda") if optional else None,
               positions=torch.full((rows + shift + 4,), -9, dtype=i32, device="cuda")[shift:],
               slots=torch.full((rows + shift + 4,), -9, dtype=i32, device="cuda")[shift:],
               info=torch.full((4,), -9, dtype=i32, device="cuda") if optional else None)
    ws = torch.empty(av.aurora_cache_plan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    call = lambda: av.aurora_cache_plan(d, h, w, t, f, c, out["count"], out["seq_lens"], out["row_start"],
                                        out["positions"] if max_rows is not None else None, out["slots"] if max_rows is not None else None,
                                        out["info"], ws, stream)
    call()
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in out.items() if v is not None}
    got.update(table=t.cpu().numpy(), free=f.cpu().numpy())
    return got, call


def _check(av, held, want, table, free, n, page, max_rows, **kw):
    print(f"[case] B={len(want)} page={page} width={table.shape[1]} free={n} max_rows={max_rows} {kw}", flush=True)
    ref = cache_plan(held if held is not None else np.zeros(len(want), np.int32), want, table, free, n, page, max_rows)
    got, call = _run(av, held, want, table, free, n, page, max_rows, **kw)
    B = len(want)
    for k in ("table", "free", "row_start", "info"):
        if k in got:
            assert np.array_equal(got[k], ref[k]), k
    assert np.array_equal(got["seq_lens"][:B], ref["seq_lens"])
    assert got["count"][0] == ref["count"]
    rows = max_rows or 0
    assert np.array_equal(got["positions"][:rows], ref["positions"]) and np.array_equal(got["slots"][:rows], ref["slots"])
    assert (got["positions"][rows:] == -9).all() and (got["slots"][rows:] == -9).all()
    return ref, call


@pytest.mark.parametrize("batch,page,width", [(1, 16, 5), (5, 4, 9), (64, 16, 33), (255, 1, 20), (256, 16, 40), (1024, 24, 11),
                                              (1025, 16, 6), (3000, 16, 9)])
def test_plans_of_mixed_batches(gpu_lib, batch, page, width):
    rng = np.random.default_rng(batch)
    s = _state(rng, batch, page, width, chunk=5 if batch % 2 else None)
    total = int(np.maximum(s[1].astype(np.int64) - s[0], 0).sum())
    _check(gpu_lib, *s, page, total + 13)
    _check(gpu_lib, *s, page, total + 13, in_place=True)
    _check(gpu_lib, *s, page, None, optional=False)          # tables alone
    _check(gpu_lib, *s, page, total, shift=1, optional=False)  # rows that start at 4 bytes, and no spare ones


@pytest.mark.parametrize("batch", [7, 300, 2100])
def test_pages_or_rows_run_out(gpu_lib, batch):
    rng = np.random.default_rng(batch + 1)
    held, want, table, free, n = _state(rng, batch, 16, 13, free_share=0.05, grow=0.8)
    total = int(np.maximum(want.astype(np.int64) - held, 0).sum())
    ref, _ = _check(gpu_lib, held, want, table, free, n, 16, total + 5)
    assert ref["info"][3] > 0
    ref, _ = _check(gpu_lib, held, want, table, np.where(free < 0, -5, free), n, 16, total // 2)
    assert ref["info"][3] > 0
    _check(gpu_lib, held, want, table, free, 0, 16, total)


def test_lengths_that_fit_no_table_are_refused_alone(gpu_lib):
    rng = np.random.default_rng(8)
    held, want, table, free, n = _state(rng, 40, 16, 6, grow=1.0)
    want[3], want[11], want[12], held[20] = 97, -1, 2 ** 31 - 1, -4
    held[25], want[25] = 200, 10                             # holds more than its row of the table: not touched
    ref, _ = _check(gpu_lib, held, want, table, free, n, 16, 10000)
    assert ref["info"][3] >= 4


def test_no_requests_and_requests_that_begin(gpu_lib):
    free = np.arange(50, dtype=np.int32)
    _check(gpu_lib, np.zeros(0, np.int32), np.zeros(0, np.int32), np.zeros((0, 4), np.int32), free, 50, 16, 9)
    for lens in ([0], [1], [16], [17, 0, 64, 5]):
        table = np.full((len(lens), 4), -1, np.int32)
        _check(gpu_lib, None, np.array(lens, np.int32), table, free, 50, 16, sum(lens) + 2)


def test_a_long_prefill_and_its_end(gpu_lib):
    """Some 200 000 rows, then every request ends: pages go back in order."""
    rng = np.random.default_rng(9)
    B, page, width = 20, 16, 1300
    want = rng.integers(200, page * width, B).astype(np.int32)
    P = B * width
    free = rng.permutation(P).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    ref, _ = _check(gpu_lib, None, want, table, free, P, page, int(want.sum()))
    done = np.zeros(B, np.int32)
    done[3] = want[3]
    _check(gpu_lib, want, done, ref["table"], ref["free"], ref["count"], page, 0)
    _check(gpu_lib, want, done, ref["table"], ref["free"], ref["count"], page, None, in_place=True)


def test_as_many_rows_as_there_can_be(gpu_lib):
    """The padding of 2^31 - 1 rows: their numbers stay within 32 bits."""
    av = gpu_lib
    rows = 2 ** 31 - 1
    d = av.aurora_cache_plan_desc(batch=2, page_size=16, max_pages_per_seq=4, num_pages=9, max_rows=rows)
    dev = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    table, free, lens = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), torch.arange(9, dtype=torch.int32, device="cuda"), dev(0, 0)
    positions, slots = (torch.full((rows,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.empty(av.aurora_cache_plan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    count = dev(9)
    av.aurora_cache_plan(d, None, dev(3, 17), table, free, count, count, lens, None, positions, slots, None, ws)
    torch.cuda.synchronize()
    assert lens.tolist() == [3, 17] and int(count) == 6 and table.tolist() == [[8, -1, -1, -1], [7, 6, -1, -1]]
    assert slots[:20].tolist() == [128, 129, 130] + list(range(112, 128)) + [96] and positions[:20].tolist() == [0, 1, 2] + list(range(17))
    assert int(slots[20:].max()) == -1 and int(slots[20:].min()) == -1 and int(positions[20:].max()) == 0 and int(positions[20:].min()) == 0


def test_a_call_may_be_repeated_and_captured(gpu_lib):
    """Distinct outputs: the same call on the same state gives the same result, also from a graph that is replayed on new lengths."""
    av = gpu_lib
    rng = np.random.default_rng(10)
    B, page, width = 48, 16, 30
    held, want, table, free, n = _state(rng, B, page, width, chunk=9)
    rows = 2000
    d = av.aurora_cache_plan_desc(batch=B, page_size=page, max_pages_per_seq=width, num_pages=len(free), max_rows=rows)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    h, w, t, f, c = dev(held), dev(want), dev(table), dev(free), dev([n])
    o = [torch.zeros(k, dtype=torch.int32, device="cuda") for k in (1, B, B + 1, rows, rows, 4)]
    ws = torch.empty(av.aurora_cache_plan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    call = lambda: av.aurora_cache_plan(d, h, w, t, f, c, o[0], o[1], o[2], o[3], o[4], o[5], ws)
    with torch.cuda.stream(side):
        call()
        call()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for k in range(4):
        held, want, table, free, n = _state(np.random.default_rng(20 + k), B, page, width, chunk=9 + k)
        for dst, src in ((h, held), (w, want), (t, table), (f, free), (c, np.array([n]))):
            dst.copy_(dev(src))
        g.replay()
        torch.cuda.synchronize()
        ref = cache_plan(held, want, table, free, n, page, rows)
        for a, b in zip(o, ("count", "seq_lens", "row_start", "positions", "slots", "info")):
            assert np.array_equal(a.cpu().numpy(), np.atleast_1d(ref[b])), b
        assert np.array_equal(t.cpu().numpy(), ref["table"]) and np.array_equal(f.cpu().numpy(), ref["free"])


@pytest.mark.parametrize("batch,width,page", [(40, 450, 16), (1100, 20, 16), (1030, 13, 24)])
@pytest.mark.parametrize("spare", [0, 1, 1030])
def test_plans_of_two_launches_on_both_sides_of_a_row_a_thread(gpu_lib, batch, width, page, spare):
    """In place over many workgroups, and more requests than one plans at a time: up to 2^18 rows, and just past them."""
    rng = np.random.default_rng(batch + spare)
    s = _state(rng, batch, page, width, grow=0.6)
    _check(gpu_lib, *s, page, 2 ** 18 + spare, in_place=True)
    _check(gpu_lib, *s, page, 2 ** 18 + spare, shift=spare % 2)
