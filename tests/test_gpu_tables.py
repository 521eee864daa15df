"""Row starts, lengths and page tables made on the GPU, against loops over the requests."""
import random

import pytest

torch = pytest.importorskip("torch")

from oracle import cache4 as o4  # noqa: E402
from test_gpu_attention import mc  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def state(r, S, page, longest, spare):
    past = [r.randint(0, longest) for _ in range(S)]
    held = [-(-p // page) for p in past]
    n_pages = sum(held) + spare
    order = list(range(n_pages))
    r.shuffle(order)
    max_pages = max(held) + 3
    table = torch.full((S, max_pages), -1, dtype=torch.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = torch.tensor(order[at:at + h], dtype=torch.int32)
        at += h
    return past, table, order[at:] + [-5] * at


def run_reserve(mc, want, past, free, n_free, table, page, T, in_place, what):
    S = len(want)
    ref = table.clone()
    q, kl, pos, slots, left = o4.reserve(want, past, free, n_free, ref, page, T)
    d_table, d_free = table.cuda(), i32(free)
    d_past = i32(past)
    kv_len = d_past if in_place else torch.full((S + 1,), 9, dtype=torch.int32, device="cuda")[:S]
    height = i32([n_free])
    pool = mc.KVPool(page, d_free, height, None if in_place else i32([77]))
    batch = mc.KVBatch(kv_len, d_table, q_start=torch.full((S + 1,), 9, dtype=torch.int32, device="cuda"), T=T)
    positions = torch.full((T,), 9, dtype=torch.int32, device="cuda")
    d_slots = torch.full((T,), 9, dtype=torch.int64, device="cuda")
    ws = torch.full((mc.kv_tables_workspace(S),), 255, dtype=torch.uint8, device="cuda")
    print(what, flush=True)
    mc.kv_reserve(i32(want), d_past, pool, batch, ws, positions=positions, slots=d_slots)
    assert batch.q_start.tolist() == q and kv_len.tolist() == kl and pool.n_free_out.item() == left, what
    assert torch.equal(d_table.cpu(), ref) and positions.tolist() == pos and d_slots.tolist() == slots, what
    assert d_free.tolist() == free
    if not in_place:
        assert height.item() == n_free and d_past.tolist() == past


@pytest.mark.parametrize("S,page,new,longest", [(1, 16, 1, 0), (1, 256, 3000, 100), (7, 16, 40, 64), (64, 16, 1, 900),
                                                (300, 32, 20, 300), (1024, 16, 7, 50), (1025, 64, 50, 200),
                                                (5000, 16, 3, 20), (3, 128, 20000, 10)])
@pytest.mark.parametrize("short", [False, True])
def test_reserve(mc, S, page, new, longest, short):  # noqa: F811
    r = random.Random(S * 31 + short)
    want = [r.randint(0, new) for _ in range(S)]
    past, table, free = state(r, S, page, longest, 0)
    need = sum(-(-(a + b) // page) - -(-b // page) for a, b in zip(want, past))
    table = torch.cat((table, torch.full((S, new // page + 1), -1, dtype=torch.int32)), 1)
    spare = need // 2 if short else need + 3
    base = 10 ** 6
    free = [base + i for i in range(spare)] + [-5] * 4
    T = max(1, sum(want)) if not short else max(1, int(sum(want) * 0.9))
    for in_place in (False, True):
        run_reserve(mc, want, past, free, spare, table, page, T, in_place, "reserve S=%d short=%s" % (S, short))


@pytest.mark.parametrize("n_free", [-3, 0, 2, 500])
def test_reserve_odd_requests(mc, n_free):  # noqa: F811
    """Lengths that are negative, too long for their row or wrap past an int; heights outside the stack."""
    want = [5, -1, 3, 2 ** 31 - 1, 40, 0, 1, 16, 2 ** 31 - 1]
    past = [10, 5, -2, 2 ** 31 - 1, 10, 0, 64, 0, 1]
    table = torch.full((9, 4), -1, dtype=torch.int32)
    run_reserve(mc, want, past, [3, 4, 5, 6, 7, 8], n_free, table, 16, 100, False, "odd %d" % n_free)


@pytest.mark.parametrize("S,page,longest", [(1, 16, 100), (5, 32, 64), (64, 16, 900), (1024, 16, 60), (1500, 64, 500),
                                            (64, 16, 30000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_release(mc, S, page, longest, in_place):  # noqa: F811
    r = random.Random(S)
    past, table, free = state(r, S, page, longest, 11)
    done = [int(r.random() < 0.4) for _ in range(S)]
    past[0], past[-1] = past[0] if S > 1 else past[0], past[-1]
    ref = list(free)
    want_len, want_height = o4.release(done, past, ref, 11, table, page)
    d_past, d_free = i32(past), i32(free)
    kv_len = d_past if in_place else i32([9] * S)
    pool = mc.KVPool(page, d_free, i32([11]), None if in_place else i32([0]))
    ws = torch.full((mc.kv_tables_workspace(S),), 255, dtype=torch.uint8, device="cuda")
    d_table = table.cuda()
    print("release", S, flush=True)
    mc.kv_release(torch.tensor(done, dtype=torch.uint8, device="cuda"), d_past, pool, mc.KVBatch(kv_len, d_table), ws)
    assert kv_len.tolist() == want_len and pool.n_free_out.item() == want_height
    assert d_free.tolist() == ref and torch.equal(d_table.cpu(), table)


def test_release_of_too_much(mc):  # noqa: F811
    """Pages that do not fit the stack are dropped; lengths past the table's row push the row."""
    table = torch.arange(12, dtype=torch.int32).view(3, 4)
    free, past, done = [50, 51, 0, 0, 0, 0], [1000, -4, 64], [1, 1, 1]
    ref = list(free)
    want_len, height = o4.release(done, past, ref, 2, table, 16)
    pool = mc.KVPool(16, i32(free), i32([2]))
    batch = mc.KVBatch(i32(past), table.cuda())
    ws = torch.empty(mc.kv_tables_workspace(3), dtype=torch.uint8, device="cuda")
    mc.kv_release(torch.tensor(done, dtype=torch.uint8, device="cuda"), batch.kv_len, pool, batch, ws)
    assert batch.kv_len.tolist() == want_len == [0, 0, 0] and pool.n_free.item() == height == 6
    assert pool.free_list.tolist() == ref == [50, 51, 0, 1, 2, 3]


def test_pages_go_round(mc):  # noqa: F811
    """Many steps in place, replayed from a graph: no page is held twice, none is lost."""
    S, page, n_pages, T = 40, 16, 150, 64
    r = random.Random(3)
    free = list(range(n_pages))
    kv_len, table = i32([0] * S), torch.full((S, 8), -1, dtype=torch.int32, device="cuda")
    pool = mc.KVPool(page, i32(free), i32([n_pages]))
    batch = mc.KVBatch(kv_len, table, q_start=i32([0] * (S + 1)), T=T)
    ws = torch.empty(mc.kv_tables_workspace(S), dtype=torch.uint8, device="cuda")
    want, done = i32([0] * S), torch.zeros(S, dtype=torch.uint8, device="cuda")
    positions, slots = i32([0] * T), torch.zeros(T, dtype=torch.int64, device="cuda")

    def step():
        mc.kv_release(done, kv_len, pool, batch, ws)
        mc.kv_reserve(want, kv_len, pool, batch, ws, positions=positions, slots=slots)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ref_len, ref_table, ref_free, height = [0] * S, torch.full((S, 8), -1, dtype=torch.int32), list(free), n_pages
    for i in range(60):
        w = [r.choice([0, 1, 1, 2, 5]) for _ in range(S)]
        d = [int(r.random() < 0.05) for _ in range(S)]
        want.copy_(i32(w))
        done.copy_(torch.tensor(d, dtype=torch.uint8))
        graph.replay()
        ref_len, height = o4.release(d, ref_len, ref_free, height, ref_table, page)
        q, ref_len, pos, sl, height = o4.reserve(w, ref_len, ref_free, height, ref_table, page, T)
        torch.cuda.synchronize()
        assert kv_len.tolist() == ref_len and pool.n_free.item() == height and slots.tolist() == sl, i
        assert pool.free_list.tolist()[:height] == ref_free[:height]
        held = [int(ref_table[s, j]) for s in range(S) for j in range(-(-ref_len[s] // page))]
        assert sorted(held + ref_free[:height]) == list(range(n_pages)) and torch.equal(table.cpu(), ref_table)


@pytest.mark.parametrize("T", [100, 20000])
def test_without_positions_or_slots(mc, T):  # noqa: F811
    """Either array, or none; one workgroup and many."""
    r = random.Random(T)
    S, page = 30, 16
    past, table, _ = state(r, S, page, 100, 0)
    table = torch.cat((table, torch.full((S, 50), -1, dtype=torch.int32)), 1)
    want, free = [r.randint(0, T // S) for _ in range(S)], list(range(4000))
    ref = table.clone()
    q, kl, pos, sl, left = o4.reserve(want, past, free, 4000, ref, page, T)
    ws = torch.empty(mc.kv_tables_workspace(S), dtype=torch.uint8, device="cuda")
    for p, s in ((True, False), (False, True), (False, False), (True, True)):
        pool = mc.KVPool(page, i32(free), i32([4000]))
        batch = mc.KVBatch(i32([0] * S), table.cuda(), q_start=i32([0] * (S + 1)), T=T)
        positions = i32([7] * T) if p else None
        slots = torch.full((T,), 7, dtype=torch.int64, device="cuda") if s else None
        mc.kv_reserve(i32(want), i32(past), pool, batch, ws, positions=positions, slots=slots)
        assert batch.q_start.tolist() == q and batch.kv_len.tolist() == kl and pool.n_free.item() == left
        assert torch.equal(batch.page_table.cpu(), ref)
        assert positions is None or positions.tolist() == pos
        assert slots is None or slots.tolist() == sl


def test_most_requests(mc):  # noqa: F811
    """65536 requests, in place, then all of them released."""
    S, page = 65536, 16
    r = random.Random(1)
    want = [int(r.random() < 0.7) for _ in range(S)]
    past = [r.choice([0, 3, 15, 16, 31]) for _ in range(S)]
    table = torch.arange(2 * S, dtype=torch.int32).view(S, 2)
    n_pages = 3 * S
    free = list(range(2 * S, 3 * S)) + [0] * (2 * S)
    # (pages 2 s, 2 s + 1 count as held by s whether it does or not)
    ref = table.clone()
    q, kl, _, _, left = o4.reserve(want, past, free, S // 4, ref, page, S)
    pool = mc.KVPool(page, i32(free), i32([S // 4]))
    batch = mc.KVBatch(i32(past), table.cuda(), q_start=i32([0] * (S + 1)), T=S)
    ws = torch.empty(mc.kv_tables_workspace(S), dtype=torch.uint8, device="cuda")
    mc.kv_reserve(i32(want), batch.kv_len, pool, batch, ws)
    assert batch.q_start.tolist() == q and batch.kv_len.tolist() == kl and pool.n_free.item() == left
    assert torch.equal(batch.page_table.cpu(), ref)
    lens, height = o4.release([1] * S, kl, free, left, ref, page)
    mc.kv_release(torch.ones(S, dtype=torch.uint8, device="cuda"), batch.kv_len, pool, batch, ws)
    assert batch.kv_len.tolist() == lens == [0] * S and pool.n_free.item() == height <= n_pages
    assert pool.free_list.tolist() == free
