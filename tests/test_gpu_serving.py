"""Tables, append, bounds, selection and attention as one step of a serving loop: eager, on another
stream, and captured into graphs that share a workspace, over caches of each kind."""
import random

import pytest

torch = pytest.importorskip("torch")

import test_gpu_attention as ta  # noqa: E402
from oracle import cache4 as o4  # noqa: E402

pytestmark = pytest.mark.gpu

mc = ta.mc
BF16, E4M3, E2M1 = torch.bfloat16, torch.float8_e4m3fn, torch.float4_e2m1fn_x2
S, PAGE, N_PAGES, T, MAX_PAGES, N_SEL = 5, 16, 60, 64, 14, 4
HQ, HKV, D = 6, 2, 64


class Loop:
    """A program's buffers and one step over them."""

    def __init__(self, mc, kind):
        self.mc = mc

        def i32(*shape):
            return torch.zeros(shape, dtype=torch.int32, device="cuda")

        scale = torch.full((HKV,), 0.02, device="cuda") if kind == E4M3 else None
        self.cache = mc.KVCache(N_PAGES, PAGE, HKV, D, dtype=kind, k_scale=scale, v_scale=scale)
        self.summary = mc.KVSummary(self.cache)
        self.pool = mc.KVPool(PAGE, torch.arange(N_PAGES, dtype=torch.int32, device="cuda"), i32(1) + N_PAGES)
        table = torch.full((S, MAX_PAGES), -1, dtype=torch.int32, device="cuda")
        self.batch = mc.KVBatch(i32(S), table, q_start=i32(S + 1), T=T)
        self.want, self.done = i32(S), torch.zeros(S, dtype=torch.uint8, device="cuda")
        self.positions, self.slots = i32(T), torch.zeros(T, dtype=torch.int64, device="cuda")
        self.qkv = torch.zeros((T, (HQ + 2 * HKV) * D), dtype=BF16, device="cuda")
        at = torch.arange(PAGE * MAX_PAGES, dtype=torch.float64)[:, None]
        ang = at * 1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        self.prep = mc.QKPrep(rope=torch.stack((ang.cos(), ang.sin()), -1).float().cuda().contiguous())
        self.attn = mc.Attention(HQ, D ** -0.5)
        self.q = torch.zeros((T, HQ * D), dtype=BF16, device="cuda")
        self.o, self.o_all = (torch.zeros((T, HQ * D), dtype=BF16, device="cuda") for _ in range(2))
        self.lse, self.lse_all = (torch.zeros((T, HQ), device="cuda") for _ in range(2))
        self.sel, self.count = i32(T, HKV, N_SEL), i32(T, HKV)
        n = max(mc.attn_workspace(T, HQ, HKV, D), mc.attn_select_workspace(T, HKV, MAX_PAGES), mc.kv_tables_workspace(S))
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")

    def step(self, ws=None):
        m, ws = self.mc, self.ws if ws is None else ws
        m.kv_release(self.done, self.batch.kv_len, self.pool, self.batch, ws)
        m.kv_reserve(self.want, self.batch.kv_len, self.pool, self.batch, ws, positions=self.positions, slots=self.slots)
        a, b = HQ * D, (HQ + HKV) * D
        m.kv_append(self.qkv[:, :a], self.qkv[:, a:b], self.qkv[:, b:], self.prep, self.batch, self.cache, self.q)
        m.kv_summarize(self.batch, self.cache, self.summary)
        m.attn_select(self.q, self.batch, self.cache, self.summary, self.attn, self.sel, self.count, ws, keep_last=2)
        m.attn_sparse(self.q, self.batch, self.cache, self.attn, self.sel, self.count, self.o, ws, lse=self.lse)
        m.attn_prefill(self.q, self.batch, self.cache, self.attn, self.o_all, ws, lse=self.lse_all)

    def feed(self, want, done, qkv):
        self.want.copy_(torch.tensor(want, dtype=torch.int32))
        self.done.copy_(torch.tensor(done, dtype=torch.uint8))
        self.qkv.copy_(qkv)

    def results(self):
        c = self.cache
        return dict(k=c.k, v=c.v, bounds=self.summary.bounds, scale=self.summary.scale, free=self.pool.free_list,
                    n_free=self.pool.n_free, q_start=self.batch.q_start, kv_len=self.batch.kv_len,
                    table=self.batch.page_table, positions=self.positions, slots=self.slots, q=self.q, o=self.o,
                    o_all=self.o_all, lse=self.lse, lse_all=self.lse_all, sel=self.sel, count=self.count)


def inputs(seed, steps=14):
    r, g = random.Random(seed), torch.Generator().manual_seed(seed)
    for i in range(steps):
        want = [r.choice([18, 12, 5, 0]) if i % 2 == 0 else 1 for _ in range(S)]
        done = [int(i % 5 == 4 and r.random() < 0.15) for _ in range(S)]
        yield want, done, torch.randn((T, (HQ + 2 * HKV) * D), generator=g).to(BF16)


def raw(t):
    return t.view(torch.uint8) if t.dtype == E4M3 else t


def same(a, b, what):
    for name, x in a.results().items():
        assert torch.equal(raw(x), raw(b.results()[name])), (what, name)


@pytest.mark.parametrize("kind", [BF16, E4M3, E2M1])
def test_loop(mc, kind):
    """Eager steps against those on another stream and against two graphs that share a workspace and are
    replayed in turn; where all pages are selected, sparse attention is prefill's."""
    eager, side, graph = Loop(mc, kind), Loop(mc, kind), Loop(mc, kind)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):       # (a step without requests changes nothing)
        graph.step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graph.step()
        graphs.append(g)
    for i, step in enumerate(inputs(3)):
        print(kind, i, flush=True)
        for loop in (eager, side, graph):
            loop.feed(*step)
        torch.cuda.synchronize()
        eager.step()
        with torch.cuda.stream(stream):
            side.step()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        same(eager, side, "stream, step %d" % i)
        same(eager, graph, "graph, step %d" % i)
        rows = int(eager.batch.q_start[-1])
        pos = eager.positions.cpu()
        assert bool((pos[:rows] >= 0).all()) and bool((pos[rows:] == -1).all())
        for t in range(rows):
            pages = int(pos[t]) // PAGE + 1
            assert eager.count[t].tolist() == [min(pages, N_SEL)] * HKV
            if pages <= N_SEL:
                # both within 2^-8 of a weighted mean of values (weights and result rounded to bf16: 2 2^-8 each)
                most = float(eager.qkv[:, (HQ + HKV) * D:].abs().max()) * 1.2 + 5.0
                d = float((eager.o[t].float() - eager.o_all[t].float()).abs().max())
                assert d <= 4 * ta.oa.BF * most and float((eager.lse[t] - eager.lse_all[t]).abs().max()) <= 1e-5


@pytest.mark.parametrize("kind", [BF16, E2M1])
def test_loop_against_the_oracle(mc, kind):
    """After some steps: tables, what the cache holds, bounds, selection and attention of the last."""
    loop = Loop(mc, kind)
    free, n_free = list(range(N_PAGES)), N_PAGES
    table, lens = torch.full((S, MAX_PAGES), -1, dtype=torch.int32), [0] * S
    held = [[] for _ in range(S)]
    for want, done, qkv in inputs(8, 17):
        loop.feed(want, done, qkv)
        loop.step()
        lens, n_free = o4.release(done, lens, free, n_free, table, PAGE)
        q_start, lens, positions, slots, n_free = o4.reserve(want, lens, free, n_free, table, PAGE, T)
        k, v = (torch.zeros((T, HKV * D), dtype=BF16, device="cuda") for _ in range(2))
        mc.kv_read(loop.batch, loop.cache, k, v)
        for s in range(S):
            if done[s]:
                held[s] = []
            for t in range(q_start[s], q_start[s + 1]):
                held[s].append((k[t].double().cpu(), v[t].double().cpu()))
    assert loop.batch.kv_len.tolist() == lens and torch.equal(loop.batch.page_table.cpu(), table)
    assert loop.positions.tolist() == positions and loop.slots.tolist() == slots
    assert [len(h) for h in held] == lens and max(lens) > N_SEL * PAGE
    g = HQ // HKV
    q = loop.q.cpu()
    for s in range(S):
        if not lens[s]:
            continue
        ks, vs = (torch.stack([x[i] for x in held[s]]).view(-1, HKV, D) for i in (0, 1))
        for t in range(q_start[s], q_start[s + 1]):
            for h in range(HKV):
                bounds = [o4.bounds(ks[p * PAGE:(p + 1) * PAGE, h].float()) for p in range(-(-lens[s] // PAGE))]
                lo, hi, sc = (torch.stack([x[i] for x in bounds]) for i in range(3))
                qr = q[t, h * g * D:(h + 1) * g * D].view(g, D)
                sel = o4.select(qr.float(), lo, hi, sc, positions[t], PAGE, N_SEL, 1, 2)
                assert loop.sel[t, h].tolist() == sel + [-1] * (N_SEL - len(sel)), (s, t, h)
                times = torch.zeros(lens[s], dtype=torch.int64)
                for p in sel:
                    times[p * PAGE:(p + 1) * PAGE] = 1
                for i in range(g):
                    o, l, to, tl = o4.attend_some(qr[i:i + 1].double(), ks[:, h], vs[:, h], positions[t], times,
                                                  scale=D ** -0.5)
                    hq = h * g + i
                    ta.check(loop.o[t:t + 1, hq * D:(hq + 1) * D], o, to, "o t=%d hq=%d" % (t, hq))
                    ta.check(loop.lse[t:t + 1, hq], l, tl, "lse t=%d hq=%d" % (t, hq))


def test_timing_names(mc):
    """The step's launches are found under their names."""
    loop = Loop(mc, E2M1)
    want, done, qkv = next(inputs(1, 1))
    loop.feed(want, done, qkv)
    mc.timing_enable(True)
    try:
        loop.step()
        for name, n in (("kv_tables", 2), ("kv_append", 1), ("kv_summary", 1), ("attn_select", 1), ("attn_sparse", 1),
                        ("attn_prefill", 1), ("kv_read", 0)):
            ms, launches = mc.timing_read(name)
            assert launches == n and (ms > 0.0) == (n > 0), name
    finally:
        mc.timing_enable(False)
