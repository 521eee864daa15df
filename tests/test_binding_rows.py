"""Rows that the calls on selected pages take: those of a ragged batch, or, without q_start, one a
sequence whatever T says.  No GPU: the library is replaced by one that only notes its calls."""
import pytest

torch = pytest.importorskip("torch")

import test_attention_abi as t  # noqa: E402

b = t.b              # the fixture that builds and loads the binding
BF16 = torch.bfloat16
S, PAGES, HQ, HKV, D, N_SEL = 5, 4, 4, 2, 64, 3


class Noted:
    """Takes any call of the library, and returns MC_OK."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def noted(b, monkeypatch):
    per = b.kv_page_bytes(16, HKV, D)
    lib = Noted()
    monkeypatch.setattr(b, "_device_of", lambda *x: 0)
    monkeypatch.setattr(b, "_here", lambda *x: 0)
    monkeypatch.setattr(b, "_stream_on", lambda dev, stream: None)
    monkeypatch.setattr(b, "kv_page_bytes", lambda *a: per)
    monkeypatch.setattr(b, "load", lambda: lib)
    return lib


def arrays(b, T, ragged=False):
    pages = [torch.zeros((8, 16 * HKV * D), dtype=BF16) for _ in range(2)]
    cache = b.KVCache(8, 16, HKV, D, k=pages[0], v=pages[1])
    start = torch.zeros(S + 1, dtype=torch.int32) if ragged else None
    batch = b.KVBatch(torch.ones(S, dtype=torch.int32), torch.zeros((S, PAGES), dtype=torch.int32), q_start=start, T=T)
    return cache, batch, b.Attention(HQ, 0.125), torch.zeros(1 << 16, dtype=torch.uint8)


def outputs(rows):
    return (torch.zeros((rows, HQ * D), dtype=BF16), torch.zeros((rows, HKV, N_SEL), dtype=torch.int32),
            torch.zeros((rows, HKV), dtype=torch.int32), torch.zeros((rows, HQ * D), dtype=BF16), torch.zeros((rows, HQ)))


def calls(b, T, rows, ragged=False, sizes=None):
    """attn_select and attn_sparse on arrays of `rows` rows (sizes: others by place in outputs())."""
    cache, batch, attn, ws = arrays(b, T, ragged)
    q, sel, count, o, lse = [outputs((sizes or {}).get(i, rows))[i] for i in range(5)]
    yield lambda: b.attn_select(q, batch, cache, b.KVSummary(cache), attn, sel, count, ws)
    yield lambda: b.attn_sparse(q, batch, cache, attn, sel, count, o, ws, lse=lse)


@pytest.mark.parametrize("T", [None, 1, 3, 5, 9])
def test_one_row_a_sequence_without_row_starts(b, noted, T):
    for call in calls(b, T, S):
        call()
    assert noted.calls == ["mc_attn_select", "mc_attn_sparse"]


@pytest.mark.parametrize("T,rows", [(3, 3), (1, 1), (9, 9), (None, 4), (5, 6)])
def test_other_rows_refused(b, noted, T, rows):
    for call in calls(b, T, rows):
        with pytest.raises(AssertionError):
            call()
    assert noted.calls == []


@pytest.mark.parametrize("which,select,sparse", [(0, 1, 1), (1, 1, 1), (2, 1, 1), (3, 0, 1), (4, 0, 1)])
def test_each_array_is_looked_at(b, noted, which, select, sparse):
    """One array of T rows among those of S."""
    for call, refused in zip(calls(b, 3, S, sizes={which: 3}), (select, sparse)):
        if refused:
            with pytest.raises(AssertionError):
                call()
    assert noted.calls == []


def test_rows_of_a_ragged_batch(b, noted):
    for call in calls(b, 7, 7, ragged=True):
        call()
    assert len(noted.calls) == 2
    for call in calls(b, 7, S, ragged=True):
        with pytest.raises(AssertionError):
            call()
    assert len(noted.calls) == 2
