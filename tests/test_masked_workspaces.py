"""The workspace that the binding takes for attention over the cache with a window or a tree
is the one that the library asks for at that call, whatever calls went before."""
import ctypes

import pytest
import torch

from paper_2505_08098_amd import dense
from test_dense_refusals import _cache


class _Binding:
    """What the workspace's size and place follow from in a dense.Cache (no GPU needed)."""

    def __init__(self, **sizes):
        self._struct = _cache(**sizes)
        self._ref = ctypes.byref(self._struct)
        self._bytes = {}
        self.device = torch.device("cpu")


@pytest.mark.parametrize("name,sizes", [
    ("f3s_cache_attend_window", (200, 4, 8, 32, 4000, 4)),
    ("f3s_cache_attend_tree", (200, 4, 8, 32, 0)),
])
def test_rows_forced_between_calls(monkeypatch, name, sizes):
    cache = _Binding(n_kv_heads=8, d=128, page_size=64)
    need = getattr(dense._lib(), name + "_workspace_bytes")
    seen = set()
    for rows in (None, "128", "16", "256", None):
        monkeypatch.delenv("F3S_OWN_ROWS", raising=False)
        if rows:
            monkeypatch.setenv("F3S_OWN_ROWS", rows)
        want = need(cache._ref, *sizes)
        ws, nbytes = dense._attend_workspace(cache, name, sizes)
        assert nbytes == want and ws.numel() == want, rows
        seen.add(want)
    assert len(seen) > 1


@pytest.mark.parametrize("B,items", [(1024, 1024 + 512), (1025, 1025), (8192, 8192)])
def test_trees_of_many_sequences_are_not_divided(monkeypatch, B, items):
    """Every workgroup searches all lengths for its item: with 8,192 sequences that took 13
    times as long as their keys.  An item has d values and two numbers a row."""
    monkeypatch.delenv("F3S_OWN_ROWS", raising=False)
    c = _cache(n_kv_heads=8, d=64, page_size=64)
    n, heads = 16, 32
    size = dense._lib().f3s_cache_attend_tree_workspace_bytes(ctypes.byref(c), 100, B, n, heads, 0)
    up = lambda x: -(-x // 256) * 256
    rows = items * n * heads
    assert size == up(rows * 64 * 4) + up(rows * 8) + up(B * 8)


@pytest.mark.gpu
def test_rows_forced_between_calls_of_one_cache(gpu, monkeypatch):
    cache = gpu.Cache.empty(40, 64, 8, 128, device="cuda:0")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")
    table = torch.arange(40, dtype=torch.int32, device="cuda:0").view(4, 10)
    table = torch.cat([table] + [torch.full_like(table, -1)] * 19, 1)   # room for 200 pages
    lens = ints([600, 30, 0, 511])
    states = [torch.randn((4, 600, 8, 128), device="cuda:0").half() for _ in "KV"]
    gpu.cache_write(cache, *states, table, lens)
    Q = torch.randn((4, 8, 32, 128), device="cuda:0").half()
    parents = ints([[-1, 0, 0, 1, 1, 2, 5, 5]] * 4)
    K, V = gpu.cache_read(cache, table, lens, 600, torch.float32)
    # Of each of two kernels: a result's rounding, and its probabilities', which weigh V; of
    # lse, what 128 sums of a score in 32 bits lose (a sum of probabilities loses less).
    u, steps = 2.0 ** -11, 128 * 2.0 ** -24
    score = float(Q.float().norm(dim=3).max() * K.norm(dim=3).max()) * 128 ** -0.5
    calls = [lambda: gpu.cache_attend_window(cache, Q, table, lens, 4000, 4),
             lambda: gpu.cache_attend_tree(cache, Q, table, lens, parents)]
    for call in calls:
        monkeypatch.delenv("F3S_OWN_ROWS", raising=False)
        O, lse = call()
        for rows in ("128", "16", "256"):
            monkeypatch.setenv("F3S_OWN_ROWS", rows)
            O2, lse2 = call()
            assert torch.allclose(O.float(), O2.float(), rtol=2 * u, atol=2 * u * V.abs().max())
            assert torch.allclose(lse, lse2, rtol=0, atol=2 * steps * score)


@pytest.mark.skipif(torch.cuda.is_available(),
                    reason="made-up addresses: only where nothing can launch")
@pytest.mark.parametrize("B,n,kv,g,d,P,pieces", [
    (16, 63, 8, 4, 128, 2001, 2),      # of 16 units
    (16, 63, 8, 4, 128, 16000, 4),     # 1,024 workgroups: two rounds
    (16, 63, 8, 4, 128, 1 << 20, 4),
    (4, 63, 8, 4, 128, 4001, 4), (32, 63, 8, 4, 128, 4001, 2),
    (64, 256, 8, 4, 128, 6001, 1),     # one piece fills more
    (4, 63, 2, 8, 256, 30000, 16), (64, 32, 8, 4, 64, 8001, 3),
])
def test_pieces_of_a_prefix_beside_the_own_keys(monkeypatch, B, n, kv, g, d, P, pieces):
    """A piece of a prefix has d values and two numbers for every row: what the least workspace
    of a call with a prefix has more than that of one without."""
    monkeypatch.setenv("F3S_PREFIX_ROWS", "128")
    monkeypatch.setenv("F3S_OWN_ROWS", "128")
    A = 1 << 44                        # (an address that is never read)
    c = _cache(n_kv_heads=kv, d=d, page_size=64)
    heads = kv * g

    def least(prefix_len):
        def refused(nbytes):
            return dense._lib().f3s_cache_attend_tree(
                ctypes.byref(c), A, 0, 2 * A, 3 * A, 4 * A, 2000, 5 * A, B, n, heads, 6 * A,
                7 * A if prefix_len else None, prefix_len, 0.1, 8 * A, nbytes, None) == 1
        lo, hi = 0, 1 << 40
        assert not refused(hi) and refused(256)
        while hi - lo > 1:
            mid = (lo + hi) // 2
            lo, hi = (mid, hi) if refused(mid) else (lo, mid)
        return hi

    rows = B * n * heads
    more = least(P) - least(0)
    assert abs(more - pieces * rows * (d + 2) * 4) <= 3 * 256


def test_a_size_is_asked_again_where_it_does_not_do(monkeypatch):
    """A call that the library refuses with the size known so far is made once more with the
    size that it asks for now; one that it refuses for another reason is not."""
    cache, calls = _Binding(n_kv_heads=8, d=128, page_size=64), []
    sizes = (200, 4, 8, 32, 4000, 4)

    class Library:
        need = 512

        def f3s_cache_attend_window_workspace_bytes(self, *args):
            calls.append("size")
            return self.need

        def f3s_cache_attend_window(self, wrong, ws, nbytes, stream):
            calls.append(nbytes)
            return 1 if wrong or nbytes < self.need else 0

    lib = Library()
    monkeypatch.setattr(dense, "_lib", lambda: lib)
    monkeypatch.setattr(dense, "_raw_stream", lambda index: 0)
    attend = lambda wrong: dense._attend(cache, "f3s_cache_attend_window", sizes, wrong)
    attend(False)
    attend(False)
    assert calls == ["size", 512, 512]
    lib.need, calls[:] = 1024, []
    attend(False)
    attend(False)
    assert calls == [512, "size", 1024, 1024]
    lib.need, calls[:] = 256, []
    attend(False)                       # (a larger one does)
    assert calls == [1024]
    calls[:] = []
    with pytest.raises(dense.F3SError):
        attend(True)
    lib.need = 1024
    calls[:] = []
    with pytest.raises(dense.F3SError):
        attend(True)
    assert calls == [256, "size", 1024]
    calls[:] = []
    with pytest.raises(dense.F3SError):
        attend(True)
    assert calls == [1024, "size"]
