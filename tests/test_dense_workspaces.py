"""A workspace that lies over what a call reads is refused: partial results would
be written over lengths and page numbers that other workgroups still read."""
import math

import pytest
import torch

from paper_2505_08098_amd import dense
from test_dense_refusals import A, HIP, INVALID, _attend, _cache, _read, _write

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="made-up addresses: only where nothing can launch")


@pytest.fixture(scope="module")
def lib():
    return dense._lib()


@no_gpu
@pytest.mark.parametrize("what", [
    dict(Q=32 * A), dict(Q=32 * A + 256), dict(lens=32 * A + 512), dict(table=32 * A + 1024),
    dict(prefix=32 * A + 64, P=5), dict(Q=32 * A - 256),
    dict(table=32 * A - 3 * 400 * 4 + 4),                    # by its last word
    dict(cache=dict(k=32 * A)), dict(cache=dict(v=32 * A + 256)),
    dict(cache=dict(k_exp=32 * A + 16)), dict(cache=dict(v_exp=32 * A)),
])
def test_attend_workspace_over_an_input(lib, what):
    change = {n: x for n, x in what.items() if n != "cache"}
    assert _attend(lib, _cache(**what.get("cache", {})), **change) == INVALID


@no_gpu
def test_attend_workspace_beside_the_inputs(lib):
    assert _attend(lib, _cache(), table=32 * A - 3 * 400 * 4) == HIP
    # (what the call does not use does not count)
    assert _attend(lib, _cache(), pages=16, Q=32 * A, ws=32 * A) == HIP


@pytest.mark.gpu
def test_cross_workspace_over_an_input(gpu):
    dev = torch.device("cuda:0")
    plan = gpu.CrossPlan([0, 20], [0, 900], 4, 2, 64, device=dev)
    Q, G = (torch.randn((20, 4, 64), device=dev).half() for _ in "QG")
    K, V = (torch.randn((900, 2, 64), device=dev).half() for _ in "KV")
    O, lse = gpu.cross_forward(plan, Q, K, V)
    lib, dQ, dK, dV = dense._lib(), torch.empty_like(Q), torch.empty_like(K), torch.empty_like(K)
    n, m = plan._forward_bytes, plan._backward_bytes
    assert n and m
    room = torch.zeros(max(n, m) + Q.numel() * 2 + K.numel() * 2, dtype=torch.uint8, device=dev)
    assert room.data_ptr() % 256 == 0

    def forward(q=Q.data_ptr(), k=K.data_ptr(), v=V.data_ptr()):
        return lib.f3s_cross_forward(plan.handle, q, k, v, 0, O.data_ptr(), lse.data_ptr(), 0.125,
                                     room.data_ptr(), n, None)

    def backward(q=Q.data_ptr(), k=K.data_ptr(), v=V.data_ptr(), o=O.data_ptr(), g=G.data_ptr(),
                 s=lse.data_ptr()):
        return lib.f3s_cross_backward(plan.handle, q, k, v, 0, o, g, s, dQ.data_ptr(),
                                      dK.data_ptr(), dV.data_ptr(), 0.125, room.data_ptr(), m,
                                      None)

    for inside in (room.data_ptr(), room.data_ptr() + 256):
        for name in "qkv":
            assert forward(**{name: inside}) == INVALID, name
        for name in "qkvogs":
            assert backward(**{name: inside}) == INVALID, name
    # right behind it
    room[n: n + Q.numel() * 2] = Q.flatten().view(torch.uint8)
    assert forward(q=room.data_ptr() + n) == 0
    room[m: m + Q.numel() * 2] = Q.flatten().view(torch.uint8)
    assert backward(q=room.data_ptr() + m) == 0
    torch.cuda.synchronize()
    want = gpu.cross_forward(plan, Q, K, V)
    assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
    for a, b in zip((dQ, dK, dV), gpu.cross_backward(plan, Q, K, V, O, G, lse)):
        assert torch.equal(a, b) and math.isfinite(float(a.float().sum()))


@no_gpu
@pytest.mark.parametrize("over", [
    dict(v=A), dict(v=A + 256), dict(k_exp=A), dict(v_exp=2 * A + 16384 - 16),
    dict(v_exp=3 * A), dict(k_exp=4 * A + 16),
])
def test_cache_whose_parts_overlap_is_not_written(lib, over):
    """(It may be read: K and V may be the same rows.)"""
    assert _write(lib, _cache(**over)) == INVALID
    assert _read(lib, _cache(**over)) == HIP
    assert _attend(lib, _cache(**over)) == HIP
    assert _write(lib, _cache(v=A + 16384, k_exp=4 * A - 256)) == HIP      # side by side


@no_gpu
def test_one_place_for_keys_and_values_takes_the_same_rows(lib):
    one = _cache(v=A, v_exp=3 * A)
    assert _write(lib, one, K=5 * A, V=5 * A) == HIP
    assert _write(lib, one) == INVALID
    assert _write(lib, _cache(v=A), K=5 * A, V=5 * A) == INVALID      # (powers apart)
    assert _write(lib, _cache(v=A, k_exp=A + 64, v_exp=A + 64), K=5 * A, V=5 * A) == INVALID


@pytest.mark.gpu
def test_rows_that_are_keys_and_values(gpu):
    dev = torch.device("cuda:0")
    two, one = gpu.Cache.empty(6, 16, 2, 64), gpu.Cache.empty(6, 16, 2, 64)
    one = gpu.Cache(one.k, one.k, one.k_exp, one.k_exp)
    X = torch.randn((2, 40, 2, 64), device=dev).bfloat16()
    table = torch.tensor([[0, 2, 4], [5, 3, 1]], dtype=torch.int32, device=dev)
    lens = torch.tensor([40, 33], dtype=torch.int32, device=dev)
    Q = torch.randn((2, 3, 6, 64), device=dev).bfloat16()
    results = []
    for cache in (two, one):
        gpu.cache_write(cache, X, X, table, lens)
        results.append(gpu.cache_attend(cache, Q, table, lens)
                       + gpu.cache_read(cache, table, lens, 40, torch.bfloat16))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    with pytest.raises(gpu.F3SError):
        gpu.cache_write(one, X, X.clone(), table, lens)
