"""Arguments that the operators around the scan refuse, on the host and before any launch (no GPU needed)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2512_07884_amd import binding
    return binding.load_library()


OK, NULL, SHAPE, DTYPE, ALIGN, UNSUPPORTED = range(6)
p = ctypes.c_void_p(0x1000)              # aligned, never dereferenced: every call below fails validation
odd = ctypes.c_void_p(0x1008)


def test_products_refuse_on_the_host(lib):
    dims = (2, 16, 8, 5, 7)
    big = 1 << 40
    for fwd, bwd, size in ((lambda *a: lib.gspn_proxy_project_fused(*a[:3], None, *a[3:]), lib.gspn_proxy_project_fused_bwd, lib.gspn_proxy_project_fused_bwd_bytes),
                           (lib.gspn_gated_project, lib.gspn_gated_project_bwd, lib.gspn_gated_project_bwd_bytes)):
        for hole in (0, 1, 3):
            args = [p, p, p, p]
            args[hole] = None
            assert fwd(*args, *dims, 1, 1, None) == NULL
        for bad in ((0, 16, 8, 5, 7), (2, 0, 8, 5, 7), (2, 16, 0, 5, 7), (2, 16, 8, 0, 7), (2, 16, 8, 5, -1)):
            assert fwd(p, p, p, p, *bad, 1, 1, None) == SHAPE and size(*bad, 1, 1) == 0
            assert bwd(p, p, p, p, p, p, p, p, big, *bad, 1, 1, None) == SHAPE
        assert fwd(p, p, p, p, *dims, 1, 3, None) == DTYPE and size(*dims, 1, 3) == 0
        assert fwd(p, p, p, p, *dims, 4, 1, None) == UNSUPPORTED and fwd(p, p, p, p, *dims, -1, 1, None) == UNSUPPORTED and size(*dims, 4, 1) == 0
        assert fwd(p, p, p, p, 2, 16, 8, 5, 20000, 1, 1, None) == UNSUPPORTED
        assert fwd(p, p, p, p, 1, 1 << 20, 1 << 12, 5, 7, 1, 1, None) == UNSUPPORTED          # a matrix of 2^32 values
        assert fwd(p, p, p, p, 1 << 20, 16, 8, 256, 256, 1, 1, None) == UNSUPPORTED           # more tiles than a launch counts
        for hole in range(4):
            args = [p, p, p, p]
            args[hole] = odd
            assert fwd(*args, *dims, 1, 1, None) == ALIGN
        need = size(*dims, 1, 1)
        assert need > 0 and need % 256 == 0
        assert bwd(p, p, p, p, p, p, p, p, need - 1, *dims, 1, 1, None) == SHAPE
        assert bwd(p, p, p, p, p, p, p, None, big, *dims, 1, 1, None) == NULL
        assert bwd(p, p, p, p, None, None, None, p, big, *dims, 1, 1, None) == NULL           # no gradient asked for
        for hole in (0, 1, 2):
            args = [p] * 8
            args[hole] = None
            assert bwd(*args, big, *dims, 1, 1, None) == NULL
        for hole in range(8):
            args = [p] * 8
            args[hole] = odd
            assert bwd(*args, big, *dims, 1, 1, None) == ALIGN
    assert lib.gspn_proxy_project_fused(p, p, p, odd, p, *dims, 1, 1, None) == ALIGN           # the residual


def test_sizes_that_no_launch_counts(lib):
    """Refused before anything is launched, the backward call's other launches included; what is just below has a workspace's size."""
    def back(*d, act=1):
        return lib.gspn_proxy_project_fused_bwd(p, p, p, p, p, p, p, p, 1 << 62, *d, act, 1, None)
    for act, sizes in ((1, [(1 << 24, 8, 8, 5, 8), (1 << 20, 1024, 8, 1, 1), (1, 1 << 30, 1, 1, 1)]), (0, [(1 << 22, 8, 32, 1, 1)])):
        for d in sizes:
            assert back(*d, act=act) == UNSUPPORTED and lib.gspn_proxy_project_fused_bwd_bytes(*d, act, 1) == 0, d
    assert lib.gspn_proxy_project_fused_bwd_bytes(1 << 18, 1024, 8, 1, 1, 1, 1) > 0
    assert lib.gspn_proxy_project_fused_bwd_bytes(1 << 22, 8, 8, 5, 8, 1, 1) > 0
    assert lib.gspn_proxy_project_fused(p, p, p, p, p, 1 << 24, 8, 8, 5, 8, 1, 1, None) == UNSUPPORTED
    assert lib.gspn_proxy_project_fused(p, p, p, p, p, 1, 1 << 30, 1, 1, 1, 1, 1, None) == UNSUPPORTED
    tokens = (64, 64, 64, 8, 1, 1, 1 << 24)
    assert lib.gspn_cross_attention(p, p, p, p, p, p, p, 1 << 62, *tokens, 0.3, 1, None) == UNSUPPORTED


def test_refusals_come_before_the_workspace(lib):
    """A backward call without a workspace that is refused anyway says why."""
    assert lib.gspn_gated_project_bwd(p, p, p, p, p, p, p, None, 0, 2, 16, 8, 5, 20000, 1, 1, None) == UNSUPPORTED
    assert lib.gspn_cross_attention_bwd(*(p,) * 10, None, 0, 2, 4, 2, 12, 5, 7, 33, 0.25, 1, None) == UNSUPPORTED


def test_attention_refuses_on_the_host(lib):
    dims = (2, 4, 2, 16, 5, 7, 33)
    big = 1 << 40
    f = lambda *d, scale=0.25, dtype=1, a=(p, p, p, p, p, p, p): lib.gspn_cross_attention(*a, big, *d, scale, dtype, None)
    b = lambda *d, scale=0.25, dtype=1, a=(p,) * 11, n=big: lib.gspn_cross_attention_bwd(*a, n, *d, scale, dtype, None)
    for i in range(7):
        bad = list(dims)
        bad[i] = 0
        assert f(*bad) == SHAPE and b(*bad) == SHAPE and lib.gspn_cross_attention_bwd_bytes(*bad, 1) == 0 and lib.gspn_cross_attention_bytes(*bad, 1) == 0
    assert f(2, 4, 3, 16, 5, 7, 33) == SHAPE                                                   # heads that do not share evenly
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert f(*dims, scale=scale) == SHAPE and b(*dims, scale=scale) == SHAPE
    assert f(*dims, dtype=3) == DTYPE and b(*dims, dtype=-1) == DTYPE
    for bad in ((2, 4, 2, 12, 5, 7, 33), (2, 4, 2, 136, 5, 7, 33), (2, 4, 2, 16, 20000, 7, 33), (2, 4, 2, 16, 5, 7, (1 << 24) + 1), (1 << 20, 64, 64, 16, 128, 128, 3)):
        assert f(*bad) == UNSUPPORTED and b(*bad) == UNSUPPORTED, bad
    for hole in (0, 1, 2, 4):
        a = [p] * 7
        a[hole] = None
        assert f(*dims, a=a) == NULL
    for hole in (0, 1, 2, 4, 5, 6):
        a = [p] * 7
        a[hole] = odd
        assert f(*dims, a=a) == ALIGN
    for hole in (0, 1, 2, 3, 5, 6, 10):
        a = [p] * 11
        a[hole] = None
        assert b(*dims, a=a) == NULL
    assert b(*dims, a=[p] * 7 + [None] * 3 + [p]) == NULL
    for hole in (0, 1, 2, 3, 5, 6, 7, 8, 9, 10):
        a = [p] * 11
        a[hole] = odd
        assert b(*dims, a=a) == ALIGN
    assert b(*dims, n=lib.gspn_cross_attention_bwd_bytes(*dims, 1) - 1) == SHAPE
    few = (1, 4, 2, 64, 1, 1, 4096)
    need = lib.gspn_cross_attention_bytes(*few, 1)
    assert need > 0 and lib.gspn_cross_attention(p, p, p, p, p, p, p, need - 1, *few, 0.125, 1, None) == SHAPE
    assert lib.gspn_cross_attention_bytes(2, 16, 16, 64, 128, 128, 77, 1) == 0                 # many positions: no stretches


def test_binding_refuses_what_does_not_fit():
    import paper_2512_07884_amd as G
    z = torch.zeros
    with pytest.raises(ValueError):                                                            # host tensors
        G.gspn_proxy_project_fused(z(1, 4, 2, 2), z(3, 4), z(1, 3, 2, 2))
    with pytest.raises(ValueError):                                                            # three dimensions
        G.gspn_gated_project(z(4, 2, 2), z(6, 4), z(3, 2, 2))
    with pytest.raises(ValueError):                                                            # an odd number of rows
        G.gspn_gated_project(z(1, 4, 2, 2), z(5, 4), z(1, 2, 2, 2))
    with pytest.raises(ValueError):
        G.gspn_proxy_project_fused(z(1, 4, 2, 2), z(4), z(1, 3, 2, 2))
    for heads, kv in ((3, 3), (4, 3), (0, 1), (4, 0)):
        with pytest.raises(ValueError):
            G.gspn_cross_attention(z(1, 32, 2, 2), z(1, 5, 32), z(1, 5, 32), z(1, 32, 2, 2), heads=heads, kv_heads=kv)
    with pytest.raises(ValueError):
        G.gspn_cross_attention(z(1, 32, 2, 2), z(1, 5, 32), z(1, 5, 32), z(1, 32, 2, 2), heads=4)


def test_workspace_sizes_follow_the_call():
    import paper_2512_07884_amd as G
    from paper_2512_07884_amd import binding as b
    none = G.gspn_proxy_project_fused_bwd_bytes(2, 64, 96, 32, 32, G.GSPN_ACT_NONE, b.GSPN_BF16)
    silu = G.gspn_proxy_project_fused_bwd_bytes(2, 64, 96, 32, 32, G.GSPN_ACT_SILU, b.GSPN_BF16)
    assert silu - none >= 2 * 96 * 1024 * 2 - 65536                                            # the gradient at the product's result
    assert G.gspn_gated_project_bwd_bytes(2, 64, 96, 32, 32, G.GSPN_ACT_SILU, b.GSPN_BF16) >= 2 * 2 * 96 * 1024 * 2
    assert G.gspn_cross_attention_bwd_bytes(2, 4, 4, 32, 16, 16, 77, b.GSPN_BF16) >= 2 * 4 * 256 * 4
