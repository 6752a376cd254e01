"""Limits of the experts' C calls on the host: what lies past them is refused before a
device is touched.
"""
from paper_2512_05831_amd import eb, experts as ex
from test_experts_host import I, U, code_of, product, route


def test_product_refuses_experts_beyond_32_bit_steps():
    """The kernels walk the experts 64 at a time in 32 bits: within 64 of 2^31 that count would wrap, and a workgroup
    past the last tile would never end."""
    for E in ((1 << 30) + 1, (1 << 31) - 64, (1 << 31) - 1):
        assert code_of(product, E=E, ldo=256) == U
        assert code_of(product, E=E, N=16, ldo=16, out_type=ex.EB_FP8, out_scales_ptr=0x7F0000000000, ldos=4) == U
    product(E=1 << 30, M=0, x_rows=0, ldxs=0)
    assert eb.EB_ERR_UNSUPPORTED == U


def test_workspace_refuses_what_the_route_refuses():
    """More experts per token than eb_route_experts takes: no size for a call that cannot be made."""
    assert ex.eb_route_experts_workspace(1000, 1024, 64, 0, 1024) > 0
    for K in (65, 1024):
        assert code_of(route, N=1000, E=1024, ld=1024, K=K, shard_hi=1024) == U
        assert code_of(ex.eb_route_experts_workspace, N=1000, E=1024, K=K, shard_lo=0, shard_hi=1024) == U


def test_product_rejects_unknown_bits_of_act():
    for act in (ex.EB_EXACT_SUMS | 3, 0x200, ex.EB_EXACT_SUMS | 0x200, -1):
        assert code_of(product, act=act) == I
    assert code_of(product, act=ex.EB_EXACT_SUMS | ex.EB_ACT_SILU_GATE, N=255) == I
    product(act=ex.EB_EXACT_SUMS, M=0, x_rows=0, ldxs=0)
