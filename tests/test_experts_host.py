"""The experts' C calls on the host: bad arguments are rejected with the documented
codes before a device is touched, and calls without work succeed.

No call here reaches a kernel launch.
"""
import pytest

from paper_2512_05831_amd import eb, experts as ex

FAKE = 0x7F0000000000  # 16-byte aligned, never dereferenced by these tests
I, U = eb.EB_ERR_INVALID, eb.EB_ERR_UNSUPPORTED


def code_of(f, **kw):
    with pytest.raises(eb.EbError) as e:
        f(**kw)
    assert str(e.value) and eb.eb_last_error()
    return e.value.code


def route(**kw):
    a = dict(N=4, E=32, K=4, scores_ptr=FAKE, dtype=eb.EB_F32, ld=32, bias_ptr=None, mode=ex.EB_SOFTMAX, groups=1, top_groups=1,
             scale=1.0, shard_lo=0, shard_hi=32, ids_ptr=FAKE, weights_ptr=FAKE, offsets_ptr=FAKE, tokens_ptr=FAKE, slots_ptr=FAKE,
             workspace_ptr=FAKE, workspace_bytes=1 << 30, stream_ptr=None)
    a.update(kw)
    return ex.eb_route_experts(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), I), (dict(E=0, K=1), I), (dict(K=0), I), (dict(K=33), I), (dict(dtype=3), I), (dict(mode=2), I), (dict(mode=0x400), I),
    (dict(ld=31), I), (dict(groups=0), I), (dict(groups=5), I), (dict(top_groups=2), I), (dict(top_groups=0), I),
    (dict(mode=ex.EB_GROUP_PAIR, groups=32), I), (dict(shard_lo=-1), I), (dict(shard_lo=9, shard_hi=8), I), (dict(shard_hi=33), I),
    (dict(scores_ptr=None), I), (dict(ids_ptr=None), I), (dict(weights_ptr=None), I), (dict(tokens_ptr=None), I), (dict(slots_ptr=None), I),
    (dict(offsets_ptr=None), I), (dict(E=1025, ld=1025, shard_hi=1025), U), (dict(E=1024, ld=1024, K=65), U),
    (dict(E=66, ld=66, groups=33, shard_hi=66), U), (dict(N=1 << 30), U),
    (dict(N=5000, workspace_ptr=None), I), (dict(N=5000, workspace_bytes=100), I), (dict(N=5000, workspace_ptr=FAKE + 2), I)])
def test_route_rejects(kw, code):
    assert code_of(route, **kw) == code


def test_route_without_work():
    route(N=0, offsets_ptr=None, tokens_ptr=None, slots_ptr=None, scores_ptr=None, ids_ptr=None, weights_ptr=None)


def test_route_workspace():
    w = ex.eb_route_experts_workspace
    assert w(64, 256, 8, 0, 256) == 0
    assert w(16384, 256, 8, 0, 256) >= 256 * 4
    assert w(16384, 256, 8, 128, 160) < w(16384, 256, 8, 0, 256)
    for bad in ((-1, 8, 1, 0, 8), (1, 8, 0, 0, 8), (1, 8, 9, 0, 8), (1, 8, 1, -1, 8), (1, 8, 1, 5, 4), (1, 8, 1, 0, 9)):
        with pytest.raises(eb.EbError) as e:
            w(*bad)
        assert e.value.code == I
    with pytest.raises(eb.EbError) as e:
        w(1, 1025, 1, 0, 8)
    assert e.value.code == U


def quantize(**kw):
    a = dict(matrices=1, rows=4, cols=100, x_ptr=FAKE, dtype=eb.EB_F32, ldx=100, block_rows=1, q_ptr=FAKE, ldq=112, scales_ptr=FAKE, lds=4,
             stream_ptr=None)
    a.update(kw)
    return ex.eb_quantize_fp8(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(matrices=-1), I), (dict(rows=-1), I), (dict(cols=0), I), (dict(dtype=3), I), (dict(block_rows=64), I), (dict(x_ptr=None), I),
    (dict(q_ptr=None), I), (dict(scales_ptr=None), I), (dict(ldx=99), I), (dict(ldq=96), I), (dict(ldq=104), I), (dict(q_ptr=FAKE + 8), I),
    (dict(lds=3), I), (dict(rows=1 << 31, lds=1 << 31), U), (dict(rows=1 << 30, cols=1 << 20, ldx=1 << 20, ldq=1 << 20, lds=1 << 30), U)])
def test_quantize_rejects(kw, code):
    assert code_of(quantize, **kw) == code


def test_quantize_without_work():
    quantize(rows=0, x_ptr=None, q_ptr=None, scales_ptr=None)
    quantize(matrices=0)


def product(**kw):
    a = dict(M=4, E=2, N=256, K=128, x_ptr=FAKE, ldx=128, x_rows=4, x_scales_ptr=FAKE, ldxs=4, tokens_ptr=None, w_ptr=FAKE, ldw=128,
             w_scales_ptr=FAKE, offsets_ptr=FAKE, bias_ptr=None, act=ex.EB_ACT_NONE, out_type=eb.EB_BF16, out_ptr=FAKE, ldo=256,
             out_scales_ptr=None, ldos=0, stream_ptr=None)
    a.update(kw)
    return ex.eb_expert_product(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), I), (dict(E=0), I), (dict(N=0), I), (dict(K=0), I), (dict(x_rows=-1), I), (dict(act=3), I), (dict(out_type=4), I),
    (dict(act=ex.EB_ACT_SILU_GATE, N=255), I), (dict(offsets_ptr=None), I), (dict(x_ptr=None), I), (dict(x_scales_ptr=None), I),
    (dict(w_ptr=None), I), (dict(w_scales_ptr=None), I), (dict(out_ptr=None), I), (dict(out_type=ex.EB_FP8), I), (dict(x_rows=3, ldxs=3), I),
    (dict(ldx=112), I), (dict(ldx=136), I), (dict(ldw=112), I), (dict(ldw=136), I), (dict(x_ptr=FAKE + 4), I), (dict(w_ptr=FAKE + 4), I),
    (dict(ldo=255), I), (dict(ldxs=3), I), (dict(out_ptr=FAKE + 1), I), (dict(out_type=ex.EB_FP8, out_scales_ptr=FAKE, ldos=3), I),
    (dict(out_type=ex.EB_FP8, out_scales_ptr=FAKE, ldos=4, ldo=264), I), (dict(out_type=ex.EB_FP8, out_scales_ptr=FAKE, ldos=4, out_ptr=FAKE + 4), I),
    (dict(M=1 << 31, x_rows=1 << 31, ldxs=1 << 31), U), (dict(N=(1 << 30) + 1, ldo=1 << 31), U), (dict(ldo=1 << 62), U)])
def test_product_rejects(kw, code):
    assert code_of(product, **kw) == code


def test_product_without_work():
    product(M=0, x_rows=0, ldxs=0, x_ptr=None, out_ptr=None)


def test_more_than_one_launch_holds():
    """A launch has fewer than 2^32 threads."""
    assert code_of(route, N=1 << 28, E=1, K=1, ld=1, shard_hi=1, workspace_bytes=1 << 40) == U
    assert code_of(quantize, rows=1 << 28, cols=1, ldx=1, ldq=16, lds=1 << 28) == U
    assert code_of(quantize, matrices=1 << 24, rows=1, cols=1, ldx=1, ldq=16, block_rows=128) == U
    assert code_of(product, M=1 << 28, E=1, N=1 << 20, ldo=1 << 20, x_rows=1 << 28, ldxs=1 << 28) == U
