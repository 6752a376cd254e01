"""The C calls of eb_train.h on the host: bad arguments are rejected with the documented
codes before a device is touched, and calls without work succeed.

No call here reaches a kernel launch.
"""
import pytest

from paper_2512_05831_amd import eb, experts as ex, train
from test_experts_host import FAKE, I, U, code_of

F32, F16, BF16, FP8 = eb.EB_F32, eb.EB_F16, eb.EB_BF16, ex.EB_FP8
HUGE = (1 << 30) + 1


def caller(f, **defaults):
    return lambda **kw: f(**{**defaults, **kw})


norm = caller(train.eb_layer_norm, rows=4, cols=100, x_ptr=FAKE, dtype=F32, ldx=100, weight_ptr=None, bias_ptr=None, eps=1e-5, out_type=F32,
              y_ptr=FAKE, ldy=100, y_scales_ptr=None, ldys=0, kept_ptr=None, ldk=0, kept_scales_ptr=None, ldks=0, mean_ptr=None, rstd_ptr=None,
              stream_ptr=None)
fp8_y = dict(out_type=FP8, ldy=112, y_scales_ptr=FAKE, ldys=4)
kept = dict(kept_ptr=FAKE, ldk=112, kept_scales_ptr=FAKE, ldks=4)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), I), (dict(cols=0), I), (dict(dtype=FP8), I), (dict(dtype=-1), I), (dict(out_type=4), I), (dict(eps=-1e-9), I),
    (dict(eps=float("nan")), I), (dict(x_ptr=None), I), (dict(y_ptr=None), I), (dict(ldx=99), I), (dict(ldy=99), I), (dict(x_ptr=FAKE + 2), I),
    (dict(dtype=F16, x_ptr=FAKE + 1), I), (dict(y_ptr=FAKE + 2), I), (dict(fp8_y, ldys=3), I), (dict(fp8_y, y_scales_ptr=None), I),
    (dict(fp8_y, ldy=104), I), (dict(fp8_y, y_ptr=FAKE + 8), I), (dict(kept, ldk=96), I), (dict(kept, ldk=104), I), (dict(kept, ldks=3), I),
    (dict(kept, kept_scales_ptr=None), I), (dict(kept, kept_ptr=FAKE + 4), I), (dict(cols=HUGE, ldx=HUGE, ldy=HUGE), U),
    (dict(rows=1 << 40, ldx=1 << 40), U), (dict(rows=1 << 27), U), (dict(fp8_y, ldys=1 << 62), U)])
def test_layer_norm_rejects(kw, code):
    assert code_of(norm, **kw) == code


norm_back = caller(train.eb_layer_norm_backward, rows=4, cols=100, dy_ptr=FAKE, dy_type=F32, lddy=100, x_ptr=FAKE, x_type=F32, ldx=100,
                   x_scales_ptr=None, ldxs=0, mean_ptr=FAKE, rstd_ptr=FAKE, weight_ptr=None, dx_ptr=FAKE, lddx=100, dweight_ptr=FAKE,
                   dbias_ptr=FAKE, workspace_ptr=FAKE, workspace_bytes=1 << 30, stream_ptr=None)
fp8_x = dict(x_type=FP8, ldx=112, x_scales_ptr=FAKE, ldxs=4, mean_ptr=None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), I), (dict(cols=0), I), (dict(dy_type=FP8), I), (dict(x_type=4), I), (dict(dy_ptr=None), I), (dict(x_ptr=None), I),
    (dict(dx_ptr=None), I), (dict(rstd_ptr=None), I), (dict(mean_ptr=None), I), (dict(fp8_x, mean_ptr=FAKE), I), (dict(fp8_x, ldxs=3), I),
    (dict(fp8_x, x_scales_ptr=None), I), (dict(fp8_x, ldx=104), I), (dict(lddy=99), I), (dict(lddx=99), I), (dict(ldx=99), I), (dict(dx_ptr=FAKE + 1), I),
    (dict(workspace_ptr=None), I), (dict(workspace_ptr=FAKE + 8), I), (dict(workspace_bytes=100), I), (dict(dweight_ptr=None, workspace_ptr=None), I),
    (dict(cols=HUGE, ldx=HUGE, lddy=HUGE, lddx=HUGE), U), (dict(rows=1 << 24), U)])
def test_layer_norm_backward_rejects(kw, code):
    assert code_of(norm_back, **kw) == code


def test_layer_norm_without_work():
    norm(rows=0, x_ptr=None, y_ptr=None)
    norm_back(rows=0, dy_ptr=None, x_ptr=None, dx_ptr=None, rstd_ptr=None, mean_ptr=None, dweight_ptr=None, dbias_ptr=None, workspace_ptr=None)
    w = train.eb_layer_norm_backward_workspace
    assert w(0, 100) == 0 and w(1, 100) >= 800 and w(1 << 20, 100) <= 1024 * 800 and w(100, 1 << 20) >= 8 << 20
    for bad, code in (((-1, 5), I), ((1, 0), I), ((1, HUGE), U), ((1 << 24, 4), U)):
        assert code_of(w, rows=bad[0], cols=bad[1]) == code
    assert train.library().eb_layer_norm_backward_workspace(1, 1, None) == I


act = caller(train.eb_activation, rows=4, cols=100, act=ex.EB_ACT_SILU_GATE, v_ptr=FAKE, v_type=F32, ldv=200, v_scales_ptr=None, ldvs=0,
             out_type=F32, h_ptr=FAKE, ldh=100, h_scales_ptr=None, ldhs=0, stream_ptr=None)
act_back = caller(train.eb_activation_backward, rows=4, cols=100, act=ex.EB_ACT_SILU_GATE, dh_ptr=FAKE, dh_type=F32, lddh=100, v_ptr=FAKE,
                  v_type=F32, ldv=200, v_scales_ptr=None, ldvs=0, out_type=F32, dv_ptr=FAKE, lddv=200, dv_scales_ptr=None, lddvs=0, stream_ptr=None)
fp8_v = dict(v_type=FP8, ldv=208, v_scales_ptr=FAKE, ldvs=4)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), I), (dict(cols=0), I), (dict(act=ex.EB_ACT_NONE), I), (dict(act=3), I), (dict(act=-1), I), (dict(v_type=4), I), (dict(out_type=-1), I),
    (dict(v_ptr=None), I), (dict(ldv=199), I), (dict(v_ptr=FAKE + 1), I), (dict(fp8_v, ldvs=3), I), (dict(fp8_v, v_scales_ptr=None), I),
    (dict(fp8_v, ldv=200), I), (dict(fp8_v, v_ptr=FAKE + 8), I), (dict(cols=1 << 30, ldv=1 << 31), U), (dict(rows=1 << 60), U)])
@pytest.mark.parametrize("f", [act, act_back])
def test_activation_rejects(f, kw, code):
    assert code_of(f, **kw) == code


def test_activation_rejects_outputs():
    for kw in (dict(h_ptr=None), dict(ldh=99), dict(h_ptr=FAKE + 2), dict(out_type=FP8, ldh=112), dict(out_type=FP8, ldh=104, h_scales_ptr=FAKE, ldhs=4),
               dict(out_type=FP8, ldh=112, h_scales_ptr=FAKE, ldhs=3)):
        assert code_of(act, **kw) == I
    for kw in (dict(dv_ptr=None), dict(lddv=199), dict(dh_ptr=None), dict(lddh=99), dict(dh_type=FP8), dict(out_type=FP8, lddv=208),
               dict(out_type=FP8, lddv=200, dv_scales_ptr=FAKE, lddvs=4)):
        assert code_of(act_back, **kw) == I
    assert code_of(act, rows=1 << 28, cols=1 << 20, ldv=1 << 21, ldh=1 << 20) == U
    act(rows=0, v_ptr=None, h_ptr=None)
    act_back(rows=0, v_ptr=None, dh_ptr=None, dv_ptr=None)


dispatch = caller(train.eb_dispatch, M=4, cols=100, x_ptr=FAKE, dtype=F32, ldx=100, x_rows=3, x_scales_ptr=None, ldxs=0, tokens_ptr=FAKE,
                  out_ptr=FAKE, ldo=100, out_scales_ptr=None, ldos=0, stream_ptr=None)
fp8_rows = dict(dtype=FP8, ldx=112, x_scales_ptr=FAKE, ldxs=3, ldo=112, out_scales_ptr=FAKE, ldos=4)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), I), (dict(cols=0), I), (dict(x_rows=-1), I), (dict(dtype=4), I), (dict(x_ptr=None), I), (dict(out_ptr=None), I),
    (dict(tokens_ptr=None), I), (dict(ldx=99), I), (dict(ldo=99), I), (dict(x_ptr=FAKE + 2), I), (dict(fp8_rows, ldxs=2), I),
    (dict(fp8_rows, ldos=3), I), (dict(fp8_rows, out_scales_ptr=None), I), (dict(fp8_rows, ldo=104), I), (dict(M=1 << 31), U),
    (dict(cols=HUGE, ldx=HUGE, ldo=HUGE), U)])
def test_dispatch_rejects(kw, code):
    assert code_of(dispatch, **kw) == code


combine = caller(train.eb_combine, N=4, K=2, cols=100, y_ptr=FAKE, y_type=F32, ldy=100, y_rows=8, slots_ptr=FAKE, weights_ptr=None, out_type=F32,
                 out_ptr=FAKE, ldo=100, stream_ptr=None)
combine_back = caller(train.eb_combine_backward, N=4, K=2, cols=100, dout_ptr=FAKE, dout_type=F32, lddo=100, y_ptr=FAKE, y_type=F32, ldy=100,
                      y_rows=8, slots_ptr=FAKE, weights_ptr=None, dy_type=F32, dy_ptr=FAKE, lddy=100, dy_scales_ptr=None, lddys=0,
                      dweights_ptr=FAKE, stream_ptr=None)


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), I), (dict(K=0), I), (dict(cols=0), I), (dict(y_rows=-1), I), (dict(y_type=FP8), I), (dict(y_ptr=None), I), (dict(slots_ptr=None), I),
    (dict(ldy=99), I), (dict(y_ptr=FAKE + 2), I), (dict(K=65), U), (dict(N=1 << 30), U), (dict(N=1 << 31), U), (dict(cols=HUGE, ldy=HUGE), U)])
@pytest.mark.parametrize("f", [combine, combine_back])
def test_combine_rejects(f, kw, code):
    assert code_of(f, **kw) == code


def test_combine_rejects_outputs():
    for kw in (dict(out_type=FP8), dict(out_ptr=None), dict(ldo=99), dict(out_ptr=FAKE + 1)):
        assert code_of(combine, **kw) == I
    for kw in (dict(dout_type=FP8), dict(dout_ptr=None), dict(lddo=99), dict(dy_type=4), dict(lddy=99), dict(dy_type=FP8, lddy=112),
               dict(dy_type=FP8, lddy=112, dy_scales_ptr=FAKE, lddys=7), dict(dy_ptr=FAKE + 2)):
        assert code_of(combine_back, **kw) == I


def test_sorting_without_work():
    dispatch(M=0, out_ptr=None, tokens_ptr=None)
    dispatch(x_rows=0, x_ptr=None)
    combine(N=0, out_ptr=None, slots_ptr=None)
    combine_back(N=0, dout_ptr=None, slots_ptr=None)
    combine_back(dy_ptr=None, dweights_ptr=None, y_ptr=None)


gradient = caller(train.eb_weight_gradient, M=4, E=2, N=100, K=60, dy_ptr=FAKE, dy_type=BF16, lddy=100, dy_scales_ptr=None, lddys=0, x_ptr=FAKE,
                  x_type=F16, ldx=60, x_rows=4, x_scales_ptr=None, ldxs=0, tokens_ptr=None, offsets_ptr=FAKE, out_type=F32, accumulate=0,
                  dw_ptr=FAKE, lddw=60, workspace_ptr=None, workspace_bytes=0, stream_ptr=None)
fp8_in = dict(x_type=FP8, ldx=64, x_scales_ptr=FAKE, ldxs=4)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), I), (dict(E=0), I), (dict(N=0), I), (dict(K=0), I), (dict(dy_type=F32), I), (dict(x_type=F32), I), (dict(x_type=4), I),
    (dict(out_type=FP8), I), (dict(x_rows=-1), I), (dict(x_rows=3), I), (dict(accumulate=2), I), (dict(offsets_ptr=None), I), (dict(dy_ptr=None), I),
    (dict(x_ptr=None), I), (dict(dw_ptr=None), I), (dict(lddy=99), I), (dict(ldx=59), I), (dict(lddw=59), I), (dict(dy_ptr=FAKE + 1), I),
    (dict(fp8_in, ldxs=3), I), (dict(fp8_in, x_scales_ptr=None), I), (dict(fp8_in, ldx=72), I), (dict(M=1 << 31, x_rows=1 << 31), U),
    (dict(E=HUGE), U), (dict(N=HUGE, lddy=HUGE), U), (dict(K=HUGE, ldx=HUGE, lddw=HUGE), U), (dict(E=1 << 28, lddw=60), U),
    (dict(M=20000, E=1, x_rows=20000), I), (dict(M=20000, E=1, x_rows=20000, workspace_ptr=FAKE, workspace_bytes=100), I),
    (dict(M=20000, E=1, x_rows=20000, workspace_ptr=FAKE + 4, workspace_bytes=1 << 40), I)])
def test_weight_gradient_rejects(kw, code):
    assert code_of(gradient, **kw) == code


def test_weight_gradient_workspace():
    w = train.eb_weight_gradient_workspace
    assert w(65536, 64, 2048, 1024) == 0 and w(0, 1, 64, 64) == 0 and w(100, 1, 128, 128) == 0
    assert w(1 << 20, 1, 128, 128) >= 2 * 4 * 128 * 128
    for bad, code in (((-1, 1, 1, 1), I), ((1, 0, 1, 1), I), ((1, 1, 0, 1), I), ((1, 1, 1, 0), I), ((1 << 31, 1, 1, 1), U), ((1, 1, HUGE, 1), U),
                      ((1, 1 << 30, 1 << 30, 1 << 30), U)):
        assert code_of(w, M=bad[0], E=bad[1], N=bad[2], K=bad[3]) == code
    assert train.library().eb_weight_gradient_workspace(1, 1, 1, 1, None) == I
