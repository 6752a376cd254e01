"""What the tests of eb_train.h share: matrices in 8 bits, and how far roundings may be off."""
import torch

from paper_2512_05831_amd import experts as ex

U = 2.0 ** -24  # a rounding to fp32, relative
HALF_STEP = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
FP8 = torch.float8_e4m3fn
WIDE = [torch.float32, torch.float16, torch.bfloat16]


def generator(device, seed):
    return torch.Generator(device=device).manual_seed(seed)


def held(q, s):
    """The values of an 8-bit matrix, in 64 bits."""
    return q.double() * s.double().repeat_interleave(128, 1)[:, :q.shape[1]]


def eight(x):
    """(values, scales) of a matrix, or (matrix, None) as it is."""
    return ex.quantize_fp8(x)


def as_type(x, dtype):
    """(stored, scales or None, its values in 64 bits)."""
    if dtype == FP8:
        q, s = ex.quantize_fp8(x)
        return q, s, held(q, s)
    x = x.to(dtype)
    return x, None, x.double()


def rounded(err, want, dtype):
    """A bound on the error after one more rounding, of values known to err."""
    return err + (want.abs() + err) * HALF_STEP[dtype] + LEAST[dtype]


def check(got, want, err, dtype):
    off = (got.double() - want).abs()
    bound = rounded(err * (1 + 2.0 ** -10), want, dtype)
    assert got.dtype == dtype and got.shape == want.shape
    bad = ~(off <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((off / bound)[bad].max()):.3g} times the bound at {bad.nonzero()[0].tolist()}"


def check8(q, s, want, err):
    """An 8-bit matrix against values known to err: the scale within their error, its own rounding and the
    quotients' (2 ulp of fp32, half a step of e4m3: 2^-4 of a normal, 2^-10 scales of a subnormal)."""
    rows, cols = want.shape
    pad = lambda v: torch.nn.functional.pad(v, (0, -cols % 128)).view(rows, -(-cols // 128), 128).amax(2)  # noqa: E731
    scale = (pad(want.abs()) / 448).clamp(min=2.0 ** -126)
    assert q.dtype == FP8 and q.shape == want.shape and s.shape == scale.shape
    assert ((s.double() - scale).abs() <= pad(err.expand_as(want)) / 448 * (1 + 2.0 ** -10) + scale * 2 * U).all()
    each = s.double().repeat_interleave(128, 1)[:, :cols]
    off = (held(q, s) - want).abs()
    bound = err * (1 + 2.0 ** -3) + want.abs() * 2.0 ** -4 * (1 + 2.0 ** -10) + each * 2.0 ** -10 + each * 448 * 4 * U
    assert (off <= bound).all(), float((off / bound).max())
    if q.stride(0) > cols and rows:  # zeros up to the next multiple of 16
        whole = q.as_strided((rows, cols + 15 & -16), (q.stride(0), 1)).contiguous().view(torch.uint8)
        assert (whole[:, cols:] == 0).all()


def route_of(N, E, top, device, seed, shards=1):
    scores = torch.randn(N, E, generator=generator(device, seed), device=device)
    return ex.route(scores, top, shard_hi=-(-E // shards))


EVERY_REMAINDER = [*range(2, 25), *range(121, 137), *range(506, 518)]


def among_nans(x):
    """The same values as part of a matrix that holds NaN around them, also behind the last row."""
    room = torch.full((x.shape[0] + 2, x.shape[1] + 9), float("nan"), dtype=x.dtype, device=x.device)
    room[1:-1, 3:-6] = x
    return room[1:-1, 3:-6]
