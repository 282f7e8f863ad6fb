"""8-bit activation checkpoints: pins of the plain form on CPU, refusals, and bit-for-bit parity
of codes, scales and decoded values through the C ABI."""
import numpy as np
import pytest
import torch

import act8_reference as ref
import paper_1905_10988_b200 as nc

TYPES = {"f32": (nc.DTYPE_F32, torch.float32), "bf16": (nc.DTYPE_BF16, torch.bfloat16),
         "f16": (nc.DTYPE_F16, torch.float16)}


# ---- the plain form against hand-written values -------------------------------------------------

def test_unit_is_the_smallest_power_of_two_that_holds_the_largest_magnitude():
    for top, e in [(127.0, 0), (127.0001, 1), (1.0, -6), (1.984375, -6), (1.98438, -5),
                   (0.0, -118), (2.0 ** -130, -118), (2.0 ** 127 * 1.5, 121)]:
        x = np.zeros((1, 40))
        x[0, 3] = -top
        assert ref.scale_bytes(x).tolist() == [[e + 127, 127 - 118]]
    x = np.zeros((1, 33))
    x[0, 32] = np.inf
    assert ref.scale_bytes(x).tolist() == [[9, 255]]


def test_plain_codes_by_hand():
    x = np.float32([[127.0, -1.0, 0.5, 1.5, -2.5, 0.49, -0.2, 0.0, -0.0]])
    codes, scales = ref.encode(x)
    assert scales.tolist() == [[127]]
    # ties to even: 0.5 -> 0, 1.5 -> 2, -2.5 -> -2; a sign stays where the magnitude rounds to 0
    assert codes[0, :9].tolist() == [127, 129, 0, 2, 130, 0, 128, 0, 128]
    assert ref.decode(codes, scales, 9)[0].tolist() == [127, -1, 0, 2, -2, 0, 0, 0, 0]


def test_stream_bytes_follow_the_generator_of_the_oracle():
    import oracle
    got = ref.stream_bytes(0x123456789ABCDEF0, 7, 64, domain=6).view("<u4")
    want = oracle.stream_words(0x123456789ABCDEF0, 7, 6, 0, 16)
    assert np.array_equal(got, np.asarray(want, np.uint32))


def test_random_rounding_has_the_right_expectation_over_all_draws():
    # floor((Y + r) / 256) over the 256 draws: Y / 256 on average
    y = np.arange(0, 127 * 256 + 1, 37)
    m = (y[:, None] + np.arange(256)[None, :]) >> 8
    assert np.array_equal(m.sum(1), y) and m.max() == 127


def test_decoded_values_are_exact_in_bfloat16():
    codes = np.arange(256, dtype=np.uint8).reshape(8, 32)
    for s in (9, 60, 127, 200, 247):
        v = ref.decode(codes, np.full((8, 1), s, np.uint8), 32).astype(np.float32)
        assert np.array_equal(torch.from_numpy(v).bfloat16().float().numpy(), v)


def test_sizes():
    assert nc.nc_act8_code_bytes(3, 33) == 3 * 64 and nc.nc_act8_code_bytes(0, 5) == 0
    assert nc.nc_act8_scale_bytes(3, 33) == 16 and nc.nc_act8_scale_bytes(9, 33) == 32


def _status(call):
    with pytest.raises(nc.NatcompError) as err:
        call()
    return nc.status_string(err.value.status)


def _place():
    """Real device memory where there is some (2 MiB), a made-up aligned address elsewhere."""
    if torch.cuda.is_available():
        buf = torch.zeros(2 << 20, dtype=torch.uint8, device="cuda")
        return buf, buf.data_ptr()
    return None, 1 << 20


def test_refusals_need_no_gpu():
    keep, A = _place()
    s = 0                                  # the default stream

    def comp(x=A, dt=nc.DTYPE_BF16, r=4, c=40, ld=40, mode=0, codes=A, scales=A):
        return nc.nc_act8_compress(x, dt, r, c, ld, mode, 0, 0, codes, scales, stream=s)

    def back(codes=A, scales=A, r=4, c=40, out=A, dt=nc.DTYPE_BF16, ld=40):
        return nc.nc_act8_decompress(codes, scales, r, c, out, dt, ld, stream=s)

    for f in (comp, back):
        assert _status(lambda: f(dt=3)) == "NC_ERR_UNSUPPORTED"
        assert _status(lambda: f(ld=39)) == "NC_ERR_INVALID"
        assert _status(lambda: f(codes=None)) == "NC_ERR_INVALID"
        assert _status(lambda: f(scales=None)) == "NC_ERR_INVALID"
        assert _status(lambda: f(codes=A + 8)) == "NC_ERR_ALIGN"
        assert _status(lambda: f(scales=A + 4)) == "NC_ERR_ALIGN"
        assert _status(lambda: f(r=1 << 36, c=32, ld=32)) == "NC_ERR_TOO_LARGE"
        assert _status(lambda: f(r=1 << 63, c=1 << 63, ld=1 << 63)) == "NC_ERR_TOO_LARGE"
        f(r=0)
        f(c=0)
    assert _status(lambda: comp(x=None)) == "NC_ERR_INVALID"
    assert _status(lambda: comp(mode=2)) == "NC_ERR_INVALID"
    assert _status(lambda: comp(x=A + 1)) == "NC_ERR_ALIGN"
    assert _status(lambda: comp(x=A + 2, dt=nc.DTYPE_F32)) == "NC_ERR_ALIGN"
    assert _status(lambda: back(out=None)) == "NC_ERR_INVALID"
    assert _status(lambda: back(out=A + 1)) == "NC_ERR_ALIGN"
    del keep


# ---- GPU ------------------------------------------------------------------------------------

def matrix(rows, cols, ld, offset, kind, fill=None):
    """A (rows, cols) view with row stride ld that starts `offset` elements into its storage."""
    dt = TYPES[kind][1]
    store = torch.zeros(offset + rows * ld + 64, dtype=dt, device="cuda")
    v = store[offset:offset + rows * ld].view(rows, ld)[:, :cols] if rows * ld else \
        store[:0].view(rows, cols)
    if fill is not None:
        v.copy_(fill)
    return v


def special_rows(rng, rows, cols, kind):
    """Blocks of every loudness: zeros, subnormals, huge, single spikes, inf and NaN."""
    x = rng.standard_normal((rows, cols))
    lim = 60000.0 if kind == "f16" else 3.0e38
    p = ref.pitch_of(cols)
    for r in range(rows):
        for b in range(0, p, 32):
            pick = rng.integers(0, 10)
            blk = x[r, b:b + 32]
            if pick == 0:
                blk *= 0.0
            elif pick == 1:
                blk *= 2.0 ** rng.integers(-24, 15)
            elif pick == 2 and kind != "f16":
                blk *= 2.0 ** float(rng.integers(-140, 120))
            elif pick == 3:
                blk[:] = np.clip(blk * lim, -lim, lim)
            elif pick == 4:
                blk[rng.integers(0, blk.size)] = rng.choice([np.inf, -np.inf, np.nan])
            elif pick == 5:
                blk[rng.integers(0, blk.size)] = 127.0 * 2.0 ** rng.integers(-8, 8)
    with np.errstate(over="ignore"):
        return torch.from_numpy(x.astype(np.float32)).to(TYPES[kind][1])


SHAPES = [(1, 1), (1, 32), (2, 31), (3, 33), (5, 16), (7, 1001), (64, 768), (33, 4096), (2, 70001)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("random", [False, True])
def test_gpu_codes_and_values_are_bit_exact(kind, rows, cols, random):
    from gpu_util import Guarded
    rng = np.random.default_rng(rows * 1000 + cols)
    x = special_rows(rng, rows, cols, kind)
    code, dt = TYPES[kind]
    wide = ref.pitch_of(cols) + 32
    # contiguous; rows on 32-, on 16-byte boundaries; rows at any element
    for ld, offset in [(cols, 0), (wide, 0), (wide + 16 // x.element_size(), 0), (cols + 3, 1)]:
        v = matrix(rows, cols, ld, offset, kind, x.cuda())
        codes = Guarded(nc.nc_act8_code_bytes(rows, cols))
        scales = Guarded(nc.nc_act8_scale_bytes(rows, cols))
        seed, worker = 0xABCDEF0123 + cols, 5
        nc.nc_act8_compress(v, code, rows, cols, ld, int(random), seed, worker, codes.buf,
                            scales.buf)
        torch.cuda.synchronize()
        codes.check()
        scales.check()
        want_c, want_s = ref.encode(x.float().numpy(), random, seed, worker)
        got_c = codes.numpy(np.uint8).reshape(rows, -1)
        got_s = scales.numpy(np.uint8)[:want_s.size].reshape(want_s.shape)
        assert np.array_equal(got_s, want_s)
        assert np.array_equal(got_c, want_c)
        for out_kind in ("f32", "bf16", "f16"):
            out = matrix(rows, cols, ld, offset, out_kind)
            nc.nc_act8_decompress(codes.buf, scales.buf, rows, cols, out, TYPES[out_kind][0], ld)
            with np.errstate(over="ignore"):
                want = torch.from_numpy(ref.decode(want_c, want_s, cols).astype(np.float32))
            want = want.to(TYPES[out_kind][1]).float()
            got = out.cpu().float()
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))
            # nothing outside the rows was touched
            store = out.untyped_storage()
            whole = torch.empty(0, dtype=out.dtype, device="cuda").set_(store)
            mask = torch.ones_like(whole, dtype=torch.bool)
            mask[offset:offset + rows * ld].view(rows, ld)[:, :cols] = False
            assert not bool(whole[mask].float().ne(0).any())


@pytest.mark.gpu
def test_gpu_every_code_and_scale_decodes_as_defined():
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))             # 8 blocks a row
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 8, 1)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    for kind in TYPES:
        for ld, offset in [(256, 0), (257, 1)]:
            out = matrix(256, 256, ld, offset, kind)
            nc.nc_act8_decompress(c, s, 256, 256, out, TYPES[kind][0], ld)
            with np.errstate(over="ignore"):
                want = torch.from_numpy(ref.decode(codes, scales, 256).astype(np.float32))
            want = want.to(TYPES[kind][1]).float()
            got = out.cpu().float()
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


@pytest.mark.gpu
def test_gpu_random_rounding_is_unbiased_over_seeds():
    # n seeds: the mean of a value's codes is off by at most half a 1/256 unit (Y is rounded) and
    # five standard errors, the variance of a Bernoulli variable being at most 1/4
    rows, cols, n = 4, 256, 400
    g = torch.Generator().manual_seed(3)
    x = torch.randn(rows, cols, generator=g).cuda()
    codes = torch.empty(nc.nc_act8_code_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    scales = torch.empty(nc.nc_act8_scale_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    total = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    for seed in range(n):
        nc.nc_act8_compress(x, nc.DTYPE_F32, rows, cols, cols, nc.ROUND_RANDOM, seed, 0, codes,
                            scales)
        nc.nc_act8_decompress(codes, scales, rows, cols, out, nc.DTYPE_F32, cols)
        total += out.double()
    unit = torch.exp2(scales[:rows * cols // 32].double() - 127).repeat_interleave(32)
    off = ((total / n - x.double()).reshape(-1) / unit).abs()
    assert float(off.max()) <= 1 / 512 + 5 * 0.5 / n ** 0.5


@pytest.mark.gpu
def test_gpu_checkpoint_on_another_stream():
    rows, cols = 513, 1024
    x = torch.randn(rows, cols, device="cuda")
    codes = torch.empty(nc.nc_act8_code_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    scales = torch.empty(nc.nc_act8_scale_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        nc.nc_act8_compress(x, nc.DTYPE_F32, rows, cols, cols, 0, 0, 0, codes, scales)
    nc.nc_act8_decompress(codes, scales, rows, cols, out, nc.DTYPE_F32, cols, stream=side)
    side.synchronize()
    c, s = ref.encode(x.cpu().numpy())
    assert np.array_equal(out.cpu().numpy(), ref.decode(c, s, cols).astype(np.float32))
