"""Paths of the MX4 operators and the norm that only some sizes take, on the GPU: every kernel of the
product with every rest of its loop, subnormal sums, the longest rows of the norm, outputs past the
cache whose rows share lines, and problems of more than one launch."""
import numpy as np
import pytest
import torch

import paper_2508_19087_amd as apt
from mx_sizes import FUSED, KERNELS
from oracle import mx_oracle as ref
from test_gpu_mx4 import TYPES, dev, f64, packed, random_mx4, rows, same_operand
from test_gpu_rmsnorm import inputs, on, same

pytestmark = pytest.mark.gpu
EPS = 1e-5
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def stream():
    return torch.cuda.current_stream().cuda_stream


def scaled(seed, R, K, low):
    """An operand with scales of 2^low or twice that, made on the device, and its values in fp64."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    nibbles = torch.randint(0, 16, (R, K), dtype=torch.uint8, device="cuda", generator=g)
    bits = torch.randint(0, 2, (R, -(-K // 32)), dtype=torch.uint8, device="cuda", generator=g)
    even = torch.nn.functional.pad(nibbles, (0, K % 2))
    values = LEVELS.cuda()[(nibbles & 7).long()] * (1 - 2 * (nibbles >> 3).double())
    values = values * (1.0 + bits.double()).repeat_interleave(32, 1)[:, :K] * 2.0 ** low
    return apt.mx4_pack(even[:, ::2] | even[:, 1::2] << 4, bits + (low + 127), K), values


def check_exact(got, want, what):
    torch.cuda.synchronize()
    assert torch.equal(got, want), what


@pytest.mark.parametrize("size", [s for k in KERNELS.values() for s in k], ids=lambda s: "%dx%dx%d" % s)
def test_product_of_every_kernel(size):
    """Scales of 1 and 2: every partial sum is a multiple of 1/4 below 144 * 8200 < 2^22, 24 bits, which fp32
    holds, so the outputs are its roundings."""
    M, N, K = size
    (a, va), (w, vw) = scaled(M, M, K, 0), scaled(N + 1, N, K, 0)
    want = va @ vw.t().contiguous()
    for kind, dtype in TYPES.items():
        check_exact(apt.mx4_gemm(a, w, dtype), want.float().to(dtype), kind)


@pytest.mark.parametrize("size", FUSED, ids=lambda s: "%dx%dx%d" % s)
def test_rows_quantized_by_the_product(size):
    """The same from rows that quantizing leaves as they are (a scale is 2^-2 or more of the block's largest
    value's power of two, so multiples of the old scale's half are ones of the new's)."""
    M, N, K = size
    (_, va), (w, vw) = scaled(M, M, K, 0), scaled(N + 1, N, K, 0)
    want = (va @ vw.t().contiguous()).float()
    for kind, dtype in TYPES.items():
        x = va.to(dtype)
        assert torch.equal(x.double(), va)
        check_exact(apt.mx4_gemm_act(x, w, torch.float32), want, kind)
        wide = torch.full((M, K + 9), float("nan"), dtype=dtype, device="cuda")
        wide[:, 3:K + 3] = x
        check_exact(apt.mx4_gemm_act(wide[:, 3:K + 3], w, torch.float32), want, "%s, rows apart" % kind)


@pytest.mark.parametrize("size", [(3, 21840, 4000), (3, 21841, 4000), (16, 16384, 1000), (16, 16385, 1000), (2, 33001, 4000)],
                         ids=lambda s: "%dx%dx%d" % s)
def test_few_rows_by_many_weight_rows(size):
    """On both sides of the limit on repeated conversions."""
    M, N, K = size
    (_, va), (w, vw) = scaled(M, M, K, 0), scaled(N + 1, N, K, 0)
    want = (va @ vw.t().contiguous()).float()
    check_exact(apt.mx4_gemm_act(va.half(), w, torch.float32), want, size)


@pytest.mark.parametrize("workspace", ["none", "short", "off alignment"])
def test_few_rows_need_no_workspace(workspace):
    """Rows that the product's kernel can quantize are taken without a workspace of use, where one would be faster."""
    M, N, K = 4, 20011, 4000
    need = apt.apt_mx4_gemm_act_workspace_bytes(M, N, K)
    assert need == apt.apt_mx4_bytes(M, K)
    x, w = dev(rows(1, M, K, "bf16", 1.0), "bf16"), packed(*random_mx4(2, N, K, 118, 121))
    buf = torch.full((need + 64, ), 0xA5, dtype=torch.uint8, device="cuda")
    ptr, n = {"none": (None, 0), "short": (buf.data_ptr(), need - 1), "off alignment": (buf.data_ptr() + 8, need)}[workspace]
    c = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    apt.check(apt.apt_mx4_gemm_act(M, N, K, x.data_ptr(), apt.APT_TYPE_BF16, K, w.data.data_ptr(), apt.APT_TYPE_BF16,
                                   c.data_ptr(), ptr, n, stream()), "apt_mx4_gemm_act")
    check_exact(c, apt.mx4_gemm_act(x, w), workspace)
    assert (buf == 0xA5).all()


SOME = [(5, 20, 703), (17, 2052, 208), (17, 4206, 2120), (34, 5672, 4797), (33, 20, 353), (4100, 133, 686),
        (193, 8225, 436), (457, 8194, 473), (1089, 7413, 2770)]


@pytest.mark.parametrize("size", SOME, ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("low_a,low_w", [(-127, -20), (-20, -127), (-127, -15), (-70, -77), (-124, -19)])
def test_subnormal_sums(size, low_a, low_w):
    """Products are multiples of 2^(low_a + low_w - 2), sums below 144 * 4800 < 2^20 times 2^(low_a + low_w):
    22 bits of which none lies below 2^-149, so fp32 with its subnormal numbers holds every sum."""
    M, N, K = size
    assert low_a + low_w - 2 >= -149 and K < 4800
    (a, va), (w, vw) = scaled(M, M, K, low_a), scaled(N + 1, N, K, low_w)
    want = va @ vw.t().contiguous()
    # (on the host: no device rounds or flushes the expected values)
    want = want.cpu().float()
    assert low_a + low_w > -145 or (want.abs() < 2.0 ** -126).any()
    for kind in ("fp32", "bf16"):
        check_exact(apt.mx4_gemm(a, w, TYPES[kind]).cpu(), want.to(TYPES[kind]), kind)


@pytest.mark.parametrize("size", SOME, ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("low", [-32, -26])
def test_subnormal_fp16_outputs(size, low):
    """Multiples of 2^(low - 2), of 22 bits: exact in fp32, then one rounding to fp16, most of them subnormal."""
    M, N, K = size
    (a, va), (w, vw) = scaled(M, M, K, low + 5), scaled(N + 1, N, K, -5)
    want = (va @ vw.t().contiguous()).cpu()
    assert (want.abs() < 2.0 ** -14).any()
    check_exact(apt.mx4_gemm(a, w, torch.float16).cpu(), want.half(), low)


# ---- the norm's longest rows ----------------------------------------------------------
# (up to 32768 elements a row stays in registers, four vectors a thread; beyond, it is read again in
# each pass, its last vector from eight elements that its neighbour's overlap)

LONG = [16640, 20000, 32767, 32768, 32769, 33001, 40003]


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("K", LONG)
@pytest.mark.parametrize("into", [None, "x", "residual"])
def test_norm_of_long_rows(K, kind, into):
    x, r, g = inputs(K, 3, K, kind)
    h, y = ref.norm(x, r, g, EPS, kind)
    want_c, want_s = ref.codes(y, 7)
    for to in ("codes", "mx4"):
        tx, tr, tg = dev(x, kind), dev(r, kind), dev(g, kind)
        own = {"x": tx, "residual": tr}.get(into)
        if to == "codes":
            codes, scale, got_h, got_y = apt.rmsnorm_codes(tx, tg, 7, EPS, residual=tr, h=own, out_y=True)
            same(scale, want_s)
            assert np.array_equal(codes.cpu().numpy(), want_c)
        else:
            op, got_h, got_y = apt.rmsnorm_mx4(tx, tg, EPS, residual=tr, h=own, out_y=True)
            same_operand(op, *ref.quantize(y))
        assert own is None or got_h is own
        same(got_h, h)
        same(got_y, y)
        if into != "x":
            same(tx, x)
        if into != "residual":
            same(tr, r)


@pytest.mark.parametrize("K", [20000, 33001])
def test_norm_of_long_rows_alone(K):
    """No residual, no gain, no h; rows apart and off alignment."""
    x, _, _ = inputs(K, 2, K, "bf16", False, False)
    _, y = ref.norm(x, None, None, EPS, "bf16")
    wide = torch.full((2, K + 77), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 5:K + 5] = dev(x, "bf16")
    codes, scale, h = apt.rmsnorm_codes(wide[:, 5:K + 5], None, 8, EPS)
    assert h is None
    same(scale, ref.codes(y, 8)[1])
    assert np.array_equal(codes.cpu().numpy(), ref.codes(y, 8)[0])
    same_operand(apt.rmsnorm_mx4(wide[:, 5:K + 5], None, EPS)[0], *ref.quantize(y))


# ---- values past the cache whose rows share lines --------------------------------------

@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("R,K", [(2048, 4099), (1600, 4097), (12345, 613)])
@pytest.mark.parametrize("shift", [0, 1, 5])
def test_large_ragged_values(R, K, kind, shift):
    """12 MiB and more, from an odd element on, with a border on both sides that stays as it was."""
    codes, scales = random_mx4(R, R, K, 105, 140)
    op = packed(codes, scales)
    want = torch.from_numpy(ref.rounded(ref.values(codes, scales), kind)).cuda()
    t = {"fp16": apt.APT_TYPE_FP16, "bf16": apt.APT_TYPE_BF16, "fp32": apt.APT_TYPE_FP32}[kind]
    assert R * K * TYPES[kind].itemsize >= 12 << 20
    buf = torch.full((R * K + 64, ), 7.0, dtype=TYPES[kind], device="cuda")

    def check(got, what):
        torch.cuda.synchronize()
        assert torch.equal(got[shift:shift + R * K].view(R, K).double(), want), what
        assert (got[:shift] == 7.0).all() and (got[shift + R * K:] == 7.0).all(), what

    apt.check(apt.apt_mx4_dequantize(op.data.data_ptr(), R, K, t, buf[shift:].data_ptr(), stream()), "values")
    check(buf, "MX4")
    g = np.random.default_rng(K)
    c = torch.from_numpy(g.integers(-128, 128, (R, K)).astype(np.int8)).cuda()
    s = torch.from_numpy(np.exp(g.standard_normal(R)).astype(np.float16)).cuda()
    # (20 bits: exact in fp32 and fp64, then one rounding)
    want = ((2.0 * c.double() + 1) * s.double()[:, None]).float().to(TYPES[kind]).double()
    buf.fill_(7.0)
    apt.check(apt.apt_dequantize_codes(c.data_ptr(), s.data_ptr(), R, K, t, buf[shift:].data_ptr(), stream()), "values")
    check(buf, "codes")


# ---- more than one launch ----------------------------------------------------------------

@pytest.mark.parametrize("K", [8, 520])
def test_norms_of_more_rows_than_a_launch_takes(K):
    """Beyond 2^21 rows a second launch follows: the rows around the border and the last ones against
    the oracle, everything behind the border against a call of its own."""
    M, at = (1 << 21) + 37, (1 << 21) - 48
    g = torch.Generator(device="cuda")
    g.manual_seed(K)
    x = torch.randn((M, K), device="cuda", generator=g).bfloat16()
    r = torch.randn((M, K), device="cuda", generator=g).bfloat16()
    gain = (1 + 0.25 * torch.randn(K, device="cuda", generator=g)).bfloat16()
    pick = torch.cat([torch.arange(20), torch.arange(M // 2, M // 2 + 20), torch.arange(at, M)]).cuda()
    h, y = ref.norm(f64(x[pick]), f64(r[pick]), f64(gain), EPS, "bf16")
    want_c, want_s = ref.codes(y, 8)
    codes, scale, got_h, got_y = apt.rmsnorm_codes(x, gain, 8, EPS, residual=r, out_y=True)
    same(got_h[pick], h)
    same(got_y[pick], y)
    same(scale[pick], want_s)
    assert np.array_equal(codes[pick].cpu().numpy(), want_c)
    tail = apt.rmsnorm_codes(x[at:], gain, 8, EPS, residual=r[at:], out_y=True)
    assert all(torch.equal(p[at:], q) for p, q in zip((codes, scale, got_h, got_y), tail))
    op, got_h, got_y = apt.rmsnorm_mx4(x, gain, EPS, residual=r, out_y=True)
    same(got_h[pick], h)
    same(got_y[pick], y)
    part, _ = apt.rmsnorm_mx4(x[at:], gain, EPS, residual=r[at:])
    same_operand(part, *ref.quantize(f64(got_y[at:])))
    # the operand's last groups, codes and scales
    groups, steps, of_part = -(-M // 16), -(-K // 256), -(-(M - at) // 16)
    real = of_part - 1  # the last group is not full
    assert M % 16 and at % 16 == 0

    def last(data, first, bytes_, count):
        return data[first:first + groups_of(data) * steps * bytes_].view(-1, steps * bytes_)[-of_part:][:count]

    def groups_of(data):
        return data.numel() // (steps * 2176)

    for first, bytes_ in ((lambda d: 0, 2048), (lambda d: groups_of(d) * steps * 2048, 128)):
        a = last(op.data, first(op.data), bytes_, real)
        b = last(part.data, first(part.data), bytes_, real)
        assert groups_of(op.data) == groups and torch.equal(a, b)
    # and the rows of the last one, by their values
    assert torch.equal(apt.mx4_dequantize(op)[at:], apt.mx4_dequantize(part))


@pytest.mark.parametrize("M,K", [((1 << 23) + 5, 1), ((1 << 22) + 3, 2049)])
def test_values_of_more_rows_than_a_launch_takes(M, K):
    """2^23 parts of up to 2048 elements to a launch."""
    g = torch.Generator(device="cuda")
    g.manual_seed(K)
    codes = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    scale = (0.5 + torch.rand(M, device="cuda", generator=g)).half()
    got = apt.dequantize(codes, scale)
    torch.cuda.synchronize()
    for at in (0, M // 2, (1 << 22) - 30, M - 60):
        p = slice(at, at + 60)
        want = ((2.0 * codes[p].double() + 1) * scale[p].double()[:, None]).half()
        assert torch.equal(got[p], want), at


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("M,K", [(4, 300), (2100, 96), (3, 33001)])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_norm_at_the_types_ends(M, K, kind, eps):
    """Whole rows of the largest values (in bf16 the row's factor is a subnormal fp32 number), of the
    smallest and of subnormal ones, and all of them mixed."""
    info = torch.finfo(TYPES[kind])
    sign = np.where(np.random.default_rng(K).random(K) < 0.5, -1.0, 1.0)
    x = np.zeros((M, K))
    x[0] = sign * float(info.max)
    x[1] = sign * float(info.smallest_normal)
    x[2] = sign * {"fp16": 2.0 ** -24, "bf16": 2.0 ** -133}[kind]
    if M > 3:
        x[3:] = np.where(np.arange(K) % 3 == 0, x[0], np.where(np.arange(K) % 3 == 1, x[1], x[2]))
    h, y = ref.norm(x, None, None, eps, kind)
    codes, scale, _, got_y = apt.rmsnorm_codes(dev(x, kind), None, 8, eps, out_y=True)
    same(got_y, y)
    want_c, want_s = ref.codes(y, 8)
    same(scale, want_s)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    op, _, got_y = apt.rmsnorm_mx4(dev(x, kind), None, eps, out_y=True)
    same(got_y, y)
    same_operand(op, *ref.quantize(y))
