"""The quantizing RMS norm on the GPU against the 64-bit oracle: h and y bit for bit (the definition
fixes every rounding), and with them codes, scales and MX4 operands."""
import numpy as np
import pytest
import torch

import paper_2508_19087_amd as apt
from oracle import mx_oracle as ref
from test_gpu_mx4 import TYPES, check_product, dev, f64, packed, random_mx4, rows, same_operand

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 7), (2, 8), (3, 33), (17, 257), (130, 512), (5, 1000), (1, 4096), (20, 4097), (9, 8192),
          (3, 11008), (2, 16385), (2, 33000)]
EPS = 1e-5


def inputs(seed, M, K, kind, residual=True, gain=True):
    x = rows(seed, M, K, kind, spread=1.0)
    r = rows(seed + 1, M, K, kind, spread=1.0) if residual else None
    g = ref.rounded(1 + 0.25 * np.random.default_rng(seed + 2).standard_normal(K), kind) if gain else None
    return x, r, g


def on(v, kind):
    return None if v is None else dev(v, kind)


def same(t, want):
    assert np.array_equal(f64(t), want, equal_nan=True)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("M,K", SHAPES)
def test_norm_codes(M, K, kind):
    for q, residual, gain in ((8, True, True), (4, False, True), (1, True, False), (5, False, False)):
        x, r, g = inputs(M + K + q, M, K, kind, residual, gain)
        h, y = ref.norm(x, r, g, EPS, kind)
        want_c, want_s = ref.codes(y, q)
        codes, scale, got_h, got_y = apt.rmsnorm_codes(on(x, kind), on(g, kind), q, EPS, residual=on(r, kind), out_y=True)
        if residual:
            same(got_h, h)
        else:
            assert got_h is None
        same(got_y, y)
        same(scale, want_s)
        assert np.array_equal(codes.cpu().numpy(), want_c)
        assert torch.equal(apt.rmsnorm_codes(on(x, kind), on(g, kind), q, EPS, residual=on(r, kind))[0], codes)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("M,K", SHAPES)
def test_norm_mx4(M, K, kind):
    for residual, gain in ((True, True), (False, False)):
        x, r, g = inputs(M + K, M, K, kind, residual, gain)
        h, y = ref.norm(x, r, g, EPS, kind)
        op, got_h, got_y = apt.rmsnorm_mx4(on(x, kind), on(g, kind), EPS, residual=on(r, kind), out_y=True)
        if residual:
            same(got_h, h)
        same(got_y, y)
        same_operand(op, *ref.quantize(y))


@pytest.mark.parametrize("K", [100, 40000])
@pytest.mark.parametrize("which", ["x", "residual"])
def test_h_in_place(which, K):
    x, r, g = inputs(3, 4, K, "bf16")
    h, y = ref.norm(x, r, g, EPS, "bf16")
    tx, tr = dev(x, "bf16"), dev(r, "bf16")
    into = tx if which == "x" else tr
    codes, scale, got = apt.rmsnorm_codes(tx, dev(g, "bf16"), 8, EPS, residual=tr, h=into)
    assert got is into
    same(got, h)
    want_c, want_s = ref.codes(y, 8)
    same(scale, want_s)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    tx, tr = dev(x, "bf16"), dev(r, "bf16")
    op, got = apt.rmsnorm_mx4(tx, dev(g, "bf16"), EPS, residual=tr, h=tx if which == "x" else tr)
    same(got, h)
    same_operand(op, *ref.quantize(y))


def test_strided_rows_and_h_without_a_residual():
    x, r, g = inputs(5, 6, 301, "fp16")
    wide = torch.zeros(6, 2, 999, dtype=torch.float16, device="cuda")
    wide[:, 0, 7:308], wide[:, 1, 3:304] = dev(x, "fp16"), dev(r, "fp16")
    h, y = ref.norm(x, r, g, EPS, "fp16")
    codes, scale, got = apt.rmsnorm_codes(wide[:, 0, 7:308], dev(g, "fp16"), 8, EPS, residual=wide[:, 1, 3:304])
    same(got, h)
    assert np.array_equal(codes.cpu().numpy(), ref.codes(y, 8)[0])
    out = torch.zeros(6, 301, dtype=torch.float16, device="cuda")
    assert apt.rmsnorm_codes(wide[:, 0, 7:308], dev(g, "fp16"), 8, EPS, h=out)[2] is out
    same(out, x)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_rows_of_zeros_extremes_and_bad_values(kind):
    K = 300
    x = np.repeat(rows(8, 1, K, kind, spread=1.0), 9, axis=0)
    tiny = {"fp16": 2.0 ** -24, "bf16": 2.0 ** -133}[kind]
    x[1] = 0.0
    x[2] = -0.0
    x[3] = tiny
    x[4, 17] = float(torch.finfo(TYPES[kind]).max)
    x[5, 0] = np.inf
    x[6, 299] = np.nan
    x[7], x[7, 5] = tiny, -4 * tiny
    g = np.ones(K)
    g[:4] = [0.0, -2.0, 3.0, -0.0]
    for eps in (EPS, 0.0, 1e-30):
        h, y = ref.norm(x, None, g, eps, kind)
        for q in (8, 3):
            codes, scale, _, got_y = apt.rmsnorm_codes(dev(x, kind), dev(g, kind), q, eps, out_y=True)
            same(got_y, y)
            want_c, want_s = ref.codes(y, q)
            same(scale, want_s)
            assert np.array_equal(codes.cpu().numpy(), want_c)
        op, _, got_y = apt.rmsnorm_mx4(dev(x, kind), dev(g, kind), eps, out_y=True)
        same(got_y, y)
        same_operand(op, *ref.quantize(y))


def test_sums_that_overflow_the_type_have_no_codes():
    x = np.full((2, 64), 40000.0)
    x[1] = 1.0
    codes, scale, h = apt.rmsnorm_codes(dev(x, "fp16"), None, 8, EPS, residual=dev(x, "fp16"))
    assert np.isinf(f64(h)[0]).all() and np.isnan(f64(scale)[0]) and not codes[0].any()
    assert f64(scale)[1] > 0


@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (5, 2049), (130, 512)])
def test_dequantize_codes(M, K, kind):
    g = np.random.default_rng(M + K)
    codes = g.integers(-128, 128, (M, K)).astype(np.int8)
    scale = np.exp(g.standard_normal(M)).astype(np.float16)
    scale[0] = np.nan if M > 1 else scale[0]
    got = apt.dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda(), TYPES[kind])
    # (2 code + 1) scale has at most 9 + 11 bits: exact in fp32, then one rounding
    same(got, ref.rounded((2.0 * codes + 1) * scale.astype(np.float64)[:, None], kind))


@pytest.mark.parametrize("M", [1, 3, 70])
def test_norm_into_the_products(M):
    """residual + norm -> codes -> W4A8 GEMM, and residual + norm -> MX4 -> product, as a decoder layer runs them."""
    K, N = 512, 300
    x, r, g = inputs(M, M, K, "fp16")
    h, y = ref.norm(x, r, g, EPS, "fp16")
    wc = np.random.default_rng(1).integers(-8, 8, (N, K)).astype(np.int8)
    w = apt.pack(torch.from_numpy(wc).cuda(), 4)
    ws = torch.full((N, ), 0.0625, dtype=torch.float16, device="cuda")
    codes, scale, got_h = apt.rmsnorm_codes(dev(x, "fp16"), dev(g, "fp16"), 8, EPS, residual=dev(r, "fp16"))
    c32, c16, _ = apt.gemm_act(codes, 8, w, a_scale=scale, w_scale=ws, out_fp16=True)
    same(got_h, h)
    want_c, want_s = ref.codes(y, 8)
    want = (2 * want_c.astype(np.int64) + 1) @ (2 * wc.astype(np.int64) + 1).T
    assert np.array_equal(c32.cpu().numpy(), want)
    out = want * want_s[:, None] * 0.0625
    assert (np.abs(f64(c16) - out) <= 2.0 ** -10 * np.abs(out) + 2.0 ** -24).all()
    # the same from y through the fp16 quantizer
    y16 = torch.from_numpy(y).half().cuda()
    assert torch.equal(apt.gemm_act(y16, 8, w)[0], c32)
    wm = random_mx4(2, N, K, 118, 124)
    pw = packed(*wm)
    op, _ = apt.rmsnorm_mx4(dev(x, "fp16"), dev(g, "fp16"), EPS, residual=dev(r, "fp16"))
    got = apt.mx4_gemm(op, pw, torch.float32)
    assert torch.equal(got, apt.mx4_gemm_act(y16, pw, torch.float32))
    check_product(got, ref.values(*ref.quantize(y)), ref.values(*wm), K, "fp32")


# several rows to a workgroup: full and ragged workgroups, rows of every width that shares one
SHORT = [(1, 128), (15, 128), (17, 120), (33, 127), (1000, 128), (1024, 64), (1039, 120), (1100, 8), (1027, 127),
         (1040, 129), (1500, 200), (1033, 256), (1050, 260), (1029, 500), (2100, 512), (1031, 1),
         (2051, 250), (2049, 120), (2063, 31), (2048, 256), (2060, 481)]


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("M,K", SHORT)
def test_norm_of_short_rows(M, K, kind):
    x, r, g = inputs(M + K, M, K, kind)
    h, y = ref.norm(x, r, g, EPS, kind)
    codes, scale, got_h, got_y = apt.rmsnorm_codes(on(x, kind), on(g, kind), 6, EPS, residual=on(r, kind), out_y=True)
    want_c, want_s = ref.codes(y, 6)
    same(got_h, h)
    same(got_y, y)
    same(scale, want_s)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    op, got_h, got_y = apt.rmsnorm_mx4(on(x, kind), on(g, kind), EPS, residual=on(r, kind), out_y=True)
    same(got_h, h)
    same(got_y, y)
    same_operand(op, *ref.quantize(y))


@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,K", SHORT + [(7, 1000), (5, 1030), (9, 2048)])
def test_values_of_short_rows(M, K, kind):
    g = np.random.default_rng(M + K)
    codes, scale = g.integers(-128, 128, (M, K)).astype(np.int8), np.exp(g.standard_normal(M)).astype(np.float16)
    got = apt.dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda(), TYPES[kind])
    same(got, ref.rounded((2.0 * codes + 1) * scale.astype(np.float64)[:, None], kind))


def test_a_bad_short_row_stays_alone():
    x = np.ones((1030, 96))
    x[5, 3], x[20, 95] = np.nan, np.inf
    codes, scale, _ = apt.rmsnorm_codes(dev(x, "bf16"), None, 8, EPS)
    bad = np.isnan(f64(scale))
    assert bad[5] and bad[20] and bad.sum() == 2 and not codes[5].any() and not codes[20].any()
    assert (codes.cpu().numpy()[~bad] == 127).all()


@pytest.mark.parametrize("K", [61, 128, 300])
@pytest.mark.parametrize("which", ["x", "residual"])
def test_short_rows_in_place(which, K):
    M = 2100
    x, r, g = inputs(K, M, K, "bf16")
    h, y = ref.norm(x, r, g, EPS, "bf16")
    want_c, want_s = ref.codes(y, 8)
    for to in ("codes", "mx4"):
        tx, tr, tg = dev(x, "bf16"), dev(r, "bf16"), dev(g, "bf16")
        own = tx if which == "x" else tr
        if to == "codes":
            codes, scale, got_h = apt.rmsnorm_codes(tx, tg, 8, EPS, residual=tr, h=own)
            same(scale, want_s)
            assert np.array_equal(codes.cpu().numpy(), want_c)
        else:
            op, got_h = apt.rmsnorm_mx4(tx, tg, EPS, residual=tr, h=own)
            same_operand(op, *ref.quantize(y))
        assert got_h is own
        same(own, h)
