"""The MX4 operators and the norm as a program runs them: on other streams, several at once, captured
and replayed, on memory beyond 32-bit offsets; and what the helpers refuse."""
import numpy as np
import pytest
import torch

import paper_2508_19087_amd as apt
from oracle import mx_oracle as ref
from test_gpu_mx4 import check_product, dev, f64, packed, random_mx4, rows, same_operand

pytestmark = pytest.mark.gpu
EPS = 1e-5


def layer(x, r, g, w_up, w_down, stream=None):
    """The MX4 half of a decoder layer's MLP: residual, norm, up product, down product."""
    a, h = apt.rmsnorm_mx4(x, g, EPS, residual=r, stream=stream)
    up = apt.mx4_gemm(a, w_up, torch.bfloat16, stream=stream)
    return h, up, apt.mx4_gemm_act(up, w_down, torch.bfloat16, stream=stream)


def layer_inputs(seed, M, K, N):
    x, r = dev(rows(seed, M, K, "bf16", 1.0), "bf16"), dev(rows(seed + 1, M, K, "bf16", 1.0), "bf16")
    g = dev(ref.rounded(1 + 0.25 * np.random.default_rng(seed).standard_normal(K), "bf16"), "bf16")
    return x, r, g, packed(*random_mx4(seed + 2, N, K, 118, 121)), packed(*random_mx4(seed + 3, K, N, 118, 121))


@pytest.mark.parametrize("M", [1, 7, 130])
def test_layer_against_its_parts(M):
    K, N = 512, 640
    x, r, g, up_w, down_w = layer_inputs(10 + M, M, K, N)
    h, up, down = layer(x, r, g, up_w, down_w)
    wh, wy = ref.norm(f64(x), f64(r), f64(g), EPS, "bf16")
    assert np.array_equal(f64(h), wh)
    check_product(up, ref.values(*ref.quantize(wy)), f64(apt.mx4_dequantize(up_w, torch.float32)), K, "bf16")
    check_product(down, ref.values(*ref.quantize(f64(up))), f64(apt.mx4_dequantize(down_w, torch.float32)), N, "bf16")


@pytest.mark.parametrize("M", [1, 40, 300])
def test_side_streams_at_once(M):
    """Layers on three streams at once, with work on the current stream that reuses freed blocks."""
    ins = [layer_inputs(100 * i + M, M, 768, 512) for i in range(3)]
    want = [layer(*v) for v in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        got = [layer(*v, stream=s) for v, s in zip(ins, streams)]
        junk = torch.empty(32 << 20, dtype=torch.uint8, device="cuda").fill_(0xA5)
        del junk
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_copies_are_made_on_the_calls_stream():
    """Rows whose elements are apart are copied on the stream of the call, behind what fills them there."""
    s = torch.cuda.Stream()
    x = torch.zeros(300, 64, dtype=torch.float16, device="cuda")
    w = packed(*random_mx4(1, 100, 300))
    src = dev(rows(2, 300, 64), "fp16")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        x.copy_(src)
    got = apt.mx4_gemm_act(x.t(), w, torch.float32, stream=s)
    s.synchronize()
    assert torch.equal(got, apt.mx4_gemm_act(src.t().contiguous(), w, torch.float32))


@pytest.mark.parametrize("M", [1, 5, 200])
def test_captured_and_replayed(M):
    """A captured layer over several replays, with new inputs, eager calls and synchronizations between."""
    K, N = 512, 640
    x, r, g, up_w, down_w = layer_inputs(M, M, K, N)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(x, r, g, up_w, down_w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(x, r, g, up_w, down_w)
    for i in range(4):
        x.copy_(dev(rows(1000 + i, M, K, "bf16", 1.0), "bf16"))
        graph.replay()
        want = layer(x, r, g, up_w, down_w)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_codes_captured_with_the_bipolar_gemm():
    """residual + norm -> 8-bit codes -> W4A8 GEMM in one graph, replayed on new rows."""
    K, N, M = 512, 256, 16
    g = dev(np.ones(K), "fp16")
    x, r = dev(rows(1, M, K, "fp16", 1.0), "fp16"), dev(rows(2, M, K, "fp16", 1.0), "fp16")
    w = apt.pack(torch.randint(-8, 8, (N, K), dtype=torch.int8, device="cuda"), 4)

    def run():
        codes, scale, h = apt.rmsnorm_codes(x, g, 8, EPS, residual=r)
        return apt.gemm_act(codes, 8, w)[0], scale, h

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(3):
        x.copy_(dev(rows(50 + i, M, K, "fp16", 1.0), "fp16"))
        graph.replay()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_a_given_workspace():
    x, w = dev(rows(1, 70, 500), "fp16"), packed(*random_mx4(2, 90, 500))
    need = apt.apt_mx4_gemm_act_workspace_bytes(70, 90, 500)
    ws = torch.full((need + 64, ), 0xA5, dtype=torch.uint8, device="cuda")
    got = apt.mx4_gemm_act(x, w, torch.float32, workspace=ws[:need])
    assert torch.equal(got, apt.mx4_gemm_act(x, w, torch.float32))
    assert (ws[need:] == 0xA5).all()
    with pytest.raises(apt.AptError) as e:
        apt.mx4_gemm_act(x, w, workspace=ws[:need - 1])
    assert e.value.status == apt.APT_ERR_WORKSPACE


@pytest.mark.parametrize("M,N", [(3, 70), (100, 200), (200, 131)])
def test_outputs_end_where_they_should(M, N):
    """Nothing is written behind the last element of an output."""
    K = 300
    a, w = packed(*random_mx4(1, M, K)), packed(*random_mx4(2, N, K))
    for t, dt in ((apt.APT_TYPE_FP16, torch.float16), (apt.APT_TYPE_FP32, torch.float32)):
        c = torch.full((M * N + 64, ), 7.0, dtype=dt, device="cuda")
        apt.check(apt.apt_mx4_gemm(M, N, K, a.data.data_ptr(), w.data.data_ptr(), t, c.data_ptr(),
                                   torch.cuda.current_stream().cuda_stream), "apt_mx4_gemm")
        assert torch.equal(c[:M * N].view(M, N), apt.mx4_gemm(a, w, dt)) and (c[M * N:] == 7.0).all()
        # an output that starts off any vector's alignment
        c[:] = 7.0
        apt.check(apt.apt_mx4_gemm(M, N, K, a.data.data_ptr(), w.data.data_ptr(), t, c[1:].data_ptr(),
                                   torch.cuda.current_stream().cuda_stream), "apt_mx4_gemm")
        assert torch.equal(c[1:M * N + 1].view(M, N), apt.mx4_gemm(a, w, dt)) and c[0] == 7.0 and (c[M * N + 1:] == 7.0).all()


def test_rows_beyond_32_bit_offsets():
    """Rows 4 GiB apart through the quantizer, the norm and both forms of the product."""
    K, far = 300, (1 << 31) + 5
    big = torch.empty(2 * far + K, dtype=torch.float16, device="cuda")
    x = rows(3, 3, K, "fp16", 1.0)
    view = big.as_strided((3, K), (far, 1))
    view.copy_(dev(x, "fp16"))
    op = apt.mx4_quantize(view)
    torch.cuda.synchronize()
    same_operand(op, *ref.quantize(x))
    w = packed(*random_mx4(4, 50, K))
    assert torch.equal(apt.mx4_gemm_act(view, w, torch.float32), apt.mx4_gemm(op, w, torch.float32))
    h, y = ref.norm(x, x, None, EPS, "fp16")
    codes, scale, got_h = apt.rmsnorm_codes(view, None, 8, EPS, residual=view)
    assert np.array_equal(f64(got_h), h) and np.array_equal(codes.cpu().numpy(), ref.codes(y, 8)[0])


def test_output_beyond_32_bit_offsets():
    M, N, K = 66000, 33000, 64
    a, w = random_mx4(1, M, K, 127, 129), random_mx4(2, N, K, 127, 129)
    c = apt.mx4_gemm(packed(*a), packed(*w), torch.float16)
    pick = np.array([0, 1, 31000, 32537, 32538, M - 2, M - 1])
    # the sums are multiples of 1/4 that fp32 holds; fp16 takes one rounding
    want = ref.rounded(ref.values(a[0][pick], a[1][pick]) @ ref.values(*w).T, "fp16")
    torch.cuda.synchronize()
    assert np.array_equal(c[torch.from_numpy(pick).cuda()].double().cpu().numpy(), want)


def test_helpers_refuse():
    x = torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    g = torch.ones(64, dtype=torch.float16, device="cuda")
    w = apt.mx4_quantize(torch.zeros(8, 64, dtype=torch.float16, device="cuda"))
    odd = apt.mx4_quantize(torch.zeros(8, 65, dtype=torch.float16, device="cuda"))
    calls = [
        lambda: apt.mx4_quantize(x.double()), lambda: apt.mx4_quantize(x[0]), lambda: apt.mx4_quantize(x[:0]),
        lambda: apt.mx4_quantize(x[:, :0]), lambda: apt.mx4_dequantize(w, torch.int8),
        lambda: apt.mx4_gemm(w, odd), lambda: apt.mx4_gemm_act(x, odd), lambda: apt.mx4_gemm_act(x[:0], w),
        lambda: apt.mx4_gemm_act(x, w, torch.float64),
        lambda: apt.mx4_gemm_act(torch.zeros(400, 64, device="cuda"), w, workspace=x.t()),
        lambda: apt.rmsnorm_codes(x, g[:63], 8, EPS), lambda: apt.rmsnorm_codes(x, g.float(), 8, EPS),
        lambda: apt.rmsnorm_codes(x, g, 9, EPS), lambda: apt.rmsnorm_codes(x, g, 8, -1.0),
        lambda: apt.rmsnorm_codes(x, g, 8, EPS, residual=x[:3]),
        lambda: apt.rmsnorm_codes(x, g, 8, EPS, residual=x.float()),
        lambda: apt.rmsnorm_mx4(x, g, EPS, h=x[:, :63]), lambda: apt.rmsnorm_mx4(x, g, float("nan")),
        lambda: apt.rmsnorm_mx4(x[:0], g, EPS), lambda: apt.dequantize(x, g[:4]),
        lambda: apt.dequantize(x.to(torch.int8), g[:3]),
        lambda: apt.mx4_pack(x.to(torch.uint8), x.to(torch.uint8), 64),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(apt.AptError) as e:
            call()
        assert e.value.status == apt.APT_ERR_INVALID_ARG, i
    torch.cuda.synchronize()


def test_operands_that_are_not_are_refused():
    w = apt.mx4_quantize(torch.zeros(16, 256, dtype=torch.float16, device="cuda"))
    x = torch.zeros(1, 256, dtype=torch.float16, device="cuda")
    for bad in (apt.Mx4(w.data[:-1], 16, 256), apt.Mx4(w.data, 17, 256), apt.Mx4(w.data, 16, 257), apt.Mx4(w.data, 0, 256),
                apt.Mx4(w.data.to(torch.int8), 16, 256), apt.Mx4(w.data.cpu(), 16, 256),
                apt.Mx4(torch.zeros(2 * w.data.numel(), dtype=torch.uint8, device="cuda")[::2], 16, 256),
                apt.Mx4(torch.zeros(w.data.numel() + 1, dtype=torch.uint8, device="cuda")[1:], 16, 256)):
        for call in (lambda: apt.mx4_dequantize(bad), lambda: apt.mx4_unpack(bad), lambda: apt.mx4_gemm(w, bad),
                     lambda: apt.mx4_gemm(bad, w), lambda: apt.mx4_gemm_act(x, bad)):
            with pytest.raises(apt.AptError) as e:
                call()
            assert e.value.status == apt.APT_ERR_INVALID_ARG
    # the operand's own bytes in a larger buffer are one
    again = apt.Mx4(torch.cat([w.data, w.data])[:w.data.numel()], 16, 256)
    assert torch.equal(apt.mx4_gemm_act(x, again), apt.mx4_gemm_act(x, w))
