"""Checks that the MX4 helpers make of operands and sizes before C sees them, on the host: stand-ins
take the place of device tensors, and of the C function that must not be reached."""
import copy

import pytest
import torch

import paper_2508_19087_amd as apt
from paper_2508_19087_amd import mx

BAD, UNSUPPORTED = apt.APT_ERR_INVALID_ARG, apt.APT_ERR_UNSUPPORTED


class OnDevice:
    """What the helpers ask of a device tensor: sizes, type and place; no memory behind it."""
    is_cuda = True
    device = torch.device("cuda", 0)

    def __init__(self, shape, dtype=torch.uint8, contiguous=True):
        self.shape, self.dtype, self._contiguous = torch.Size(shape), dtype, contiguous

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self._contiguous

    def stride(self, i):
        return self.shape[1:].numel() if i == 0 else 1

    def data_ptr(self):
        return 1 << 20

    def new_empty(self, shape, dtype=None):
        return OnDevice((shape, ) if isinstance(shape, int) else shape, dtype or self.dtype)


@pytest.fixture
def reached(monkeypatch):
    """Names of the C functions that a helper would have called."""
    names = []
    monkeypatch.setattr(mx, "_call", lambda name, *a: names.append(name))
    return names


def operand(rows=16, K=256):
    return apt.Mx4(OnDevice((apt.apt_mx4_bytes(rows, K), )), rows, K)


def refused(call, status=BAD):
    with pytest.raises(apt.AptError) as e:
        call()
    assert e.value.status == status


def uses(a):
    x = OnDevice((1, a.K), torch.float16)
    good = operand(16, a.K)
    return [lambda: apt.mx4_dequantize(a), lambda: apt.mx4_unpack(a), lambda: apt.mx4_gemm(a, good),
            lambda: apt.mx4_gemm(good, a), lambda: apt.mx4_gemm_act(x, a)]


def change_rows(a):
    a.rows = 4096


def change_K(a):
    a.K = 257


def shrink_data(a):
    a.data.shape = torch.Size((a.data.numel() - 1, ))


def retype_data(a):
    a.data.dtype = torch.int8


def scatter_data(a):
    a.data._contiguous = False


def exchange_data(a):
    a.data = OnDevice((2175, ))


@pytest.mark.parametrize("change", [change_rows, change_K, shrink_data, retype_data, scatter_data, exchange_data])
@pytest.mark.parametrize("copied", [False, True])
@pytest.mark.parametrize("use", range(5))
def test_an_operand_changed_after_a_use_is_refused(reached, change, copied, use):
    a = operand()
    uses(a)[use]()
    assert reached  # as it was made it is good, and has now been used
    del reached[:]
    if copied:
        a = copy.copy(a)
    change(a)
    refused(uses(a)[use])
    assert not reached


def test_an_operand_that_a_helper_made_is_checked_too(reached):
    a = apt.mx4_quantize(OnDevice((16, 256), torch.float16))
    assert reached == ["apt_mx4_quantize"]
    a.rows = 17
    refused(lambda: apt.mx4_dequantize(a))
    assert reached == ["apt_mx4_quantize"]


def test_a_changed_operand_that_still_fits_is_taken(reached):
    a = operand(17, 256)
    apt.mx4_dequantize(a)
    a.rows = 5
    apt.mx4_dequantize(a)
    assert reached == ["apt_mx4_dequantize"] * 2


@pytest.mark.parametrize("rows", [-1, 0, 1, 15, 16, 17, 4096, 2 ** 31 - 1])
@pytest.mark.parametrize("K", [-1, 0, 1, 255, 256, 257, 11008, 2 ** 30])
def test_sizes_are_the_librarys(rows, K):
    assert mx._bytes(rows, K) == apt.apt_mx4_bytes(rows, K)


# ---- sizes that an int of C does not hold -----------------------------------------
# (C takes them modulo 2^32: 2^32 + 16 rows as 16)

HUGE = [2 ** 31, 2 ** 32 + 16, 2 ** 40 + 256]
F16, P = apt.APT_TYPE_FP16, 1 << 20
# (names and arguments in order; the C function is called with the numbers that are asked for)
ENTRIES = [
    ("apt_mx4_quantize", dict(x=P, type=F16, rows=16, K=256, stride=2 ** 41, mx=P, stream=None), ("rows", "K", "type")),
    ("apt_mx4_dequantize", dict(mx=P, rows=16, K=256, type=F16, out=P, stream=None), ("rows", "K", "type")),
    ("apt_mx4_pack", dict(codes=P, scales=P, rows=16, K=256, mx=P, stream=None), ("rows", "K")),
    ("apt_mx4_unpack", dict(mx=P, rows=16, K=256, codes=P, scales=P, stream=None), ("rows", "K")),
    ("apt_mx4_gemm", dict(M=16, N=16, K=256, a_mx=P, w_mx=P, type=F16, c=P, stream=None), ("M", "N", "K", "type")),
    ("apt_mx4_gemm_act", dict(M=16, N=16, K=256, x=P, x_type=F16, x_stride=2 ** 41, w_mx=P, type=F16, c=P,
                              workspace=P, workspace_bytes=1 << 40, stream=None), ("M", "N", "K", "type", "x_type")),
    ("apt_rmsnorm_codes", dict(M=16, K=256, type=F16, x=P, x_stride=2 ** 41, residual=None, residual_stride=0, gain=None,
                               eps=1e-5, q=8, h=None, y=None, codes=P, scale=P, stream=None), ("M", "K", "type", "q")),
    ("apt_rmsnorm_mx4", dict(M=16, K=256, type=F16, x=P, x_stride=2 ** 41, residual=None, residual_stride=0, gain=None,
                             eps=1e-5, h=None, y=None, mx=P, stream=None), ("M", "K", "type")),
    ("apt_dequantize_codes", dict(codes=P, scale=P, M=16, K=256, type=F16, out=P, stream=None), ("M", "K", "type")),
]


class Library:
    """A library whose functions record that they were called, and do nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append(name) or 0


@pytest.mark.parametrize("name,args,numbers", ENTRIES, ids=[e[0] for e in ENTRIES])
def test_entry_points_refuse_numbers_beyond_c(monkeypatch, name, args, numbers):
    library = Library()
    monkeypatch.setattr(mx, "_lib", library)
    assert getattr(apt, name)(**args) == apt.APT_OK and library.calls == [name]
    for number in numbers:
        for huge in HUGE + [-2 ** 31 - 1, 2 ** 32 + args[number]]:
            assert getattr(apt, name)(**(args | {number: huge})) == BAD, (number, huge)
    assert library.calls == [name]


def test_sizes_in_bytes_beyond_c():
    for huge in HUGE + [-2 ** 32 + 16]:
        assert apt.apt_mx4_bytes(huge, 1) == 0 and apt.apt_mx4_bytes(1, huge) == 0
        for sizes in ((huge, 16, 256), (300, huge, 256), (300, 16, huge)):
            assert apt.apt_mx4_gemm_act_workspace_bytes(*sizes) == 0


@pytest.mark.parametrize("huge", HUGE)
def test_helpers_refuse_sizes_beyond_c(reached, huge):
    w = operand(16, 256)
    for shape in ((huge, 256), (16, huge)):
        x, codes = OnDevice(shape, torch.float16), OnDevice(shape, torch.int8)
        refused(lambda: apt.mx4_quantize(x))
        refused(lambda: apt.rmsnorm_codes(x, None, 8, 1e-5))
        refused(lambda: apt.rmsnorm_mx4(x, None, 1e-5))
        refused(lambda: apt.dequantize(codes, OnDevice(shape[:1], torch.float16)))
        refused(lambda: apt.mx4_gemm_act(x, apt.Mx4(w.data, 16, shape[1])))
        refused(lambda: apt.mx4_pack(OnDevice((shape[0], -(-shape[1] // 2))), OnDevice((shape[0], -(-shape[1] // 32))),
                                     shape[1]))
        big = apt.Mx4(OnDevice((2 ** 60, )), *shape)
        for use in uses(apt.Mx4(big.data, huge, 256)) + [lambda: apt.mx4_dequantize(big), lambda: apt.mx4_unpack(big),
                                                          lambda: apt.mx4_gemm(big, big)]:
            refused(use)
    assert not reached


@pytest.mark.parametrize("q", [0, 9, -1, 2 ** 32 + 8])
def test_norm_refuses_bits_out_of_range(reached, q):
    refused(lambda: apt.rmsnorm_codes(OnDevice((16, 256), torch.float16), None, q, 1e-5))
    assert not reached


@pytest.mark.parametrize("K", [2 ** 31 - 1, 2 ** 31 - 255, 2 ** 31 - 256, 2 ** 30 + 1])
def test_bytes_of_the_longest_rows(K):
    for rows in (1, 17, 2 ** 31 - 1):
        assert apt.apt_mx4_bytes(rows, K) == -(-rows // 16) * -(-K // 256) * 2176
