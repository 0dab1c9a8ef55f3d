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
