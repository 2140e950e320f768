"""Arguments of the layer norm and of the orthogonalised updates that the library refuses before any CUDA call: no GPU is
needed, and no address that is passed here is looked at."""
import ctypes

import pytest

import paper_2204_08211_b200 as co3
from paper_2204_08211_b200 import build as cuda_build

AT = 1 << 20                      # an aligned address; refused calls do not use it
U64, SZ = ctypes.c_uint64, ctypes.c_size_t


@pytest.fixture(scope="module")
def lib():
    L = ctypes.CDLL(cuda_build.build())
    vp = ctypes.c_void_p
    L.co3_layer_norm_backward.argtypes = [vp, vp, ctypes.c_int, vp, vp, vp, vp, vp, vp, U64, ctypes.c_uint32, U64, U64, U64,
                                          ctypes.c_uint32, U64, ctypes.c_int, vp, SZ, vp]
    return L


@pytest.mark.parametrize("rows,clients", [(1 << 36, 1 << 28), (1 << 35, 1 << 29), (3 << 35, 1 << 29), (1 << 39, 2), ((1 << 40) - 1, 1 << 24)])
def test_layer_norm_backward_refuses_more_rows_than_it_counts(lib, rows, clients):
    """rows x clients of 2^64 and more must not come out as a small number."""
    assert rows * clients >= 1 << 40
    assert lib.co3_layer_norm_backward(AT, AT, 0, None, AT, AT, AT, AT, AT, rows, 1, 1, 1, 1, clients, 1, 0, AT, 1 << 40,
                                       None) == co3.ERR_INVALID_ARG
