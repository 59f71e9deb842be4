"""The token-model operators' C ABI on the CPU: the library exports what
include/nuts_token.h declares, the binding's records match the header's, and
refusals and workspace sizes need no GPU."""
import ctypes
import os
import re

import pytest

import paper_1912_11554_amd as nuts
from paper_1912_11554_amd import token_ops as ops

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "nuts_token.h")


def _source():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_exports_every_declared_function():
    declared = set(re.findall(r"\b(nuts_[a-z_]+)\s*\(", _source()))
    assert declared == set(ops.EXPORTED)
    L = nuts.load_library()
    for name in declared:
        assert hasattr(L, name), name


@pytest.mark.parametrize("record", [c for c, _ in ops._CALLS.values()], ids=lambda c: c.__name__)
def test_records_match_the_header(record):
    name = "nuts" + re.sub(r"([A-Z])", lambda m: "_" + m.group(1).lower(), record.__name__[1:]) + "_args"
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, _source()).group(1)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "double": ctypes.c_double}
    fields = []
    for decl in body.split(";"):
        words = decl.replace("const ", "").split()
        if not words:
            continue
        kind = words[0]
        for f in "".join(words[1:]).split(","):
            pointer = kind.endswith("*") or f.startswith("*")
            fields.append((f.lstrip("*"), ctypes.c_void_p if pointer else kinds[kind]))
    assert fields == list(record._fields_)


def test_null_handle_and_bad_queries():
    L = nuts.load_library()
    assert L.nuts_embedding(None, None, None) == nuts.NUTS_EINVAL
    assert L.nuts_categorical(None, None, None) == nuts.NUTS_EINVAL
    assert L.nuts_gated(None, None, None, 0, None) == nuts.NUTS_EINVAL
    assert L.nuts_linear_workspace(None) == nuts.NUTS_EINVAL
    a = ops._Linear(1, 0, -1, 4, 4)
    assert L.nuts_linear_workspace(ctypes.byref(a)) == nuts.NUTS_EINVAL  # a negative size
    a = ops._Linear(0, 0, 4, 4, 4)
    assert L.nuts_linear_workspace(ctypes.byref(a)) == nuts.NUTS_EINVAL  # fp64
    a = ops._Linear(1, 9, 4, 4, 4)
    assert L.nuts_linear_workspace(ctypes.byref(a)) == nuts.NUTS_EINVAL  # no such activation
    a = ops._Linear(1, 0, (1 << 31) - 1, (1 << 31) - 1, 1)
    assert L.nuts_linear_workspace(ctypes.byref(a)) == nuts.NUTS_EUNSUPPORTED  # too many tiles


def test_workspace_sizes():
    L = nuts.load_library()
    p = 1 << 20  # (an address: a query reads nothing)
    a = ops._EmbeddingGrad(2, 0, 1000, 50, 64, p, p, 64, 1.0, p, 64)
    need = L.nuts_embedding_grad_workspace(ctypes.byref(a))
    # sorted tokens and positions, first and last of every token, two fp32 rows a chunk of 32
    assert need >= 2 * 4000 + 2 * 200 + 32 * 2 * 64 * 4
    # a projection that fills the device needs none; a long sum of few tiles is split
    a = ops._Linear(2, 0, 4096, 4096, 4096, p, 4096, p, 4096, None, None, 0, p, 4096, None)
    assert L.nuts_linear_workspace(ctypes.byref(a)) == 0
    a = ops._Linear(2, 0, 100, 128, 1 << 16, p, 1 << 16, p, 1 << 16, None, None, 0, p, 128, None)
    assert L.nuts_linear_workspace(ctypes.byref(a)) > 0


def test_rounding_is_a_gradients_choice():
    # NUTS_ROUND_DZ halves the matrices of a bf16 gradient, at any size; it is no activation
    L = nuts.load_library()
    assert ops.NUTS_ROUND_DZ == int(re.search(r"NUTS_ROUND_DZ = (\d+)", _source()).group(1))
    p, silu = 1 << 20, ops.ACTIVATIONS["silu"]
    for M, N, K in ((64, 64, 64), (4096, 4096, 4096)):
        need = [L.nuts_linear_grad_workspace(ctypes.byref(ops._LinearGrad(
            2, silu + flag, M, N, K, p, N, p, K, p, K, p, p, K, None, 0, None))) for flag in (0, ops.NUTS_ROUND_DZ)]
        assert need[0] == 2 * M * N * 2 and need[1] == M * N * 2
    for flag in (ops.NUTS_ROUND_DZ, 512):
        a = ops._Linear(2, silu + flag, 64, 64, 64, p, 64, p, 64, None, None, 0, p, 64, None)
        assert L.nuts_linear_workspace(ctypes.byref(a)) == nuts.NUTS_EINVAL
    a = ops._LinearGrad(2, silu + 512, 64, 64, 64, p, 64, p, 64, p, 64, p, p, 64, None, 0, None)
    assert L.nuts_linear_grad_workspace(ctypes.byref(a)) == nuts.NUTS_EINVAL


@pytest.mark.parametrize("scale", [1e39, -1e300, 3.4028236e38, 1e-46, -1e-39, float("inf"), float("-inf"), float("nan")])
def test_scales_outside_fp32_are_refused(scale):
    # (in fp32 they are an infinity, whose product with a zero is no zero, or lose their digits)
    L = nuts.load_library()
    p = 1 << 20
    a = ops._EmbeddingGrad(1, 0, 100, 9, 65, p, p, 65, scale, p, 65)
    assert L.nuts_embedding_grad_workspace(ctypes.byref(a)) == nuts.NUTS_EINVAL


@pytest.mark.parametrize("scale", [0.0, -0.0, 2.0 ** -126, -3.4028234663852886e38, 1.0 / 3])
def test_scales_of_fp32_are_taken(scale):
    L = nuts.load_library()
    p = 1 << 20
    a = ops._EmbeddingGrad(1, 0, 100, 9, 65, p, p, 65, scale, p, 65)
    assert L.nuts_embedding_grad_workspace(ctypes.byref(a)) > 0
