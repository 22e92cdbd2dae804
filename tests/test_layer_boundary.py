"""CPU-only checks of layer norm, the product in 8-bit integers and sampling: arguments are refused before anything touches a GPU, and what
the compiler made of their kernels."""
import ctypes as C
import math
import re

import pytest
import torch

SOURCES = ["qadam_layer_norm.hip", "qadam_linear8.hip", "qadam_sampler.hip"]


@pytest.fixture(scope="module")
def lib():
    from paper_2004_14180_amd import binding
    from paper_2004_14180_amd.build import build_library
    import os
    if not os.path.exists(binding.library_path()):
        build_library(verbose=False)
    return binding.load_library()


def test_init_refuses_on_the_host(lib):
    h = C.c_void_p()
    for dim, eps, want in [(0, 1e-5, -1), (-4, 1e-5, -1), ((1 << 20) + 1, 1e-5, -3), (4, -1.0, -1), (4, math.nan, -1), (4, math.inf, -1)]:
        assert lib.qadam_layer_norm_init(C.byref(h), dim, eps) == want and lib.qadam_last_error()
    for outputs, inputs, tokens, want in [(0, 1, 1, -1), (1, 0, 1, -1), (1, 1, -1, -1), ((1 << 24) + 1, 1, 1, -3), (1, 1 << 17, 1, -3),
                                          (1, 1, (1 << 24) + 1, -3), (1, 1 << 16, (1 << 20) + 1, -3)]:
        assert lib.qadam_linear8_init(C.byref(h), outputs, inputs, tokens) == want, (outputs, inputs, tokens)
    for vocab, rows, want in [(0, 1, -1), (1, -1, -1), ((1 << 22) + 1, 1, -3), (1, (1 << 24) + 1, -3)]:
        assert lib.qadam_sampler_init(C.byref(h), vocab, rows) == want, (vocab, rows)
    assert lib.qadam_layer_norm_init(None, 4, 1e-5) == -1 and lib.qadam_linear8_init(None, 1, 1, 1) == -1 and lib.qadam_sampler_init(None, 1, 1) == -1


def test_calls_without_a_handle(lib):
    from paper_2004_14180_amd.binding import _Filters
    assert lib.qadam_layer_norm_destroy(None) == 0 and lib.qadam_linear8_destroy(None) == 0 and lib.qadam_sampler_destroy(None) == 0
    assert lib.qadam_layer_norm(None, 1, None, 0, 4, None, None, 0, None, 0, 4, None, None, None) == -1
    assert lib.qadam_layer_norm_grad(None, 1, None, 0, 4, None, 0, 4, None, 0, None, None, None, 0, 4, None, None, 0, 0, None) == -1
    assert lib.qadam_linear8_quantize(None, 1, None, 0, 4, None, 4, None, None) == -1
    assert lib.qadam_linear8_forward(None, 1, None, 0, 4, None, None, 4, None, 6, None, 0, None, 0, 4, None) == -1
    assert lib.qadam_sampler_sample(None, 1, None, 0, 4, None, C.byref(_Filters()), None, 4, None) == -1
    assert lib.qadam_sampler_get_status(None, None, 0, None) == -1


def test_integers_beyond_the_boundary_types_are_refused(lib):
    from paper_2004_14180_amd import LayerNorm, Linear8, Sampler
    for make in (lambda: LayerNorm((1 << 32) + 4), lambda: Linear8((1 << 64) + 1, 4, 4), lambda: Linear8(4, (1 << 32) + 4, 4),
                 lambda: Linear8(4, 4, (1 << 64) + 4), lambda: Sampler((1 << 64) + 4, 4), lambda: Sampler(4, (1 << 64) + 4)):
        with pytest.raises(ValueError, match="does not fit"):
            make()


def test_native_calls_leave_other_forms_to_the_python_checks(lib):
    """None, and nothing called: the entry points of these plans are address 0."""
    from paper_2004_14180_amd import binding
    native = binding._native
    plan = native.layer_plan(0, 8, 4, 0, 0)
    x, v, n, i = torch.zeros(2, 8), torch.zeros(8), torch.zeros(2), torch.zeros(2, dtype=torch.int64)
    for p in (None, plan):
        assert native.layer_norm(p, -1, 0, x, v, v, x, n, n) is None
        assert native.layer_norm_grad(p, -1, 0, x, x, v, n, n, x, v, v, False) is None
        assert native.linear8_quantize(p, -1, 0, x, x.to(torch.int8), n) is None
        assert native.linear8_forward(p, -1, 0, x, torch.zeros(4, 8, dtype=torch.int8), torch.zeros(2, 4), None, 6, None, None) is None
        assert native.sample(p, -1, 0, x, n, i, 1.0, 0, 1.0, 0.0) is None
        assert native.sample(p, 0, 0, None, 3, "x", None, 2.0, [], 1 << 70) is None
        assert native.layer_norm(p, 0, 0, None, 3, "x", None, 2.0, []) is None
        assert native.layer_norm_grad(p, 0, 0, None, 3, "x", None, 2.0, [], 1 << 70, None, None) is None
        assert native.linear8_forward(p, 0, 0, None, 3, "x", None, None, [], 1 << 70) is None
    for bad in (lambda: native.layer_plan(0, 8), lambda: native.layer_plan(0, 0, 4, 0, 0), lambda: native.layer_norm(plan), lambda: native.sample(plan, 0),
                lambda: native.layer_plan(0, "8", 4, 0, 0)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        native.layer_norm(native.embedding_plan(0, 2, 8, 0, 0), 0, 0, x, v, v, x, n, n)         # another plan


@pytest.mark.parametrize("source", SOURCES)
def test_the_kernels_keep_out_of_scratch_and_hold_no_packed_fp32(source):
    from paper_2004_14180_amd.build import device_assembly, device_resource_usage
    usage = device_resource_usage(source)
    assert usage
    for name, u in usage.items():
        assert u["scratch_bytes"] == 0, "%s: %d bytes of scratch per lane" % (name, u["scratch_bytes"])
    assert not re.findall(r"\bv_pk_(?:add|mul|fma)_f32\b", device_assembly(source))
