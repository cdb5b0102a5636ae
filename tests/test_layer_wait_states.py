"""The checks of test_wait_states.py on the kernels of libpf_layer.so (CPU only), with the rule for the 8-bit matrix product:
its result has to be left alone for twelve wait states (what the compiler puts behind it in straight code: eight
passes).  Its accumulator operand is always the constant zero here."""
import os

import pytest

import test_wait_states as w
from test_layer_host import LIB, layer  # noqa: F401  (fixture: builds / loads the library)

EIGHT_BITS = "v_mfma_f32_16x16x128_f8f6f4"


@pytest.fixture
def rules(layer, monkeypatch):  # noqa: F811
    if not os.path.exists(w.OBJDUMP):
        pytest.skip("no llvm-objdump")
    monkeypatch.setattr(w, "LIB", LIB)
    monkeypatch.setattr(w, "PRODUCTS", {**w.PRODUCTS, EIGHT_BITS: (12, 0)})


@pytest.mark.parametrize("between,missing", [(10, 2), (11, 1), (12, 0)])
def test_rule(rules, between, missing):
    body = [f"{EIGHT_BITS} v[0:3], v[8:15], v[16:23], 0", f"s_nop {between - 1}", "v_mov_b32_e32 v30, v1", "s_endpgm"]
    assert sum(w.missing_waits(body, {}).values()) == missing


def test_no_kernel_uses_a_result_too_early(rules, tmp_path):
    kernels = 0
    for listing in w._listings(tmp_path):
        for name, body, labels in w._functions(listing):
            kernels += any(t.startswith("v_mfma") for t in body)
            assert all(t.endswith(", 0") for t in body if t.startswith(EIGHT_BITS)), name
            early = w.missing_waits(body, labels)
            assert not early, (name, [(body[by], body[i], n) for (i, by), n in list(early.items())[:4]])
    assert kernels >= 4


def test_no_kernel_keeps_registers_in_memory(rules, tmp_path):
    for listing in w._listings(tmp_path):
        for name, body, _ in w._functions(listing):
            assert not [t for t in body if t.startswith("scratch_")], name
