"""The checks of test_isa_cpu.py on the kernels of the 8-bit caches and the normed appends."""
import pytest

import test_isa_cpu as isa


@isa.needs_hipcc
def test_no_mfma_under_exec_mask(tmp_path):
    bad, n_mfma = isa._mfmas_under_exec_mask(isa._assembly(tmp_path, "decode_q8.hip"))
    assert n_mfma > 0
    assert not bad, bad[:5]


@isa.needs_hipcc
@pytest.mark.parametrize("src", ["decode_q8.hip", "append_normed.hip", "cache_q8.hip"])
def test_kernels_do_not_spill(tmp_path, src):
    isa.test_kernels_do_not_spill(tmp_path, src)


@isa.needs_hipcc
@pytest.mark.parametrize("src", ["decode_q8.hip", "append_normed.hip", "cache_q8.hip"])
def test_no_packed_fp32(tmp_path, src):
    asm = isa._assembly(tmp_path, src)
    assert not any(x in asm for x in ("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32"))
