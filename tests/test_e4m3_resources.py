"""What the kernels of norms, 8-bit pages and attention over them may spend in registers and scratch: their launch rules count on it.  Read from
the metadata of the built library, no GPU needed."""
import pytest

from test_kernel_resources import kernels  # noqa: F401  (the fixture)
from test_matrix_waits import kernels as disassembly  # noqa: F401  (the fixture)
from test_matrix_waits import too_early


def test_attention_over_8_bit_pages_uses_no_scratch(kernels):  # noqa: F811
    names = [n for n in kernels if n.startswith(("e4m3_few_kernel<", "e4m3_chunk_kernel<"))]
    assert len(names) == 27
    assert {n: kernels[n][".private_segment_fixed_size"] for n in names} == dict.fromkeys(names, 0)


@pytest.mark.parametrize("d", [64, 128])
def test_eight_wavefronts_a_compute_unit(kernels, d):  # noqa: F811
    """Two wavefronts a SIMD have 256 registers each: what single tokens and bf16 chunks are planned with."""
    for name in [f"e4m3_few_kernel<unsigned short, {d}, {rb}, {ks}>" for rb in (1, 2) for ks in (1, 4, 8)] + [f"e4m3_chunk_kernel<unsigned short, {d}, 4>"]:
        assert kernels[name][".vgpr_count"] + kernels[name][".agpr_count"] <= 256, name


def test_rows_that_move_once_have_registers_for_their_workgroups(kernels):  # noqa: F811
    """2048 workgroups of 256 threads at a time are eight wavefronts a SIMD, 1536 six."""
    for t in ("unsigned short", "float"):
        assert kernels[f"norm_rope_kernel<{t}, 128, 0>"][".vgpr_count"] <= 64
        assert kernels[f"append_e4m3_kernel<{t}, 128, 0>"][".vgpr_count"] <= 84
    names = [n for n in kernels if n.startswith(("norm_rope_", "append_e4m3_kernel<"))]
    assert {n: kernels[n][".private_segment_fixed_size"] for n in names} == dict.fromkeys(names, 0)


def test_results_of_the_chunks_products_are_waited_for(disassembly):  # noqa: F811
    some = {n: code for n, code in disassembly.items() if "e4m3_chunk_kernel" in n}
    assert len(some) == 5
    assert {n: bad for n, bad in ((n, too_early(code)) for n, code in some.items()) if bad} == {}
