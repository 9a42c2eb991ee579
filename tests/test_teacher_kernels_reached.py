"""Kernels that learn from a teacher which the rules of a call never choose are not in the library (CPU only)."""
import re

from test_kernel_resources import kernels  # noqa: F401


def instances(kernels, name):  # noqa: F811
    """(type, template's numbers) of a kernel's instances."""
    found = set()
    for symbol in kernels:
        m = re.search(rf"\d+{name}IN4ccdc\d+(Elem\w+?)E((?:L[ib]\d+E)+)E", symbol)
        if m:
            found.add((m[1], tuple(int(v) for v in re.findall(r"L[ib](\d+)E", m[2]))))
    return found


def test_several_groups_for_nine_rows_and_more_are_those_of_fp32_results(kernels):  # noqa: F811
    """16-bit results go by tiles from 9 rows of x on where the weights have 8192 or more."""
    few = instances(kernels, "k_few8")
    assert {kind for kind, _ in few} == {"ElemF32", "ElemBF16", "ElemF16"}
    assert {kind for kind, numbers in few if numbers == (1, 1, 4, 4, 2)} == {"ElemF32"}


def test_rows_of_eight_packs_by_sixteen_wavefronts_are_those_of_fp32_logits(kernels):  # noqa: F811
    """16-bit rows of that length are held in registers and LDS."""
    rows = instances(kernels, "k_distill")
    assert {kind for kind, _ in rows} == {"ElemF32", "ElemBF16", "ElemF16"}
    assert {kind for kind, numbers in rows if numbers == (16, 8, 0, 0)} == {"ElemF32"}
    assert {kind for kind, numbers in rows if numbers == (16, 4, 4, 0)} == {"ElemBF16", "ElemF16"}
