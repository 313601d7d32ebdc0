"""CPU tests of the reading of kernels' names, and that no form passes for another."""
import itertools

import pytest

from tests.kernel_names import parse

NAMES = [
    ("_ZN3wpk16linear_q8_kernelIDF16bLi128ELi128ELi2ELi4ELi2ELb1ELb0EEEvNS_6Q8ArgsE", ("linear_q8_kernel", "bf16", (128, 128, 2, 4, 2, 1, 0))),
    ("_ZN3wpk16linear_q8_kernelIDF16_Li64ELi128ELi1ELi4ELi2ELb0ELb0EEEvNS_6Q8ArgsE", ("linear_q8_kernel", "f16", (64, 128, 1, 4, 2, 0, 0))),
    ("void wpk::linear_q8_kernel<float, 64, 128, 1, 4, 2, false, true>(wpk::Q8Args)", ("linear_q8_kernel", "f32", (64, 128, 1, 4, 2, 0, 1))),
    ("void wpk::linear_q8_kernel<__bf16, 128, 128, 2, 4, 2, false, false>(wpk::Q8Args)", ("linear_q8_kernel", "bf16", (128, 128, 2, 4, 2, 0, 0))),
    ("void wpk::linear_q8_rows_kernel<bool _Accum, int, E, 2, 4, true, false>(wpk::Q8Args)", ("linear_q8_rows_kernel", "bf16", (1, 2, 4, 1, 0))),
    ("_ZN3wpk19grouped_rows_kernelIDF16_Li1ELi2ELi4ELb0EEEvNS_10LinearArgsE", ("grouped_rows_kernel", "f16", (1, 2, 4, 0))),
    ("_ZN3wpk18linear_join_kernelIDF16bEEvNS_10LinearArgsE", ("linear_join_kernel", "bf16", ())),
    ("void wpk::linear_join_kernel<float>(wpk::LinearArgs)", ("linear_join_kernel", "f32", ())),
]


@pytest.mark.parametrize("name,want", NAMES)
def test_names_are_read_whole(name, want):
    assert parse(name) == want


@pytest.mark.parametrize("name", ["", "linear_q8_kernel", "_ZN3wpk16linear_q8_kernelIdLi64EEEvNS_6Q8ArgsE", "_ZN3wpk16linear_q8_kernel",
                                  "void wpk::linear_q8_kernel<128, 1, 4, 2, false, false>(wpk::Q8Args)",
                                  "void wpk::linear_q8_kernel<E, 128, 1, 4, 2, false, false>(wpk::Q8Args)",
                                  "void other::linear_q8_kernel<float, 64, 128, 1, 4, 2, false, false>(other::Q8Args)"])
def test_names_that_hide_an_argument_are_no_form(name):
    assert parse(name) is None


def names_of(kernel, ty, numbers, bools):
    """As the compiler makes it, and as demanglers spell it."""
    letters, spelled = {"bf16": "DF16b", "f16": "DF16_", "f32": "f"}[ty], {"bf16": "__bf16", "f16": "_Float16", "f32": "float"}[ty]
    mangled = "_ZN3wpk%d%sI%s%s%sEEvNS_6Q8ArgsE" % (len(kernel), kernel, letters, "".join("Li%dE" % v for v in numbers),
                                                    "".join("Lb%dE" % v for v in bools))
    args = [str(v) for v in numbers] + ["true" if v else "false" for v in bools]
    out = [mangled, "void wpk::%s<%s>(wpk::Q8Args)" % (kernel, ", ".join([spelled] + args))]
    if ty == "bf16" and numbers[0] == 1:
        out.append("void wpk::%s<%s>(wpk::Q8Args)" % (kernel, ", ".join(["bool _Accum", "int", "E"] + args[1:])))
    return out


def test_every_form_is_told_from_every_other():
    tiles = [(64, 128, 1, 4, 2), (128, 128, 2, 4, 2), (256, 256, 2, 4, 2)]
    rows = [(mt, nt, u) for mt in (1, 2, 4) for nt in (1, 2, 3) for u in (1, 2)]
    forms = [(kernel, ty, numbers, bools) for kernel, some in (("linear_q8_kernel", tiles), ("linear_q8_rows_kernel", rows))
             for ty in ("bf16", "f16", "f32") for numbers in some for bools in itertools.product((0, 1), repeat=2)]
    read = {}
    for form in forms:
        for name in names_of(*form):
            got = parse(name)
            assert got == (form[0], form[1], form[2] + form[3]), name
            assert read.setdefault(got, form) == form
