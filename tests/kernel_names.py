"""Which kernel a name stands for, with all of its template arguments: the profiler gives names as the compiler made them, or
demangled, in one of two ways that it has for 16-bit types."""
import re

MANGLED_TYPES = {"f": "f32", "DF16b": "bf16", "DF16_": "f16"}
SPELLED_TYPES = {"float": "f32", "__bf16": "bf16", "_Float16": "f16", "half": "f16"}


def parse(name):
    """(kernel, type, numbers and truth values as a tuple) of a kernel of this library, or None."""
    m = re.match(r"_ZN3wpk(\d+)", name)
    if m:
        at = m.end() + int(m.group(1))
        kernel, rest = name[m.end():at], name[at:]
        m = re.match(r"I(f|DF16b|DF16_)((?:L[ib]\d+E)*)E", rest)
        if not m:
            return None
        return kernel, MANGLED_TYPES[m.group(1)], tuple(int(v) for v in re.findall(r"L[ib](\d+)E", m.group(2)))
    m = re.fullmatch(r"void wpk::(\w+)<(.*)>\(wpk::\w+\)", name)
    if not m:
        return None
    args = m.group(2).split(", ")
    if args[:3] == ["bool _Accum", "int", "E"]:
        # a demangler that takes DF16b for another type and then "bLi1E" for the types of a bool and an int and a name of one letter:
        # so it goes where bf16 is followed by a 1, and by no other number
        ty, numbers = "bf16", ["1"] + args[3:]
    else:
        ty, numbers = SPELLED_TYPES.get(args[0]), args[1:]
    values = {"true": 1, "false": 0}
    if ty is None or not all(v in values or v.isdigit() for v in numbers):
        return None
    return m.group(1), ty, tuple(values[v] if v in values else int(v) for v in numbers)
