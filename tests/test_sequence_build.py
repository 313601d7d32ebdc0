"""CPU tests of what the compiler makes of the sequence layers' shared code."""
import re
import subprocess

import pytest

from paper_2008_04567_amd import build


@pytest.fixture(scope="module")
def ir(tmp_path_factory):
    d = tmp_path_factory.mktemp("ir")
    (d / "k.hip").write_text('''#include "wpk_seq.h"
__global__ void load_rows(const void *p, unsigned bytes, int *out)
{
    __shared__ int room[1024];
    const wpk::Rows rows = wpk::rows_at(p, 1, bytes);
    wpk::load_to_lds(rows, threadIdx.x * 16, 0, wpk::lds_offset(room));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    out[threadIdx.x] = room[threadIdx.x ^ 1];
}
''')
    subprocess.check_call([build._hipcc()] + build.COMMON + build.DEVICE +
                          ["--cuda-device-only", "-S", "-emit-llvm", str(d / "k.hip"), "-o", str(d / "k.ll")])
    return (d / "k.ll").read_text()


def test_loads_to_lds_say_that_they_write_m0(ir):
    calls = re.findall(r'asm sideeffect "([^"]*)", "([^"]*)"', ir)
    writes = [c for c in calls if re.search(r"\bm0\b", c[0])]
    assert writes, "no such load in the kernel"
    for text, constraints in writes:
        assert "~{m0}" in constraints.split(","), text
