"""The machine code that was built here for the training operators' ring kernels, on the CPU: the distances around the MFMAs that are written as
assembly, and that nothing between them waits for the loads into LDS but the barrier of a K step, which leaves all but one step under way."""
import os
import subprocess

import pytest

from test_kernel_code_cpu import LIB, OBJDUMP, code_objects, parse, violations


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(LIB):
        import __graft_entry__
        __graft_entry__.build()
    found = {}
    for i, obj in enumerate(code_objects(LIB)):
        if b"matmul_ring" not in obj:
            continue
        path = tmp_path_factory.mktemp("code") / ("%d.o" % i)
        path.write_bytes(obj)
        listing = subprocess.run([OBJDUMP, "-d", str(path)], capture_output=True, text=True, check=True).stdout
        found.update(parse(listing, "matmul_ring"))
    return found


def test_mfma_results_are_waited_for(kernels):
    assert len(kernels) >= 23
    bad = {name: violations(code) for name, code in kernels.items() if violations(code)}
    assert not bad, bad


def test_nothing_waits_for_the_loads_but_the_barrier(kernels):
    # loads per wave and step, and the steps that stay under way
    rings = {"Li256ELi256ELi5E": (8, 3), "Li128ELi128ELi5E": (4, 3), "Li64ELi128ELi6E": (3, 4), "Li128ELi128ELi3E": (12, 1), "Li64ELi128ELi4E": (9, 2)}
    for name, code in kernels.items():
        loads, steps = next(n for shape, n in rings.items() if shape in name)
        want = loads * steps
        mfmas = [i for i, ins in enumerate(code) if ins[1] == "v_mfma_f32_16x16x32_bf16"]
        loop = code[mfmas[0]:mfmas[-1]]
        waits = {ins[2] for ins in loop if ins[1] == "s_waitcnt" and "vmcnt" in ins[2]}
        assert waits == {"vmcnt(%d)" % want}, (name, waits)
        # three copies of a step are in the code: the two of the loop and the odd last one
        assert sum(ins[1] == "buffer_load_dwordx4" and "lds" in ins[2].split() for ins in loop) == 3 * loads, name
        assert not [ins for ins in loop if ins[1].startswith(("scratch_", "global_", "flat_", "buffer_store"))], name
