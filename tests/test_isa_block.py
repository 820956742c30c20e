"""What the assembly statements of the operators around the attention take for granted, checked in the compiler's output
for gfx950 (CPU only); the reader of the listing is the attention kernels'."""
import os
import re
import subprocess

import pytest

from paper_2502_01776_amd import build as B
from test_isa_waits import WAIT_STATES, parse

pytestmark = pytest.mark.skipif(not os.path.exists(B.hipcc_path()), reason="needs hipcc")


@pytest.fixture(scope="module", params=["svg_gate_norm.hip", "svg_fp4_linear.hip"])
def compiled(request, tmp_path_factory):
    out = str(tmp_path_factory.mktemp("isa") / "kernels.s")
    subprocess.run([B.hipcc_path(), *B.compile_flags(), "--offload-device-only", "-S", os.path.join(B.CSRC, request.param), "-o", out],
                   check=True, capture_output=True, text=True)
    kernels = parse(open(out).read())
    assert sum(len(k.direct_loads()) for k in kernels) > 0
    return request.param, kernels


def test_direct_loads_read_settled_scalar_registers(compiled):
    for k in compiled[1]:
        pred = k.predecessors()
        for at in k.direct_loads():
            n = k.nearest_vector_write(at, pred)
            assert n >= WAIT_STATES, f"{k.name}: {n} wait states in front of load {at}"


def test_m0_is_used_by_the_direct_loads_only(compiled):
    for k in compiled[1]:
        if k.direct_loads():
            other = [(op, args) for op, args, asm in k.ins if not asm and "m0" in args]
            assert not other, f"{k.name}: {other[:3]}"


def test_rows_on_their_way_are_not_waited_for(compiled):
    """Between a row's own count of outstanding operations and its last barrier the compiler waits for no load of its own: any such wait, or
    the reload of a spilt register, would wait for the rows ahead as well."""
    if compiled[0] != "svg_gate_norm.hip":
        pytest.skip("the ring of rows is the norm's")
    checked = 0
    for k in compiled[1]:
        forward = re.search(r"16gate_norm_kernelILi\dELi\dELi1ELi3ELNS0_4FormE0", k.name)
        if not forward and not re.search(r"21gate_norm_grad_kernelILi0ELi\dELi1ELi3ELNS0_4FormE0", k.name):
            continue
        waits = [i for i, (op, args, asm) in enumerate(k.ins) if asm and op == "s_waitcnt" and args[0].startswith("vmcnt(") and args[0] != "vmcnt(0)"]
        barriers = [i for i, (op, _, _) in enumerate(k.ins) if op == "s_barrier"]
        inside = [(op, args) for op, args, asm in k.ins[waits[-1] + 1:barriers[-1]] if not asm]
        bad = [(op, args) for op, args in inside if op.startswith("scratch_load") or (op == "s_waitcnt" and any("vmcnt" in a for a in args))]
        assert not bad, (k.name, bad)
        checked += 1
    assert checked == 8 + 2


def test_rows_of_every_type_depth_and_alignment_are_not_waited_for(compiled):
    """The same for every ring of one vector a lane: all types, one to three rows ahead, aligned rows and granules, with and without 4 bits.
    Gradients of two vectors have no ring."""
    if compiled[0] != "svg_gate_norm.hip":
        pytest.skip("the ring of rows is the norm's")
    checked = {"gate_norm_kernel": 0, "gate_norm_grad_kernel": 0}
    for k in compiled[1]:
        m = re.search(r"(gate_norm_kernel|gate_norm_grad_kernel)ILi\dELi\dELi(\d)ELi\dELNS0_4FormE(\d)E", k.name)
        if not m or m.group(3) == "2":
            continue
        assert m.groups()[:2] != ("gate_norm_grad_kernel", "2"), k.name
        if m.group(2) == "2":
            continue
        waits = [i for i, (op, args, asm) in enumerate(k.ins) if asm and op == "s_waitcnt" and args[0].startswith("vmcnt(") and args[0] != "vmcnt(0)"]
        barriers = [i for i, (op, _, _) in enumerate(k.ins) if op == "s_barrier"]
        inside = [(op, args) for op, args, asm in k.ins[waits[-1] + 1:barriers[-1]] if not asm]
        bad = [(op, args) for op, args in inside if op.startswith("scratch_load") or (op == "s_waitcnt" and any("vmcnt" in a for a in args))]
        assert not bad, (k.name, bad)
        checked[m.group(1)] += 1
    assert checked == {"gate_norm_kernel": 4 * 3 * 3, "gate_norm_grad_kernel": 4 * 3 * 2}
