"""The wait states in front of the loads that prefix_attn.hip writes out by hand, in the assembly that its source compiles to.  A vector
instruction that writes a scalar register has to lie five wait states before a memory instruction that reads it (as any part of its
descriptor); the compiler counts them for its own instructions and not for inline asm."""
import os
import re
import subprocess

import pytest

from paper_2412_00061_amd import build

WAIT_STATES = 5


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name of a prefix_attn_kernel: its instructions, labels among them as ''}."""
    csrc, at = os.path.join(build.HERE, "csrc"), tmp_path_factory.mktemp("asm") / "p.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    said = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-I", os.path.join(build.ROOT, "include"), "-I", csrc,
                           "--cuda-device-only", "-S", os.path.join(csrc, "prefix_attn.hip"), "-o", str(at)], check=True, capture_output=True, text=True).stderr
    assert "-Winline-asm" not in said and not any("inline-asm" in f for f in flags)  # (silent where m0 is written, and only there)
    found = {}
    for name, body in re.findall(r"; -- Begin function (\S+)(.*?); -- End function", at.read_text(), re.S):
        if "prefix_attn_kernel" not in name:
            continue
        lines = [line.split(";")[0].strip() for line in body.split("\n")]
        found[name] = ["" if line.endswith(":") else line for line in lines if line and not line.startswith(".") or line.endswith(":")]
    return found


def scalars(operands):
    regs = {int(r) for r in re.findall(r"\bs(\d+)\b", operands)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", operands):
        regs |= set(range(int(a), int(b) + 1))
    return regs


def wait_states_before(code, at):
    """Wait states between instruction `at` and the nearest vector instruction before it, or place that a jump may lead to, that could have
    written one of its scalar registers (as its first operand, or as a carry, its second); WAIT_STATES if there is none that near."""
    reads, states = scalars(code[at]), 0
    for line in reversed(code[:at]):
        if states >= WAIT_STATES:
            break
        op, _, operands = line.partition(" ")
        if not line or (op.startswith("v_") and scalars(",".join(operands.split(",")[:2])) & reads):
            return states
        states += int(operands, 0) + 1 if op == "s_nop" else 1
    return min(states, WAIT_STATES)


def test_the_count_itself():
    load = "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"
    near = ["v_readfirstlane_b32 s6, v3", "s_mov_b32 m0, s9", "s_nop 0", load]
    assert wait_states_before(near, 3) == 2
    assert wait_states_before(["v_readlane_b32 s4, v3, 1", "s_mov_b32 m0, s9", "s_nop 3", load], 3) == 5
    assert wait_states_before(["v_readfirstlane_b32 s8, v3", "s_mov_b32 m0, s9", "s_nop 0", load], 3) == 3  # (nothing before it is known)
    assert wait_states_before(["", "s_nop 2", load], 2) == 3


def test_every_request_has_its_wait_states(kernels):
    assert len(kernels) == 20
    for name, code in kernels.items():
        requests = [i for i, line in enumerate(code) if line.startswith("buffer_load") and line.endswith("lds")]
        assert requests, name
        assert min(wait_states_before(code, i) for i in requests) == WAIT_STATES, name


def test_nothing_else_uses_m0(kernels):
    """Which the requests write: the register is reserved, so the compiler keeps nothing of its own safe there."""
    for name, code in kernels.items():
        for i, line in enumerate(code):
            if re.search(r"\bm0\b", line):
                assert line.startswith("s_mov_b32 m0, ") and code[i + 1].startswith("s_nop") and code[i + 2].endswith("lds"), (name, line)
