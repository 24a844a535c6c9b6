"""The pipelines of the block-scaled product change their accumulators by assembly MFMAs, which the compiler does not know as matrix
instructions: it places no wait between one and a read of its result.  matrix_results() is that wait.  The compiler's own output is
read here: on no way through a pipeline does an instruction other than an MFMA touch an accumulator that an MFMA has changed since
the last such wait.

The copies to LDS are assembly as well, and use m0 and scalar registers in ways that the compiler does not know of: it must have
no use of m0 of its own, and no vector instruction may write a copy's scalar registers less than five instructions in front of it."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WAIT = ["s_nop 15", "s_nop 7"]


def accumulators(operand):
    """Numbers of the accumulation registers that an operand names."""
    found = {int(n) for n in re.findall(r"\ba(\d+)\b", operand)}
    for lo, hi in re.findall(r"\ba\[(\d+):(\d+)\]", operand):
        found |= set(range(int(lo), int(hi) + 1))
    return found


def early_touches(body):
    """body: the lines of one kernel -> (MFMAs, waits, lines that touch an unsettled accumulator).  The unsettled registers flow along
    every branch until nothing changes."""
    lines = [s for s in (l.split(";")[0].strip() for l in body) if s and (s.endswith(":") or not s.startswith("."))]
    label = {s[:-1]: i for i, s in enumerate(lines) if s.endswith(":")}
    at = [None] * (len(lines) + 1)  # unsettled registers in front of each line, None: not reached
    at[0], todo, bad = frozenset(), [0], {}
    while todo:
        i = todo.pop()
        if i >= len(lines):
            continue
        s, state, onward = lines[i], at[i], [i + 1]
        op = s.split()[0]
        if op.startswith("v_mfma"):
            state = state | accumulators(s.split(",")[0])
        elif lines[i:i + 2] == WAIT:
            state = frozenset()
        elif not s.endswith(":") and accumulators(s) & state:
            bad[i] = s
        if op == "s_branch":
            onward = [label[s.split()[1]]]
        elif op.startswith("s_cbranch"):
            onward.append(label[s.split()[1]])
        elif op in ("s_endpgm", "s_setpc_b64"):
            onward = []
        for j in onward:
            new = state if at[j] is None else at[j] | state
            if new != at[j]:
                at[j] = new
                todo.append(j)
    waits = sum(lines[i:i + 2] == WAIT for i in range(len(lines)))
    return sum(s.startswith("v_mfma") for s in lines), waits, list(bad.values())


def test_the_reading_itself():
    mfma, wait, read = "v_mfma_x a[0:3], v[0:7], v[8:15], a[0:3]", "\n".join(WAIT), "v_accvgpr_read_b32 v0, a3"
    look = lambda *parts: early_touches("\n".join(parts).split("\n"))[2]  # noqa: E731
    assert look(mfma, wait, read, "s_endpgm") == []
    assert look(mfma, read, wait, "s_endpgm") == [read]
    assert look(mfma, "v_accvgpr_mov_b32 a64, a2", wait) == ["v_accvgpr_mov_b32 a64, a2"]
    assert look(mfma, "v_accvgpr_read_b32 v0, a4", "buffer_load_dwordx4 v1, s[0:3], 0 offen lds") == []
    # around a loop's back edge, and over a branch that passes by the wait
    assert look("top:", read, mfma, "s_cbranch_scc1 top", wait, "s_endpgm") == [read]
    assert look(mfma, "s_cbranch_scc1 past", wait, "past:", read, "s_endpgm") == [read]
    assert look(mfma, "s_branch past", read, "past:", wait, read, "s_endpgm") == []


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    from paper_2604_27089_amd import build
    out = tmp_path_factory.mktemp("asm") / "fp8_matmul.s"
    r = subprocess.run(["hipcc", *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, "fp8_matmul.hip"), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found, name = {}, None
    for line in out.read_text().split("\n"):
        m = re.match(r"^(_Z\w*matmul_\w*_kernel\w*):", line)
        if m:
            name = m.group(1)
            found[name] = []
        elif name and line.startswith(".Lfunc_end"):
            name = None
        elif name:
            found[name].append(line)
    return found


def test_results_are_read_behind_their_wait(kernels):
    pipes = {name: body for name, body in kernels.items() if "matmul_pipe_kernel" in name}
    assert len(pipes) == 8  # three tiles and the shared-out contraction, for two types each
    for name, body in pipes.items():
        mfmas, waits, bad = early_touches(body)
        assert mfmas >= 32 and waits == 1, (name, mfmas, waits)
        assert bad == [], f"{name}: {len(bad)} accumulators touched before their wait, first by `{bad[0]}`"


def scalars(operand):
    found = {int(n) for n in re.findall(r"\bs(\d+)\b", operand)}
    for lo, hi in re.findall(r"\bs\[(\d+):(\d+)\]", operand):
        found |= set(range(int(lo), int(hi) + 1))
    return found


def test_copies_have_their_registers(kernels):
    assert len(kernels) == 34  # the pipes, few rows in six ways and fp32 tiles, for two types and (few rows) two kinds of result
    for name, body in kernels.items():
        lines = [s for s in (l.split(";")[0].strip() for l in body) if s and not s.startswith(".") and not s.endswith(":")]
        copies = [i for i, s in enumerate(lines) if s.endswith(" lds") or s.startswith("global_load_lds")]
        assert copies, name
        for i in copies:
            assert lines[i - 2].startswith("s_mov_b32 m0, s") and lines[i - 1] == "s_nop 0", f"{name}: {lines[i - 2:i + 1]}"
            near = [s for s in lines[max(i - 5, 0):i] if s.startswith("v_") and scalars(s.split(",")[0]) & scalars(lines[i])]
            assert not near, f"{name}: `{near[0]}` in front of `{lines[i]}`"
        assert sum("m0" in re.findall(r"\bm0\b", s) for s in lines) == len(copies), f"{name}: m0 is used elsewhere"
