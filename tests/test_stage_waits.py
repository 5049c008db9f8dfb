"""Loads to shared memory are written in assembly (csrc/stage.h), where the compiler puts no
waits of its own.  gfx950 wants 5 wait states between a vector instruction that writes a
scalar register and a memory instruction that reads it: the assembly that the compiler makes
of the kernels is searched for loads that come sooner, along every way that leads to them."""
import os
import re
import subprocess

from paper_2601_17091_amd import build_lib

SOURCES = ("linear8.hip", "weight_gradient.hip")
WAIT = 5


def scalars(operand):
    """The scalar registers of an operand."""
    m = re.match(r"s(?:\[(\d+):(\d+)\]|(\d+))$", operand)
    if not m:
        return set()
    return {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def kernels(text):
    """name -> [(opcode, operands)] with labels as ("label", [name])."""
    out, body = {}, None
    for line in text.splitlines():
        line = line.split(";")[0].strip()
        label = re.match(r"([.\w$]+):", line)
        if label:
            if not label[1].startswith("."):
                body = out.setdefault(label[1], [])
            elif body is not None:
                body.append(("label", [label[1]]))
        elif line and not line.startswith(".") and body is not None:
            op, _, rest = line.partition(" ")
            words = [w.strip().split() or [""] for w in rest.split(",")]
            body.append((op, [w[0] for w in words] + [w for w in words[-1][1:]]))
    return out


def too_soon(body):
    """Loads to shared memory, and those whose scalars a vector instruction wrote just before."""
    jumps = {}
    for i, (op, args) in enumerate(body):
        if op.startswith(("s_cbranch", "s_branch")):
            jumps.setdefault(args[0], []).append(i)

    def found(i, need, states):
        """Whether one of `need` is written at most WAIT - 1 - `states` wait states before i."""
        while states < WAIT and i > 0:
            i -= 1
            op, args = body[i]
            if op == "label":
                if any(found(j + 1, need, states) for j in jumps.get(args[0], [])):
                    return True
                if i == 0 or body[i - 1][0] in ("s_branch", "s_endpgm", "s_setpc_b64"):
                    return False   # nothing falls through to the label
                continue
            if op.startswith("v_") and args and scalars(args[0]) & need:
                return True
            states += int(args[0], 0) + 1 if op == "s_nop" else 1
        return False

    loads = [(i, args) for i, (op, args) in enumerate(body) if op.startswith("buffer_load") and "lds" in args]
    return loads, [(i, args) for i, args in loads if found(i, set().union(*map(scalars, args)), 0)]


def test_the_search_finds_what_it_looks_for():
    text = """
one:
  v_readfirstlane_b32 s2, v8
  s_mov_b32 s3, 0x20000
  s_mov_b32 m0, s57
  s_nop %d
  buffer_load_dwordx4 v159, s[0:3], s22 offen lds
  s_endpgm
two:
.LBB1_1:
  s_nop 1
  buffer_load_dword v1, s[4:7], 0 offen lds
  s_nop 4
  v_cmp_eq_u32_e64 s[6:7], v1, v2
  s_cbranch_scc1 .LBB1_1
  s_endpgm
"""
    for nop, sooner in ((0, 1), (1, 1), (2, 0), (4, 0)):
        loads, bad = too_soon(kernels(text % nop)["one"])
        assert len(loads) == 1 and len(bad) == sooner
    loads, bad = too_soon(kernels(text % 0)["two"])
    assert len(loads) == 1 and len(bad) == 1


def test_loads_to_shared_memory_wait_for_their_buffers(tmp_path):
    jobs = []
    for src in SOURCES:
        out = str(tmp_path / (src + ".s"))
        cmd = [build_lib.hipcc()] + build_lib.compile_flags(src) + [
            "--cuda-device-only", "-S", os.path.join(build_lib.CSRC, src), "-o", out]
        jobs.append((src, out, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    for src, out, job in jobs:
        said, _ = job.communicate()
        assert job.returncode == 0, said.decode(errors="replace")[-2000:]
    for src, out, _ in jobs:
        with open(out) as f:
            found = kernels(f.read())
        count = 0
        for name, body in found.items():
            loads, bad = too_soon(body)
            count += len(loads)
            assert not bad, "%s %s: %d of %d loads come too soon, the first %s" % (src, name, len(bad), len(loads), bad[0])
        assert count > 100, "no loads found in the assembly of " + src
