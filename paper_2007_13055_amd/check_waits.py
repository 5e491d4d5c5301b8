"""Whether compiled kernels leave a register alone between a load into it and the wait for that load.

Kernels that place the waits of their loads by hand issue them from inline assembly, and to the compiler such a register is
written at once: it may copy it (to an accumulation register, say) or use it for something else before the wait, and then the
load may still land in it.  This reads the AMD code of an object built here: along every path a load is in flight until an
s_waitcnt vmcnt(N) that at most N younger vector-memory operations leave, and no other instruction may name its registers.
(A later load into the same register is no fault: loads return in the order they were issued.)
"""
from __future__ import annotations

import os
import re
import subprocess
import tempfile

import numpy as np

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")

_REGISTERS = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")
_LINE = re.compile(r"^\t(\S+)(?: (.*?))?\s*// ([0-9A-F]+):(?: [0-9A-F]{8})+(?: <[^>]*?(?:\+0x([0-9a-f]+))?>)?\s*$")
_HEAD = re.compile(r"^([0-9a-f]+) <(.*)>:$")
_VMCNT = re.compile(r"vmcnt\((\d+)\)")
_LOADS = ("global_load", "flat_load", "buffer_load", "scratch_load")
_OTHERS = ("global_store", "flat_store", "buffer_store", "scratch_store", "global_atomic", "flat_atomic", "buffer_atomic")
_MOST, _LANDED = 64, 1 << 20                # operations since a register's load, counted so far (a wait's N is below it); none in flight


def _printed(obj: str, *tool) -> str:
    """What one of LLVM's tools prints of the AMD code in an object file that hipcc made."""
    with tempfile.TemporaryDirectory() as tmp:
        bundle, code = os.path.join(tmp, "bundle"), os.path.join(tmp, "code")
        run = lambda *cmd: subprocess.run([os.path.join(LLVM, cmd[0]), *cmd[1:]], check=True, capture_output=True, text=True).stdout  # noqa: E731
        run("llvm-objcopy", f"--dump-section=.hip_fatbin={bundle}", obj, os.devnull)
        run("clang-offload-bundler", "--type=o", "--unbundle", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={bundle}", f"--output={code}")
        return run(*tool, code)


def listing(obj: str) -> str:
    return _printed(obj, "llvm-objdump", "-d")


def accumulation_registers(obj: str) -> dict:
    """{kernel: accumulation registers that it takes}"""
    out, count = {}, 0
    for line in _printed(obj, "llvm-readelf", "--notes").splitlines():
        key, _, value = line.strip().removeprefix("- ").partition(":")
        if key == ".agpr_count":
            count = int(value)
        elif key == ".name" and "  - " not in line and value.strip().startswith("_Z"):
            out[value.strip()] = count
    return out


def kernels(text: str):
    """(name, first address, [(address, operation, operands, branch target's offset or None)]) of each function of a listing."""
    name, start, code = None, 0, []
    for line in text.splitlines():
        m = _LINE.match(line)
        if m:
            code.append((int(m.group(3), 16), m.group(1), m.group(2) or "", m.group(4)))
            continue
        m = _HEAD.match(line)
        if m:
            if name:
                yield name, start, code
            start, name, code = int(m.group(1), 16), m.group(2), []
    if name:
        yield name, start, code


def _registers(operands: str):
    out = []
    for kind, lo, hi, one in _REGISTERS.findall(operands):
        base = 0 if kind == "v" else 512
        out += range(base + int(lo), base + int(hi) + 1) if lo else [base + int(one)]
    return out


def _decoded(operation: str, operands: str):
    """(kind, registers named, registers that a load fills, N of a wait)"""
    if operation == "s_waitcnt":
        m = _VMCNT.search(operands)
        if m:
            return "wait", (), (), int(m.group(1))
        return ("wait", (), (), 0) if "cnt" not in operands else ("", (), (), 0)
    named = _registers(operands)
    if operation.startswith(_LOADS):
        if " lds" in operands or "_load_lds" in operation:
            return "memory", named, (), 0
        first, _, rest = operands.partition(",")
        return "load", _registers(rest), _registers(first), 0
    if operation.startswith(_OTHERS):
        return "memory", named, (), 0
    if operation == "s_endpgm":
        return "end", (), (), 0
    if operation == "s_branch" or operation.startswith("s_cbranch"):
        return "branch" if operation == "s_branch" else "either", (), (), 0
    return "", named, (), 0


def touched_in_flight(start: int, code, every_path: bool = False) -> list:
    """Addresses of the instructions that name a register whose load may still be in flight; every_path: is so on every path.

    For each register: how few (every_path: how many) vector-memory operations have been issued since its load, over all paths.  A
    wait for all but N ends the loads with N or more behind them; a register's own number decides, so that the extreme is exact.
    Paths are those of the branches whatever their conditions: where loads and waits hang on the same condition, only every_path tells."""
    merged, changed = (np.maximum, np.greater) if every_path else (np.minimum, np.less)
    index = {address: i for i, (address, *_) in enumerate(code)}
    cache, steps, leaders = {}, [], {0}
    for i, (_, operation, operands, offset) in enumerate(code):
        key = (operation, operands)
        if key not in cache:
            kind, named, filled, n = _decoded(*key)
            cache[key] = kind, np.array(named, dtype=np.int64), np.array(filled, dtype=np.int64), n
        kind = cache[key][0]
        target = index[start + int(offset or "0", 16)] if kind in ("branch", "either") else None
        steps.append((*cache[key], target))
        if target is not None:
            leaders |= {target, i + 1}
        elif kind == "end":
            leaders.add(i + 1)
    known, work = {0: np.full(1024, _LANDED, dtype=np.int64)}, [0]
    bad = {}                               # of each block, as it is known last
    while work:
        i = work.pop()
        state, follow, here = known[i].copy(), [], bad.setdefault(i, set())
        here.clear()
        flying = bool((state < _LANDED).any())
        while i < len(steps):
            kind, named, filled, n, target = steps[i]
            if kind == "wait":
                if flying:
                    state[state >= n] = _LANDED
                    flying = bool((state < _LANDED).any())
            else:
                if flying and len(named) and state[named].min() < _LANDED:
                    here.add(code[i][0])
                if kind == "load" or kind == "memory":
                    if flying:
                        state[state < _MOST] += 1
                    if kind == "load":
                        state[filled] = 0
                        flying = True
            if kind == "end":
                break
            if target is not None:
                follow.append(target)
            if kind == "branch":
                break
            i += 1
            if i in leaders:
                follow.append(i)
                break
        for j in follow:
            if j not in known:
                known[j] = state.copy()
            elif bool(changed(state, known[j]).any()):
                merged(known[j], state, out=known[j])
            else:
                continue
            work.append(j)
    return sorted(set().union(*bad.values()))


def check(obj: str, every_path: bool = False) -> dict:
    """{kernel: addresses} of the kernels of an object that touch a register in flight."""
    found = {}
    for name, start, code in kernels(listing(obj)):
        bad = touched_in_flight(start, code, every_path)
        if bad:
            found[name] = bad
    return found
