"""Build librose_delta.so for gfx950 with hipcc (in-tree, next to this file)."""
import os
import re
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librose_delta.so")
SOURCES = ["plan.cpp", "api.cpp", "ops_api.cpp", "kernels.hip", "embedding.hip", "grad.hip", "mx4.hip"]


DEVICE_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


_ELEMENTS = "_ZN4rose22encode_elements_kernelENS_10EncodeArgsE"


def _encode_kernel_bodies(asm):
    out, name, body = {}, None, []
    for line in asm.splitlines():
        m = re.match(r"^_ZN4rose13encode_kernelILi(\d)ELi(\d)ELi(\d)EEEvNS_10EncodeArgsE:", line)
        if m or line.startswith(_ELEMENTS + ":"):
            name, body = (int(m.group(1)), int(m.group(2)), int(m.group(3))) if m else _ELEMENTS, []
            continue
        if name is not None:
            if line.startswith(".Lfunc_end"):
                out[name] = body
                name = None
            else:
                body.append(line)
    return out


def _assembly(source, extra):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        s_path = os.path.join(tmp, "kernels.s")
        subprocess.check_call([hipcc] + DEVICE_FLAGS + list(extra) +
                              ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S",
                               os.path.join(CSRC, source), "-o", s_path], stderr=subprocess.DEVNULL)
        with open(s_path) as f:
            return f.read()


def check_reserved_vgpr(extra=()):
    """The encode kernels keep one VGPR out of the compiler's hands for the ticket that is in flight
    across iterations (see ticket_request in csrc/kernels.hip); the compiler is only ASKED to stay below
    it.  Compile the kernels to assembly and make sure that nothing but the two hand-written
    instructions ever names that register, that no kernel exceeds its register budget and that none
    spills: a toolchain or flag change that broke the reservation would hand out corrupt tickets.
    Raises RuntimeError on a violation."""
    bodies = _encode_kernel_bodies(_assembly("kernels.hip", extra))
    elements = bodies.pop(_ELEMENTS, None)
    if set(bodies) != {(f, r, a) for f in (0, 1) for r in (0, 1) for a in (0, 1)}:
        raise RuntimeError("not all eight encode kernels were found in the assembly: %s" % sorted(bodies))
    for (f32, refresh, arith), body in sorted(bodies.items()):
        _check_body("encode_kernel<%d, %d, %d>" % (f32, refresh, arith), body,
                    255 if (f32 and refresh and arith) else 167 if (f32 or arith) else 127)
    if elements is None:
        raise RuntimeError("the kernel that forms payloads of every element was not found in the assembly")
    _check_body("encode_elements_kernel", elements, 127)


def _check_body(what, body, reg):
    budget, uses = reg + 1, 0
    for line in body:
        code = line.split(";")[0]
        if not code.strip() or code.strip().startswith("."):
            continue
        for m in re.finditer(r"\bv(\d+)\b|\bv\[(\d+):(\d+)\]", code):
            lo = int(m.group(1)) if m.group(1) else int(m.group(2))
            hi = int(m.group(1)) if m.group(1) else int(m.group(3))
            if hi >= budget:
                raise RuntimeError("%s goes past its register budget: %s" % (what, code.strip()))
            if lo == hi == reg - 1 and re.match(r"\s*v_(writelane|readlane)_b32\b", code):
                continue        # the register below it: the compiler may park scalar registers there
            if lo <= reg <= hi or lo <= reg - 1 <= hi:
                # the reserved register (and otherwise the one below it) may only appear in the asm routines
                if not (re.search(r"global_atomic_add v%d, " % reg, code) or
                        re.search(r"v_mov_b32 v\d+, v%d\s*$" % reg, code)):
                    raise RuntimeError("%s: the compiler uses the reserved register: %s" % (what, code.strip()))
                uses += 1
        if "scratch_" in code:
            raise RuntimeError("%s spills: %s" % (what, code.strip()))
    if uses < 4:
        raise RuntimeError("%s: the ticket routines are missing (%d uses of v%d)" % (what, uses, reg))


def check_loads_to_lds(extra=()):
    """What the products' hand-written loads to LDS (load_to_lds in csrc/mx4.hip) assume of the compiler.  They set M0, which is
    not a register that the compiler lets assembly name as clobbered, so a use of its own that it sets up before such a load would
    find another value: make sure that nothing outside the hand-written assembly touches M0.  And they read scalar registers,
    which takes five wait states after a vector instruction has written them, inside assembly that the compiler does not
    look into: make sure that no such write is nearer.  Raises RuntimeError on a violation."""
    asm = _assembly("mx4.hip", extra)
    _check_m0(asm)
    _check_scalar_operands(asm)


def _by_hand(asm):
    """(whether it is hand-written, instruction or label) of the lines of an assembly"""
    by_hand = False
    for line in asm.splitlines():
        if "#ASMSTART" in line or "#ASMEND" in line:
            by_hand = "#ASMSTART" in line
            continue
        code = line.split(";")[0].strip()
        if code and (code.endswith(":") or not code.startswith(".")):
            yield by_hand, code


def _check_m0(asm):
    sets = 0
    for by_hand, code in _by_hand(asm):
        # by name, or by instructions that always read it: indexed moves, messages, counters, loads to LDS
        if re.search(r"\bm0\b|^s_movrel|^v_movrel|^s_set_gpr_idx|^s_sendmsg|^ds_gws|^ds_ordered|\blds$", code):
            if not by_hand:
                raise RuntimeError("the compiler uses M0: %s" % code)
            sets += code.startswith("s_mov_b32 m0")
    if not sets:
        raise RuntimeError("the loads to LDS are missing")


_SCALAR_WAIT = 5


def _scalars(operand):
    out = set()
    for m in re.finditer(r"\bs(\d+)\b|\bs\[(\d+):(\d+)\]", operand):
        out.update(range(int(m.group(1) or m.group(2)), int(m.group(1) or m.group(3)) + 1))
    return out


def _check_scalar_operands(asm):
    code = list(_by_hand(asm))
    # wait states since a vector instruction wrote each scalar register, where that is fewer than it takes; where branches meet the fewest
    at_label, changed = {}, True

    def meet(label, since):
        there = at_label.setdefault(label, {})
        nearer = {s: n for s, n in since.items() if n < there.get(s, _SCALAR_WAIT)}
        there.update(nearer)
        return bool(nearer)

    while changed:
        changed, since = False, {}
        for by_hand, line in code:
            if line.endswith(":"):
                changed |= meet(line[:-1], since)
                since = dict(at_label[line[:-1]])
                continue
            name, _, operands = line.partition(" ")
            operands = operands.split(",")
            if by_hand and name.startswith("buffer_load"):
                near = [s for s in set().union(*map(_scalars, operands)) if s in since]
                if near:
                    raise RuntimeError("a vector instruction wrote s%d too shortly before: %s" % (near[0], line))
            wait = int(operands[0], 0) + 1 if name == "s_nop" else 1
            since = {s: n + wait for s, n in since.items() if n + wait < _SCALAR_WAIT}
            if name.startswith("v_"):
                # (some have a carry or a flag for their second result)
                written = _scalars(operands[0]) | (_scalars(operands[1]) if len(operands) > 1 and re.search(r"_co_|div_scale|mad_[iu]64", name) else set())
                since.update((s, 0) for s in written)
            branch = re.match(r"s_c?branch\S*$", name)
            if branch:
                changed |= meet(operands[0].strip(), since)
                if name == "s_branch":
                    since = {}


def build(verbose=False, extra=(), out=None, check=True):
    """Compile the library; with check (the default) also verify what its hand-written assembly assumes
    of the compiler and refuse to leave a library behind that breaks it."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if check:
        check_reserved_vgpr(extra)
        check_loads_to_lds(extra)
    cmd = [hipcc] + DEVICE_FLAGS + ["-fPIC", "-shared", "-Wall", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    cmd += list(extra)
    for s in SOURCES:
        if s.endswith(".cpp"):
            cmd += ["-x", "hip", os.path.join(CSRC, s)]
        else:
            cmd += [os.path.join(CSRC, s)]
    cmd += ["-o", out or LIB]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return out or LIB


if __name__ == "__main__":
    build(verbose=True, extra=sys.argv[1:])
