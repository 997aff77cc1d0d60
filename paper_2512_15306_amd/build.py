"""Build libllmq.so (the gfx950 kernels and their C ABI) in-tree with hipcc, and the Python module over it with g++.  The library needs
nothing but hipcc: where the module does not build, the library is there without it (and llmq.py takes the ctypes path)."""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libllmq.so")
BINDING = os.path.join(HERE, "_binding.so")       # the Python module of csrc/binding.cpp
# gemm_tiles_*.hip: the tile kernels of one operand-kind pair and layout each (all tile shapes), so that they compile
# side by side; the largest come first.
TILE_SOURCES = ["gemm_tiles_e4m3_e4m3.hip", "gemm_tiles_e5m2_e4m3.hip", "gemm_tiles_e4m3_e5m2.hip", "gemm_tiles_e5m2_e5m2.hip",
                "gemm_tiles_e4m3_e4m3_abt.hip", "gemm_tiles_e4m3_e4m3_bt.hip", "gemm_tiles_e4m3_e4m3_at.hip",
                "gemm_tiles_e5m2_e4m3_abt.hip", "gemm_tiles_e5m2_e4m3_bt.hip", "gemm_tiles_e5m2_e4m3_at.hip",
                "gemm_tiles_bf16_bf16.hip"]
# the same for ragged shapes
TILE_SOURCES += ["gemm_edge_%s.hip" % kind for kind in
                 ("e4m3_e4m3", "e5m2_e4m3", "e4m3_e5m2", "e5m2_e5m2", "bf16_bf16",
                  "e4m3_e4m3_bt", "e5m2_e4m3_bt", "e4m3_e4m3_abt", "e5m2_e4m3_abt")]
# and for operands with block scales
TILE_SOURCES += ["gemm_blocks_%s.hip" % kind for kind in ("e4m3_e4m3", "e5m2_e4m3", "e4m3_e5m2", "e5m2_e5m2")]
# and for contractions joined with a SwiGLU
TILE_SOURCES += ["gemm_glu_%s.hip" % kind for kind in ("fwd_e4m3_e4m3", "fwd_e5m2_e4m3", "bwd_e4m3_e4m3", "bwd_e5m2_e4m3")]
SOURCES = TILE_SOURCES + ["gemm.hip", "gemm_blocks.hip", "gemm_glu.hip", "gemm_tmajor.hip", "quantize_blocks.hip", "api.hip", "amax.hip", "quantize.hip", "swiglu.hip", "rmsnorm.hip", "rmsnorm_blocks.hip", "rmsnorm_bwd.hip", "qk_norm_rope.hip", "adamw.hip", "calibrate.hip"]
# Sources that hold tile kernels (see check_accumulator_reads).
CHECKED_SOURCES = set(TILE_SOURCES) | {"gemm.hip"}
# Sources of kernels whose output may be one of their inputs (see check_in_place).
IN_PLACE_SOURCES = {src for src in TILE_SOURCES if src.startswith("gemm_glu_bwd_")}
# packed-fp32 VALU ops are disabled on purpose (they have produced silent wrong results on this
# hardware pool); never add -ffast-math: the scale needs a correctly rounded division.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wextra",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _registers(line: str):
    """The vector and accumulator registers an instruction names, as (file, number)."""
    found = {(f, int(n)) for f, n in re.findall(r"\b([av])(\d+)\b", line)}
    for f, lo, hi in re.findall(r"\b([av])\[(\d+):(\d+)\]", line):
        found.update((f, n) for n in range(int(lo), int(hi) + 1))
    return found


def check_accumulator_reads(src: str, asm: str) -> None:
    """The tile kernels write their MFMAs out as inline assembly, so the compiler does not know that an
    accumulator read must keep its distance from the MFMA that wrote it.  The kernels' own code keeps it: nothing
    but MFMAs touches the registers MFMAs write (accumulator registers, and in the largest tiles ordinary ones too) from the
    first MFMA to the wait states behind the K loop (`s_nop 15`).  Code the register allocator adds on its own (copies between
    the register files, spills of accumulators) would not, so any such instruction in that stretch of the generated assembly is
    a build error.  Allowed is the zeroing of the accumulators, which may be repeated on the path of a single K step, behind the K
    loop in the text: writes of an ordinary register to the accumulator file, and, in a block without MFMAs that only code in
    front of the first MFMA jumps to, to the ordinary registers among the accumulators."""
    bad = []
    checked = 0
    for m in re.finditer(r"^(_ZN4llmq16gemm_tile_kernel\w*):[^\n]*\n(.*?)^\.Lfunc_end", asm, re.S | re.M):
        name, body = m.group(1), m.group(2)
        code = [l.split(";")[0].strip() for l in body.splitlines()]
        code = [l for l in code if l and (not l.startswith(".") or l.startswith(".LBB")) and (not l.endswith(":") or l.startswith(".LBB"))]
        mfma = [i for i, l in enumerate(code) if l.startswith("v_mfma_")]
        if not mfma:
            continue                                  # the kernel that only adds up pieces
        checked += 1
        drain = next((i for i in range(mfma[-1], len(code)) if code[i] == "s_nop 15"), None)
        if drain is None:
            bad.append("%s: no wait states behind the last MFMA" % name)
            continue
        accumulators = {("a", n) for n in range(256)}
        for i in mfma:
            accumulators |= _registers(code[i].split()[1])
        label_at = {l[:-1]: i for i, l in enumerate(code) if l.endswith(":")}
        jumps = [(i, label_at[l.split()[-1]]) for i, l in enumerate(code) if re.match(r"s_c?branch", l) and l.split()[-1] in label_at]
        zeroing, end = set(), mfma[0]                 # lines of blocks that may zero accumulators
        for i in range(mfma[0], drain):
            if not code[i].endswith(":") or not re.match(r"s_branch|s_endpgm", code[i - 1]):
                continue
            end = next((k for k in range(i + 1, drain) if code[k].endswith(":") or re.match(r"s_c?branch", code[k])), drain)
            if all(k < mfma[0] for k, to in jumps if to == i) and not any(i < k < end for k in mfma):
                zeroing.update(range(i, end))
        for i in range(mfma[0], drain):
            l = code[i]
            if l.startswith("v_mfma_") or l.endswith(":") or not (_registers(l) & accumulators):
                continue
            if re.fullmatch(r"v_accvgpr_write_b32 a\d+, v\d+", l) and (i in zeroing or ("v", int(l.split("v")[-1])) not in accumulators):
                continue
            if i in zeroing and re.match(r"v_mov_b(32|64)_e32 ", l):
                continue
            bad.append("%s: %s" % (name, l))
            break
    if not checked:
        raise RuntimeError("%s: no tile kernel found in the generated assembly" % src)
    if bad:
        raise RuntimeError("%s: accumulator registers touched inside the MFMA stretch:\n  %s" % (src, "\n  ".join(bad)))


def check_scale_operands(src: str, asm: str) -> None:
    """The scaled MFMAs of the tile kernels are written out too, so the compiler keeps no distance between an ordinary vector instruction and the MFMA that reads
    what it wrote.  Their operands come from loads, which are waited for by counter, or from statements that end with wait states of their own; a copy or shift that the
    compiler adds on its own within the three instructions in front of such an MFMA is a build error."""
    bad = []
    for m in re.finditer(r"^(_ZN4llmq16gemm_tile_kernel\w*):[^\n]*\n(.*?)^\.Lfunc_end", asm, re.S | re.M):
        code = [l.split(";")[0].strip() for l in m.group(2).splitlines()]
        code = [l for l in code if l and (not l.startswith(".") or l.startswith(".LBB"))]
        for i, l in enumerate(code):
            if not l.startswith("v_mfma_scale_"):
                continue
            operands = _registers(l.split("op_sel")[0]) - _registers(l.split()[1])
            for before in code[max(0, i - 3):i]:
                if before.startswith("v_") and not before.startswith("v_mfma_") and _registers(before.split(",")[0]) & operands:
                    bad.append("%s: %s in front of %s" % (m.group(1), before, l))
    if bad:
        raise RuntimeError("%s: an operand of a scaled MFMA is written right in front of it:\n  %s" % (src, "\n  ".join(bad[:20])))


def _written(line: str):
    """The registers a vector instruction writes: its first operand, of a swap the second too."""
    operands = line.split(None, 1)[1].split(",") if " " in line else []
    return _registers(",".join(operands[:2 if "_swap_" in line.split()[0] else 1]))


# Wait states the compiler keeps on gfx950 between a buffer store of more than 8 bytes a lane and a vector instruction that writes its data.
STORE_WAIT_STATES = 2


def check_store_data(src: str, asm: str, wait_states: int = 1) -> None:
    """A buffer store of more than 8 bytes a lane reads its last registers after the next instructions have begun.  The compiler keeps STORE_WAIT_STATES between it and an instruction that writes
    them, but not where the store has a scalar offset, for which none is documented to be needed; on this hardware some are.  A write with fewer than `wait_states` in front of it, on any path from the
    store, is a build error.  An instruction is a wait state, s_nop N is N + 1."""
    bad = []
    for m in re.finditer(r"^(_ZN4llmq\w*):[^\n]*\n(.*?)^\.Lfunc_end", asm, re.S | re.M):
        code = [l.split(";")[0].strip() for l in m.group(2).splitlines()]
        code = [l for l in code if l and (not l.startswith(".") or l.startswith(".LBB"))]
        label_at = {l[:-1]: i for i, l in enumerate(code) if l.endswith(":")}
        for i, store in enumerate(code):
            if not re.match(r"buffer_store_dwordx[34] ", store):
                continue
            data, paths = _registers(store.split(",")[0]), [(i + 1, wait_states)]
            while paths:
                k, left = paths.pop()
                if left <= 0 or k >= len(code):
                    continue
                l = code[k]
                if l.endswith(":"):
                    paths.append((k + 1, left))
                    continue
                if l.startswith("v_") and _written(l) & data:
                    bad.append("%s: %s behind %s" % (m.group(1), l, store))
                    continue
                left -= int(l.split()[1], 0) + 1 if l.startswith("s_nop ") else 1
                if re.match(r"s_c?branch", l) and l.split()[-1] in label_at:
                    paths.append((label_at[l.split()[-1]], left))
                if not re.match(r"s_branch|s_endpgm|s_setpc", l):
                    paths.append((k + 1, left))
    if bad:
        raise RuntimeError("%s: registers of a buffer store written right behind it:\n  %s" % (src, "\n  ".join(bad[:20])))


def check_store_offsets(src: str, asm: str) -> None:
    """Rows and columns behind an output are dropped by the buffer's range, with which only the lane's offset of a store is documented to be compared.  A buffer store whose offset includes a
    scalar register is a build error."""
    bad = []
    for m in re.finditer(r"^(_ZN4llmq\w*):[^\n]*\n(.*?)^\.Lfunc_end", asm, re.S | re.M):
        for l in m.group(2).splitlines():
            store = re.match(r"\s*buffer_store_\w+ .*s\[\d+:\d+\], (\w+)", l)
            if store and store.group(1) != "0":
                bad.append("%s: %s" % (m.group(1), l.split(";")[0].strip()))
    if bad:
        raise RuntimeError("%s: buffer stores with a scalar offset:\n  %s" % (src, "\n  ".join(bad[:20])))


def check_in_place(src: str, asm: str) -> None:
    """A kernel that may write over one of its inputs must not promise the compiler otherwise.  The metadata calls a pointer write-only where it is declared apart from all others and only
    written: in these sources a build error."""
    bad = []
    for kernel in re.split(r"\n  - ", asm[asm.find("amdhsa.kernels:"):]):
        name = re.search(r"\.name:\s+(\S+)", kernel)
        for access, offset in re.findall(r"\.actual_access:\s+(\w+)\n(?:\s+\.\w+:\s+\w+\n)*?\s+\.offset:\s+(\d+)", kernel):
            if access != "read_only":
                bad.append("%s: the pointer at %s" % (name.group(1) if name else "?", offset))
    if "amdhsa.kernels:" not in asm:
        bad.append("no metadata in the generated assembly")
    if bad:
        raise RuntimeError("%s: an output is declared apart from the inputs that it may be:\n  %s" % (src, "\n  ".join(bad[:20])))


def check_counted_waits(src: str, asm: str) -> int:
    """The tile kernels wait for their direct-to-LDS loads by counting what they have requested since (a written-out `s_waitcnt vmcnt(N)`), so every other load must be there as often, and where, the
    kernel's own arithmetic has it: where the compiler makes one load of two, or drops some, a slab is read before it has landed.  Of the N newest requests in front of such a wait, on any path, no more
    may be loads to LDS than the stages that stay in flight have (gemm_tile_kernel: of two stages one, of four three in front of the loop, and one less in it; gemm_mini_kernel: as many of N as of the
    wait that leaves all stages but one in flight); others are a build error.  Returns the number of kernels it looked at."""
    bad = []
    checked = 0
    for m in re.finditer(r"^(_ZN4llmq16gemm_(?:tile|mini)_kernel\w*):[^\n]*\n(.*?)^\.Lfunc_end", asm, re.S | re.M):
        mini = "gemm_mini_kernel" in m.group(1)
        stages = 4 if ("ELi32E" if mini else "Deep") in m.group(1) else 2
        code, written_out = [], False                 # (kind, value): of what counts, and of the control flow
        for l in m.group(2).splitlines():
            if "#ASMSTART" in l or "#ASMEND" in l:
                written_out = "#ASMSTART" in l
                continue
            l = l.split(";")[0].strip()
            wait = re.match(r"s_waitcnt vmcnt\((\d+)\)$", l)
            if wait and written_out:
                code.append(("wait", int(wait.group(1))))
            elif re.match(r"(buffer|global|flat|scratch)_", l):
                code.append(("lds" if re.search(r" lds\b", l) else "vm", 0))
            elif re.match(r"\.LBB\w+:", l):
                code.append(("label", l[:-1]))
            elif re.match(r"s_c?branch", l):
                code.append(("jump" if l.startswith("s_branch") else "maybe", l.split()[-1]))
            elif l.startswith("s_endpgm"):
                code.append(("end", 0))
        waits = [i for i, (kind, n) in enumerate(code) if kind == "wait" and n > 0]
        slab = sum(kind == "lds" for kind, _ in code[:waits[0]]) // stages if waits else 0
        if not slab:
            continue                                  # operands through registers
        checked += 1
        jumps = {}
        for i, (kind, target) in enumerate(code):
            if kind in ("jump", "maybe"):
                jumps.setdefault(target, []).append(i)
        for i in waits:
            allowed = code[i][1] * (stages - 1) * slab // max(code[w][1] for w in waits) if mini else (stages - (1 if i == waits[0] else 2)) * slab
            paths, seen = [(i - 1, code[i][1], 0)], set()
            while paths:
                k, left, found = paths.pop()
                if (k, left, found) in seen or k < 0:
                    continue
                seen.add((k, left, found))
                kind, value = code[k]
                if kind in ("jump", "end"):
                    continue                          # (what falls through comes from elsewhere)
                if kind in ("vm", "lds"):
                    left, found = left - 1, found + (kind == "lds")
                    if found > allowed:
                        bad.append("%s: vmcnt(%d)" % (m.group(1), code[i][1]))
                        break
                    if left == 0:
                        continue
                if kind == "label":
                    paths += [(j - 1, left, found) for j in jumps.get(value, ())]
                paths.append((k - 1, left, found))
    if bad:
        raise RuntimeError("%s: a counted wait leaves loads to LDS on their way that are read behind it:\n  %s" % (src, "\n  ".join(bad[:20])))
    return checked


def check_few_rows_waits(src: str, asm: str) -> int:
    """The kernels for few rows count their requests too.  Each wave waits for its own loads only, and a step's loads stand in two branches of which one is taken, so check_counted_waits has no use for
    them; but as many steps stay in flight behind the last ones as were requested behind those, and no more: every multiple of a step's requests, up to all slots but one, is a written-out wait, and no other.
    Returns the number of kernels it looked at."""
    bad = []
    checked = 0
    for m in re.finditer(r"^(_ZN4llmq\d+gemm_(blocks|glu)_few_kernelI((?:L\w\d+E)+)E\w*):[^\n]*\n(.*?)^\.Lfunc_end", asm, re.S | re.M):
        numbers = [int(n) for n in re.findall(r"L\w(\d+)E", m.group(3))]
        slots = numbers[6] if m.group(2) == "glu" else 4
        if not re.search(r"^\s*buffer_load_\w+ .* lds\b", m.group(4), re.M):
            continue                                  # operands through registers
        checked += 1
        waits = sorted({int(n) for n in re.findall(r"#ASMSTART\n\s*s_waitcnt vmcnt\((\d+)\)\n", m.group(4))} - {0})
        if not waits or waits != [waits[0] * k for k in range(1, slots)]:
            bad.append("%s: vmcnt %s" % (m.group(1), waits))
    if bad:
        raise RuntimeError("%s: waits that do not count the steps in flight:\n  %s" % (src, "\n  ".join(bad[:20])))
    return checked


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    work = tempfile.mkdtemp(prefix="llmq_build_")
    try:
        return _build_in(work, hipcc, verbose)
    finally:
        shutil.rmtree(work, ignore_errors=True)


def binding_commands(obj: str, lib_dir: str, out: str):
    """Compile and link commands of the Python module (CPU code; the library is found beside it at run time)."""
    import torch
    root = os.path.dirname(torch.__file__)
    includes = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
    cxx = os.environ.get("CXX", "g++")
    abi = "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI)
    return ([cxx, "-O2", "-std=c++17", "-fPIC", "-Wall", abi] + [a for i in includes for a in ("-isystem", i)] + ["-c", os.path.join(CSRC, "binding.cpp"), "-o", obj],
            [cxx, "-shared", obj, "-o", out, "-L", lib_dir, "-lllmq", "-Wl,-rpath,$ORIGIN", "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])


def _run_binding(command):
    """A command of the module's build as a process, or None with a message where it cannot even start."""
    try:
        return subprocess.Popen(command, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    except OSError as e:
        print("%s: %s" % (command[0], e), file=sys.stderr)
        return None


def _finish_binding(process) -> bool:
    if process is None:
        return False
    out, _ = process.communicate()
    if process.returncode != 0:
        print(out, file=sys.stderr)
    return process.returncode == 0


def _build_in(work: str, hipcc: str, verbose: bool) -> str:
    objs = []
    procs = []
    new_lib, new_binding = os.path.join(work, "libllmq.so"), os.path.join(work, "_binding.so")
    compile_binding = link_binding = binding = None
    try:
        compile_binding, link_binding = binding_commands(os.path.join(work, "binding.o"), work, new_binding)
    except ImportError as e:                          # no PyTorch here
        print("binding.cpp: %s" % e, file=sys.stderr)
    if compile_binding:
        binding = _run_binding(compile_binding)
    for src in SOURCES:
        obj = os.path.join(work, src.replace(".hip", ".o"))
        cmd = [hipcc] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
        if src in CHECKED_SOURCES:
            cmd.append("-save-temps=obj")             # keeps the device assembly next to the object
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            failed = True
            print("FAILED: %s\n%s" % (src, out), file=sys.stderr)
        elif verbose and out.strip():
            print(out)
    binding_built = _finish_binding(binding)
    if failed:
        raise RuntimeError("hipcc failed")
    for src in sorted(CHECKED_SOURCES):
        with open(os.path.join(work, src.replace(".hip", "-hip-amdgcn-amd-amdhsa-gfx950.s"))) as f:
            asm = f.read()
        check_accumulator_reads(src, asm)
        check_scale_operands(src, asm)
        check_store_data(src, asm, STORE_WAIT_STATES)
        check_store_offsets(src, asm)
        check_counted_waits(src, asm)
        check_few_rows_waits(src, asm)
        if src in IN_PLACE_SOURCES:
            check_in_place(src, asm)
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", new_lib])
    binding_built = binding_built and _finish_binding(_run_binding(link_binding))
    # Both are there (or the module is not going to be): now they replace the old ones.  A module of another build must not stay
    # beside the new library.
    if os.path.exists(BINDING):
        os.remove(BINDING)
    _replace(new_lib, LIB)
    if binding_built:
        _replace(new_binding, BINDING)
    else:
        print("FAILED: binding.cpp: the calls of llmq.py take the ctypes path", file=sys.stderr)
    return LIB


def _replace(new: str, path: str) -> None:
    tmp = path + ".tmp.%d" % os.getpid()
    shutil.copy(new, tmp)
    os.replace(tmp, path)


if __name__ == "__main__":
    print(build(verbose=True))
