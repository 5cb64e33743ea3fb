"""Build the gfx950 HIP library in-tree: paper_2412_08521_amd/libems_hip.so.

hipcc cross-compiles without a GPU.  Usage:  python -m paper_2412_08521_amd.build
"""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
OBJ_DIR = os.path.join(_HERE, "_build")
LIB = os.path.join(_HERE, "libems_hip.so")
SOURCES = ["ems_api.hip", "score.hip", "score_m16.hip", "score_f32.hip", "select.hip", "merge.hip", "decode.hip", "stats.hip",
           "append.hip", "attend.hip", "prompt.hip"]
HEADERS = ["ems_common.h", "ems_kernels.h", "ems_red_weights.h", "ems_rows.h", "ems_score.h", "ems_stream.h", os.path.join("..", "..", "include", "ems.h")]
# the benchmark's ceiling measurements: a library of their own, outside the product's interface
PROBE_DIR = os.path.join(_HERE, "bench_probe")
PROBE_LIB = os.path.join(_HERE, "libems_probe.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         # packed-FP32 instruction selection is switched off for device code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function",
         # the LDS-DMA inline assembly names M0 as clobbered, which clang flags as reserved
         "-Wno-inline-asm"] + os.environ.get("EMS_EXTRA_HIPCC_FLAGS", "").split()
# These kernels read every accumulator element with the vector ALU: matrix results go to
# ordinary vector registers, never to the accumulation file (which the ALU cannot read).
_STREAM = ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-Rpass-analysis=kernel-resource-usage"]
FILE_FLAGS = {"score.hip": _STREAM, "score_m16.hip": _STREAM, "score_f32.hip": _STREAM, "stats.hip": _STREAM, "merge.hip": _STREAM[:2],
              "attend.hip": _STREAM[:2], "prompt.hip": _STREAM}
# Kernels that count their own vector-memory operations (s_waitcnt vmcnt(n) by hand around the
# LDS DMA): a register spill would add scratch loads/stores the count does not know about, so
# such a build is rejected instead of being allowed to run with a silent race.
NO_SCRATCH = {"score.hip": ("score_pass1", "score_pass2"), "score_m16.hip": ("score_pass1", "score_pass2"), "score_f32.hip": ("score_pass1", "score_pass2"), "stats.hip": ("redundancy_stream",),
              "prompt.hip": ("prompt_kernel",)}        # (whose waits for its DMA a spill's loads would make longer)


def _check_no_scratch(src: str, remarks: str) -> None:
    """Parse the compiler's kernel-resource-usage remarks; raise if a guarded kernel spills."""
    guarded = NO_SCRATCH.get(src, ())
    name, seen = None, set()
    for line in remarks.splitlines():
        if "remark:" not in line:
            continue
        text = re.sub(r"^\S+:\d+:\d+: ", "", line.split("remark:", 1)[1].strip()).strip()         # (the place comes before or after)
        if text.startswith("Function Name:"):
            name = text.split(":", 1)[1].split("[")[0].strip()
        elif name and any(g in name for g in guarded):
            # (a "VGPRs Spill" that costs no scratch went to the accumulation registers: moves, not memory)
            for key in ("ScratchSize [bytes/lane]:",):
                if text.startswith(key):
                    val = int(text[len(key):].split("[")[0].strip())
                    seen.add(name)
                    if val != 0:
                        raise RuntimeError(f"{src}: kernel {name} reports '{key} {val}'; the hand-counted "
                                           "s_waitcnt vmcnt() of its DMA pipeline requires zero scratch")
    if guarded and not seen:
        raise RuntimeError(f"{src}: no resource-usage remark found for kernels {guarded}")


# Kernels that write their own matrix products (inline assembly) into accumulation registers: the compiler does not know that
# these are products and keeps no distance between a vector instruction that writes an operand and the product that reads it.
OWN_PRODUCTS = {"prompt.hip"}


def _registers(text: str):
    """'v[0:3]' or 'a17' -> {('v', 0), ..}; anything else -> the empty set."""
    m = re.match(r"([va])(?:(\d+)$|\[(\d+):(\d+)\]$)", text.strip())
    if not m:
        return set()
    lo, hi = (int(m.group(2)),) * 2 if m.group(2) else (int(m.group(3)), int(m.group(4)))
    return {(m.group(1), i) for i in range(lo, hi + 1)}


def _check_own_products(src: str, assembly: str) -> None:
    """Raise if an operand of a product in inline assembly is written by a vector instruction less than two wait states before
    it (a label counts as unknown: the code there begins with a wait of its own), or if there is no such product."""
    seen, own, before = 0, False, []                       # before: (wait states, registers written) of what came before
    for line in assembly.splitlines():
        text = line.split(";")[0].strip() if "#ASM" not in line else line.strip()
        if "#ASMSTART" in text or "#ASMEND" in text:
            own = "#ASMSTART" in text
            continue
        if not text or text.startswith(("//", "#")):
            continue
        if text.endswith(":"):
            before = [(0, None)]
            continue
        if text.startswith("."):
            continue
        op, _, rest = text.partition(" ")
        args = re.findall(r"[vas]\[\d+:\d+\]|[va]\d+|[^,\s]+", rest)
        if own and op.startswith("v_mfma"):
            seen += 1
            reads, states = set().union(*(_registers(x) for x in args[1:])), 0
            for n, written in reversed(before):
                if states >= 2:
                    break
                if written is None or written & reads:
                    raise RuntimeError(f"{src}: an operand of `{text}` may be written less than two wait states before it")
                states += n
        if op == "s_nop":
            before.append((int(args[0], 0) + 1, set()))
        elif op.startswith("v_") and not op.startswith("v_mfma"):
            writes = _registers(args[0]) if args else set()
            if "swap" in op and len(args) > 1:
                writes |= _registers(args[1])
            before.append((1, writes))
        else:
            before.append((1, set()))
        before = before[-4:]
    if not seen:
        raise RuntimeError(f"{src}: no product in inline assembly found")


# Kernels in which a wave fills a ring in LDS for itself, by DMA, with no barrier between what it has read there and what it fills
# next: a read must have come to its registers before.  (Where a block's waves share a ring, a barrier lies between.)
OWN_RINGS = {"prompt.hip": r"prompt_kernelILi\d+ELb[01]ELb[01]ELi1ELi1ELi(?!1E)\d+E"}


def _blocks_of(assembly: str, names: str):
    """Every kernel whose name matches `names` -> its name, its basic blocks (label, instructions) in their order."""
    name, blocks = None, []
    for line in assembly.splitlines():
        text = line.split(";")[0].strip()
        if name is None:
            m = re.match(r"(\w+):", line)
            if m and re.search(names, m.group(1)):
                name, blocks = m.group(1), [("", [])]
        elif text.startswith(".Lfunc_end"):
            yield name, blocks
            name = None
        elif text.endswith(":"):
            blocks.append((text[:-1], []))
        elif text and not text.startswith((".", "#", "//")):
            blocks[-1][1].append(text)


def _check_reads_before_dma(src: str, assembly: str) -> None:
    """Raise if on some way through one of the kernels of OWN_RINGS a DMA to LDS may be issued while a transposed read of it is under
    way, or if there is no such kernel."""
    done, kernels = 1 << 30, 0
    for name, blocks in _blocks_of(assembly, OWN_RINGS[src]):
        kernels += 1
        number = {label: i for i, (label, _) in enumerate(blocks)}
        at, todo = {0: done}, [0]                          # LDS accesses since the last such read, at a block's begin; done: it is there

        def goes_on(block, since):
            if since < at.get(block, done + 1):
                at[block] = since
                todo.append(block)

        while todo:
            i = todo.pop()
            since, falls = at[i], i + 1 < len(blocks)
            for text in blocks[i][1]:
                op, _, rest = text.partition(" ")
                if op.startswith("ds_read_b64_tr"):
                    since = 0
                elif op.startswith("ds_") and since < done:
                    since += 1
                elif op == "s_waitcnt":                    # (they come in their order)
                    m = re.search(r"lgkmcnt\((\d+)\)", rest)
                    if m and int(m.group(1)) <= since:
                        since = done
                elif op == "global_load_lds_dwordx4" and since < done:
                    raise RuntimeError(f"{src}: {name} fills LDS (`{text}`) while a read of it may be under way")
                elif op.startswith(("s_cbranch", "s_branch")):
                    goes_on(number[rest.strip()], since)
                if op in ("s_branch", "s_endpgm"):
                    falls = False
                    break
            if falls:
                goes_on(i + 1, since)
    if not kernels:
        raise RuntimeError(f"{src}: no kernel with rings of its waves' own found")


def _stale(out: str, deps) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    hdrs = [os.path.normpath(os.path.join(CSRC, h)) for h in HEADERS]

    def compile_one(src):
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ_DIR, src.replace(".hip", ".o"))
        if force or _stale(o, [s] + hdrs):
            # with the assembly beside it, where that is looked at too, in a folder that does not stay
            temps = o.replace(".o", "_temps")
            obj = os.path.join(temps, os.path.basename(o)) if src in OWN_PRODUCTS else o
            if src in OWN_PRODUCTS:
                shutil.rmtree(temps, ignore_errors=True)
                os.makedirs(temps)
            cmd = [HIPCC] + FLAGS + FILE_FLAGS.get(src, []) + ["-c", s, "-o", obj] + (["-save-temps=obj"] if src in OWN_PRODUCTS else [])
            r = subprocess.run(cmd, capture_output=True, text=True)
            err = "\n".join(l for l in r.stderr.splitlines()
                            if "packed-fp32-ops' is not a recognized feature" not in l and not re.match(r"\d+ warnings? generated", l))
            if r.returncode != 0:
                raise RuntimeError(f"hipcc failed on {src}:\n{err}")
            try:                              # never link an object that fails a check
                if src in NO_SCRATCH:
                    _check_no_scratch(src, err)
                if src in OWN_PRODUCTS:
                    with open(obj.replace(".o", "-hip-amdgcn-amd-amdhsa-gfx950.s")) as f:
                        assembly = f.read()
                    _check_own_products(src, assembly)
                    _check_reads_before_dma(src, assembly)
            except RuntimeError:
                os.remove(obj)
                raise
            if src in NO_SCRATCH:
                err = "\n".join(l for l in err.splitlines() if "kernel-resource-usage" not in l
                                and not l.lstrip().startswith(("|", "^")) and "{" != l.strip()[-1:])
            if src in OWN_PRODUCTS:
                os.replace(obj, o)
                shutil.rmtree(temps)
            if verbose and err.strip():
                print(err, file=sys.stderr)
        return o

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    if force or _stale(LIB, objs):
        cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB + ".tmp"] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stderr}")
        os.replace(LIB + ".tmp", LIB)
    probe_src = os.path.join(PROBE_DIR, "probe.hip")
    if force or _stale(PROBE_LIB, [probe_src, os.path.join(PROBE_DIR, "ems_probe.h")] + hdrs):
        cmd = [HIPCC] + FLAGS + ["-shared", probe_src, "-o", PROBE_LIB + ".tmp"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on probe.hip:\n{r.stderr}")
        os.replace(PROBE_LIB + ".tmp", PROBE_LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
