"""Builds the HIP library (gfx950) in-tree with hipcc."""
import concurrent.futures
import glob
import os
import re
import shutil
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libtessel_hip.so")
SOURCES = ["tessel_kernels.hip", "tessel_wide.hip", "tessel_graph.hip", "tessel_mail.hip", "tessel_api.cpp",
           "tessel_attention.hip", "tessel_norm.hip", "tessel_checkpoint.hip", "tessel_weight.hip", "tessel_dropout.hip", "tessel_embedding.hip",
           "tessel_rotation.hip", "tessel_block_api.cpp"]
HEADERS = ["tessel_device.h", "tessel_common.h", os.path.join("..", "..", "include", "tessel.h"),
           "tessel_block.h", "tessel_tile.h", "tessel_rows.h", "tessel_draw.h", os.path.join("..", "..", "include", "tessel_block_ops.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-x", "hip",
    # packed FP32 instructions are kept out of every device code object of this build
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def is_stale():
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > built for f in SOURCES + HEADERS)


def _const(tok):
    try:
        return int(tok, 0)
    except ValueError:
        return None


def _word_aligned(reg, block, upto, depth=0, unknown=True):
    """Is scalar register `reg` (a number) visibly a multiple of four at line `upto` of the basic block `block`?
    Follows its latest definition inside the block: shifts left by two or more, multiples of four, sums of such;
    a register the block does not define came in whole (`unknown`: a pointer argument or a value checked elsewhere;
    not assumed of the factors of a product)."""
    if depth > 8:
        return False
    for k in range(upto - 1, -1, -1):
        t = block[k]
        m = re.search(r"\bs_lshl_b64\s+s\[(\d+):(\d+)\],\s*\S+,\s*(\S+)", t)
        if m and int(m.group(1)) <= reg <= int(m.group(2)):
            c = _const(m.group(3))
            return reg > int(m.group(1)) or (c is not None and c >= 2)
        m = re.search(r"\b(s_\w+|v_readfirstlane_b32|v_readlane_b32)\s+s(\d+),\s*(.*)$", t)
        if not m or int(m.group(2)) != reg:
            m2 = re.search(r"\bs_(?:buffer_)?load_\w+\s+s\[(\d+):(\d+)\]", t)
            if m2 and int(m2.group(1)) <= reg <= int(m2.group(2)):
                return True                                      # a pointer read from memory whole
            continue
        op, args = m.group(1), [a.strip() for a in m.group(3).split(",")]

        def ok(a, unknown=True):
            c = _const(a)
            if c is not None:
                return c % 4 == 0
            r = re.match(r"s(\d+)$", a)
            return bool(r) and _word_aligned(int(r.group(1)), block, k, depth + 1, unknown)
        if op == "v_readlane_b32":                               # a spilled scalar register coming back
            return True
        if op in ("s_lshl_b32",):
            c = _const(args[1]) if len(args) > 1 else None
            return c is not None and c >= 2
        if op in ("s_mul_i32",):
            return len(args) == 2 and (ok(args[0], False) or ok(args[1], False))
        if op in ("s_add_u32", "s_add_i32", "s_sub_u32", "s_sub_i32"):
            return len(args) == 2 and ok(args[0]) and ok(args[1])
        if op in ("s_mov_b32",):
            return len(args) == 1 and ok(args[0])
        return False
    return unknown


def misaligned_scalar_loads(asm):
    """Scalar loads of the device code whose address is not visibly a multiple of four: a register offset that its basic
    block does not show to be one (an index shifted left by two or more), or a base computed in its basic block from
    anything but indices shifted left by two or more or multiplied by a multiple of four.  The scalar memory path drops the low two bits of the base, so `base + i` with a byte index i, to which the
    compiler once added `3 i` as the offset of a load of word i, reads the wrong word.  (Seen in a variant of the
    completion kernel that read its per-type tables from global memory; the kernels keep such tables in LDS.)
    Returns the offending lines."""
    lines = asm.split("\n")
    bad = []
    start = 0                                                    # first line of the current basic block
    for n, line in enumerate(lines):
        if line.startswith(".L") or re.match(r"^\S+:", line):
            start = n + 1
            continue
        m = re.search(r"\bs_(?:buffer_)?load_\w+\s+\S+,\s+s\[(\d+):\d+\],\s*(\S+)", line)
        if not m:
            continue
        off = re.match(r"s(\d+)", m.group(2))
        if off and not _word_aligned(int(off.group(1)), lines[start:n], n - start, unknown=False):    # register offset
            bad.append("%d: %s" % (n + 1, line.strip()))
            continue
        if not _word_aligned(int(m.group(1)), lines[start:n], n - start):
            bad.append("%d: %s" % (n + 1, line.strip()))
    return bad


def _registers(text):
    """the vector and accumulation registers that an instruction's text names"""
    found = set()
    for m in re.finditer(r"\b([av])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        first, last = (m.group(2), m.group(3)) if m.group(2) else (m.group(4), m.group(4))
        found |= {(m.group(1), r) for r in range(int(first), int(last) + 1)}
    return found


# wait states between a matrix instruction of 8 passes and one of another kind that touches its result
_MFMA_WAIT = 11


def early_reads_of_products(asm):
    """Instructions of the device code that touch the result of a matrix instruction before it is written, along any path.  Nothing
    in the hardware holds them back; the compiler fills the time with other instructions and s_nop.  (Seen where accumulators were
    moved to other registers at the top of a loop that ended with the product: the way back was not counted, and the last registers
    of the result were read too early.)  Returns the offending lines."""
    code, label = [], {}
    for n, line in enumerate(asm.split("\n")):
        m = re.match(r"([^\s;]+):", line)
        if m:
            label[m.group(1)] = len(code)
            continue
        text = line.split(";")[0].strip()
        if text and not text.startswith("."):
            code.append((n + 1, text))
    bad = {}
    for i, (_, text) in enumerate(code):
        if not text.startswith("v_mfma"):
            continue
        result = _registers(text.split(",")[0])
        paths, seen = [(i + 1, 0)], {}
        while paths:
            j, waited = paths.pop()
            while j < len(code) and waited < _MFMA_WAIT and seen.get(j, _MFMA_WAIT) > waited:
                seen[j] = waited
                n, t = code[j]
                op = t.split()[0]
                if not op.startswith(("s_", "v_mfma")) and _registers(t) & result:
                    bad[n] = "%d: %s" % (n, t)
                waited += int(t.split()[1], 0) + 1 if op == "s_nop" else 8 if op.startswith("v_mfma") else 1
                if op.startswith("s_cbranch") and t.split()[1] in label:
                    paths.append((label[t.split()[1]], waited))
                if op in ("s_endpgm", "s_setpc_b64"):
                    break
                j = label.get(t.split()[1], len(code)) if op == "s_branch" else j + 1
    return [bad[n] for n in sorted(bad)]


def miscounted_reads(asm):
    """Places of the device code where a wait counts on more reads from memory than there are.  A kernel that waits for all but the last N
    of its reads (`s_waitcnt vmcnt(N) ; counted`) marks the stretches in which it starts them, `; counted reads begin` and `; counted reads
    end N`: each has to hold N of them, in one piece without labels or branches.  Fewer (merged, left out, moved away), and the wait ends
    while a read that it is for is still under way.  Returns the offending lines."""
    bad, begun, reads, stretches, waits = [], None, 0, 0, []
    for n, line in enumerate(asm.split("\n"), 1):
        mark = re.search(r"; counted reads (begin|end (\d+))", line)
        text = line.split(";")[0].strip()
        if mark and mark.group(2) is None:
            if begun:
                bad.append("%d: begins again inside the stretch of line %d" % (n, begun))
            begun, reads = n, 0
        elif mark:
            if not begun:
                bad.append("%d: ends without a beginning" % n)
            elif reads != int(mark.group(2)):
                bad.append("%d: %d reads since line %d, not %s" % (n, reads, begun, mark.group(2)))
            begun, stretches = None, stretches + 1
        elif begun and (re.match(r"[^\s;.]*\.?L?\w+:", line) or text.startswith(("s_cbranch", "s_branch", "s_endpgm", "s_setpc"))):
            bad.append("%d: %s in the stretch of line %d" % (n, text, begun))
            begun = None
        elif begun and text.startswith(("global_load", "buffer_load", "flat_load")):
            reads += 1
        if re.search(r"s_waitcnt vmcnt\(\d+\) ; counted", line):
            waits.append(n)
        if line.startswith(".Lfunc_end"):
            if begun:
                bad.append("%d: the stretch of line %d has no end" % (n, begun))
            if waits and not stretches:
                bad.append("%d: a counted wait, but no reads are marked" % waits[0])
            begun, stretches, waits = None, 0, []
    return bad


def build_library(force=True, verbose=False, check=True):
    """hipcc --offload-arch=gfx950 ... -> paper_2311_15269_amd/libtessel_hip.so.  With `check` the device assembly
    the compiler leaves behind is scanned for scalar loads at addresses that may not be word aligned, for results of matrix
    instructions that are touched too early and for reads that a wait counts on but that are not there."""
    if not force and not is_stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = tempfile.mkdtemp(prefix="tessel_build_")
    try:
        out = os.path.join(tmp, "libtessel_hip.so")
        # one object per source, compiled side by side (each in a folder of its own, which also takes what
        # -save-temps leaves behind), then one link
        def compile_one(src):
            work = os.path.join(tmp, os.path.splitext(src)[0])
            os.makedirs(work)
            obj = os.path.join(work, os.path.splitext(src)[0] + ".o")
            cmd = [hipcc] + HIPCC_FLAGS + (["-save-temps=obj"] if check else []) + ["-c", os.path.join(CSRC, src), "-o", obj]
            if verbose:
                print(" ".join(cmd))
            subprocess.check_call(cmd, cwd=work)
            return obj
        with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as pool:
            objs = list(pool.map(compile_one, SOURCES))
        link = [hipcc, "--offload-arch=gfx950", "--hip-link", "-shared", "-fPIC"] + objs + ["-o", out]
        if verbose:
            print(" ".join(link))
        subprocess.check_call(link, cwd=tmp)
        if check:
            listings = glob.glob(os.path.join(tmp, "*", "*gfx950*.s"))
            if not listings:
                raise RuntimeError("no device assembly found to check")
            for path in listings:
                asm = open(path).read()
                for what, bad in (("scalar loads at possibly unaligned addresses", misaligned_scalar_loads(asm)),
                                  ("results of matrix instructions touched too early", early_reads_of_products(asm)),
                                  ("reads from memory that a wait counts on", miscounted_reads(asm))):
                    if bad:
                        raise RuntimeError("%s in %s:\n%s" % (what, os.path.basename(path), "\n".join(bad[:10])))
        shutil.move(out, LIB)
    finally:
        shutil.rmtree(tmp, ignore_errors=True)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
