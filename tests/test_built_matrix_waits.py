"""A matrix instruction's result is not read before it is there.

Whatever reads the result of v_mfma_f32_16x16x4_f32, other than as the sum it adds to, has to come ten wait states later, that of v_mfma_f32_16x16x32_bf16 eight.  The compiler inserts those, but it has been seen to leave
none where a branch ended with such an instruction and its result was read behind a block that holds a jump alone.  Here the assembly of the kernels that keep products in registers over branches
and loops is followed along every way for so many."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2409_11600_amd import build

WAITS = {"v_mfma_f32_16x16x4_f32": 10, "v_mfma_f32_16x16x32_bf16": 8}


def _registers(text):
    out = {k + str(i) for k, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text) for i in range(int(a), int(b) + 1)}
    return out | {k + a for k, a in re.findall(r"(?<![\w\[])([va])(\d+)\b", text)}


def _functions(text):
    name, found = None, {}
    for line in text.split("\n"):
        start = re.match(r"^(_Z\w+):", line)
        if start:
            name = start.group(1)
            found[name] = []
        elif name is not None:
            line = line.split(";")[0].strip()
            if line.startswith(".Lfunc_end"):
                name = None
            elif line and (not line.startswith(".") or line.endswith(":")):
                found[name].append(line)
    return found


def early_reads(code):
    """(matrix instruction, what reads its result too early, wait states between) of a function's lines."""
    labels, found = {line[:-1]: i for i, line in enumerate(code) if line.endswith(":")}, []

    def behind(i):
        op, *rest = code[i].split(None, 1)
        if op == "s_endpgm" or op == "s_setpc_b64":
            return []
        if op == "s_branch":
            return [labels[rest[0]]]
        return ([labels[rest[0].strip()]] if op.startswith("s_cbranch") else []) + ([i + 1] if i + 1 < len(code) else [])

    for i, line in enumerate(code):
        most = WAITS.get(line.split()[0])
        if most is None:
            continue
        todo, seen = [(j, 0, frozenset(_registers(line.split(None, 1)[1].split(",")[0]))) for j in behind(i)], {}
        while todo:
            j, waits, open_ = todo.pop()
            if waits >= most or not open_ or seen.get((j, open_), most) <= waits:
                continue
            seen[j, open_] = waits
            if code[j].endswith(":"):
                todo.append((j + 1, waits, open_))
                continue
            op, _, rest = code[j].partition(" ")
            parts = [p.strip() for p in re.split(r",(?![^\[]*\])", rest)]
            if op.startswith("v_mfma"):
                if (_registers(parts[1]) | _registers(parts[2])) & open_:
                    found.append((line, code[j], waits))
                    continue
                open_ = open_ - _registers(parts[0])
            elif op.startswith(("v_", "global_", "buffer_", "ds_", "flat_", "scratch_")):
                writes = not ("store" in op or "write_b" in op or "write2" in op)
                if _registers(",".join(parts[1:]) if writes else rest) & open_:
                    found.append((line, code[j], waits))
                    continue
                if writes:
                    open_ = open_ - _registers(parts[0])
            todo += [(k, waits + (int(rest) + 1 if op == "s_nop" else 1), open_) for k in behind(j)]
    return found


def test_finds_one():
    mfma = "v_mfma_f32_16x16x4_f32 a[0:3], v3, v45, a[0:3]"
    assert early_reads([mfma, "s_branch .L1", "v_mov_b32 v0, 0", ".L1:", "v_accvgpr_read_b32 v13, a3"]) == [(mfma, "v_accvgpr_read_b32 v13, a3", 1)]
    assert not early_reads([mfma, mfma, "s_nop 9", "v_accvgpr_read_b32 v13, a3"])
    assert early_reads([mfma, "s_nop 8", "buffer_store_dword a1, v18, s[68:71], 0 offen"])


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="no compiler")
def test_no_early_reads(tmp_path):
    out = tmp_path / "delta.s"
    subprocess.run(["hipcc", *build.FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, "delta.hip"), "-o", str(out)], check=True, capture_output=True)
    functions = _functions(out.read_text())
    for kind in WAITS:
        assert sum(any(line.startswith(kind) for line in code) for code in functions.values()) > 20
    for name, code in functions.items():
        assert not early_reads(code), name


@pytest.mark.skipif(shutil.which("nm") is None or not os.path.exists(build.LIB), reason="no symbols to read")
def test_every_chain_kernel_is_reached():
    """A head's chain of chunks without preparing wavefronts: four columns' wavefronts only where LDS does not hold two chunks (fp32 keys of more than 64), eight for all."""
    names = subprocess.run(["nm", build.LIB], check=True, capture_output=True, text=True).stdout
    for kernel in ("delta_fwd_kernel", "delta_ends_kernel"):
        found = {m.groups() for m in re.finditer(r"__device_stub__" + kernel + r"I(f|DF16b)Li(\d)ELi(\d)E", names)}
        assert found == {(t, d, "8") for t in ("f", "DF16b") for d in "248"} | {("f", "8", "4")}, kernel
