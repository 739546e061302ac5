"""The matrix products that weight_many_kernel writes as instructions: the compiler does not see them, so it inserts no wait
states before what reads or copies their results.  Here its output is read: from a product until the wait that the last
products' own statement ends with, nothing but a product that adds to the same registers names them."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
WAIT = 12       # wait states from a 32x32x16 product (8 passes) to a reader of its result on gfx950, as the compiler inserts them


def registers(text):
    out = set()
    for kind, lo, hi, one_kind, one in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        out |= {(kind, n) for n in range(int(lo), int(hi) + 1)} if kind else {(one_kind, int(one))}
    return out


def statements(lines):
    """The kernel's instructions in order, those of one asm statement together."""
    inside = None
    for line in lines:
        if "#ASMSTART" in line:
            inside = []
        elif "#ASMEND" in line:
            yield inside
            inside = None
        else:
            text = line.split(";")[0].strip()
            if not text or text.startswith(".") and not re.match(r"\.LBB\w+:", text):
                continue
            if inside is None:
                yield [text]
            else:
                inside.append(text)


def check(lines):
    """Problems, and the number of products."""
    flight, recent, problems, products = set(), [], [], 0
    for block in statements(lines):
        for text in block:
            op, _, rest = text.partition(" ")
            if op.endswith(":") or op.startswith(("s_cbranch", "s_branch")):
                if flight:
                    problems.append(f"{text}: results in flight over a branch")
                recent = []
            elif op.startswith("v_mfma"):
                products += 1
                dst, a, b, c = rest.split(", ")
                if flight & (registers(a) | registers(b)):
                    problems.append(f"{text}: an operand is in flight")
                if any(w & registers(text) for w in recent[-2:]):
                    problems.append(f"{text}: an operand written right before")
                if c not in (dst, "0") or flight & registers(dst) and c != dst:
                    problems.append(f"{text}: does not add to its own result")
                flight |= registers(dst)
                recent.append(set())
            else:
                if flight & registers(rest):
                    problems.append(f"{text}: touches a result in flight")
                recent.append(registers(rest.split(",")[0]) if op.startswith("v_") else set())
        if any(t.startswith("v_mfma") for t in block):
            last = re.match(r"s_nop (\d+)$", block[-1])
            if last and int(last.group(1)) + 1 >= WAIT:
                flight = set()
    return problems, products


def test_checker():
    product = "v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], a[0:3], "
    asm = lambda *t: [";;#ASMSTART", *t, ";;#ASMEND"]
    good = asm(product + "0") + ["v_add_u32_e32 v20, v21, v22"] + asm(product + "v[0:15]", "s_nop 13") + ["v_mov_b32_e32 v30, v0", ".LBB0_1:"]
    assert check(good) == ([], 2)
    for bad in (asm(product + "0") + ["v_mov_b32_e32 v30, v5"] + asm(product + "v[0:15]", "s_nop 13"),   # a copy between products
                asm(product + "0") + asm("s_nop 13") + ["v_mov_b32_e32 v30, v0"],                        # the wait in another statement
                asm(product + "0", "s_nop 7") + ["v_mov_b32_e32 v30, v0"],                               # too short a wait
                asm(product + "0") + ["s_cbranch_vccnz .LBB0_1"],
                ["v_accvgpr_write_b32 a0, v9"] + asm(product + "0", "s_nop 13"),
                asm(product + "v[32:47]", "s_nop 13")):
        assert check(bad)[0], bad


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_nothing_touches_a_result_in_flight(tmp_path):
    from paper_2609_03949_amd.csrc import build
    flags = [f for f in build.FLAGS if f != "-shared"]
    out = tmp_path / "k_weight.s"
    subprocess.run([HIPCC, *flags, "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S",
                    os.path.join(build.HERE, "k_weight.hip"), "-o", str(out)], check=True, capture_output=True)
    lines = out.read_text().split("\n")
    start = next(i for i, l in enumerate(lines) if re.match(r"_ZN3vkv18weight_many_kernel\w*:", l))
    end = next(i for i in range(start, len(lines)) if lines[i].startswith(".Lfunc_end"))
    problems, products = check(lines[start:end])
    assert not problems, problems[:5]
    assert products == 2 * 2 * 36        # two tiles (each form of the pair), two groups of rows, 36 steps of 16 dims
