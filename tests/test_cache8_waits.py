"""The instructions that the kernels of the 8-bit cache's attention write out: LDS reads, score products, factors on
accumulators.  The compiler does not see what they take, so it puts no waits before what reads or copies their results.
Here its output is read, instruction by instruction in its order:
 - nothing names the result of an LDS read before a wait that covers it;
 - nothing but a product that adds to it names a score product's result before the wait of the last products' statement, and
   no operand of one was written in the two instructions before it;
 - an accumulator that a factor is put on was written by a product longer ago than a product takes, or a barrier is between."""
import os
import re
import subprocess

import pytest

from test_product_waits import HIPCC, ROOT, WAIT, registers, statements

SETTLED = 20     # wait states from a 32x32x16 product to a reader of its result, and more


def check(lines):
    """Problems, and the numbers of LDS reads, score products and factors."""
    problems, seen = [], dict(reads=0, products=0, factors=0)
    queue = []                   # LDS and scalar operations on their way, in order: the registers they write, or None
    flight = set()               # results of score products
    recent = [set(), set()]      # written by the last two instructions
    since = SETTLED              # wait states since the last product
    for block in filter(None, statements(lines)):
        for text in block:
            op, _, rest = text.partition(" ")
            named = registers(rest)
            if op.endswith(":"):
                continue
            if op == "s_waitcnt":
                m = re.search(r"lgkmcnt\((\d+)\)", text)
                if m:
                    queue = queue[max(len(queue) - int(m.group(1)), 0):]
            early = [q for q in queue if q and q & named]
            if early:
                problems.append(f"{text}: names what an LDS read on its way writes")
            if op.startswith("ds_") or op.startswith(("s_load", "s_buffer_load")):
                reads = op.startswith(("ds_read", "ds_bpermute"))
                seen["reads"] += op.startswith("ds_read")
                queue.append(registers(rest.split(",")[0]) if reads else None)
            if op.startswith("v_mfma"):
                dst, a, b, c = rest.split(", ")
                if dst.startswith("v") and "32x32x16" in op:
                    seen["products"] += 1
                    if flight & (registers(a) | registers(b)):
                        problems.append(f"{text}: an operand is in flight")
                    if any(w & named for w in recent):
                        problems.append(f"{text}: an operand written right before")
                    if c not in (dst, "0"):
                        problems.append(f"{text}: does not add to its own result")
                    flight |= registers(dst)
                elif flight & named:
                    problems.append(f"{text}: names a score in flight")
                since = 0
            elif flight & named:
                problems.append(f"{text}: names a score in flight")
            if op.startswith(("s_cbranch", "s_branch", "s_endpgm", "s_setpc", "s_swappc")) and flight:
                problems.append(f"{text}: scores in flight over a branch")
            if op == "v_accvgpr_read_b32" and len(block) > 2:
                seen["factors"] += 1
                if since < SETTLED:
                    problems.append(f"{text}: {since} wait states after a product")
            if op in ("s_branch", "s_setpc_b64", "s_endpgm"):     # what follows is reached from elsewhere
                queue, since = [], SETTLED
            if op == "s_nop":
                n = int(rest) + 1
                recent = (recent + [set()] * n)[-2:]
                since += n
            else:
                recent = [recent[-1], registers(rest.split(",")[0]) if op.startswith("v_") and not op.startswith("v_mfma") else set()]
                since += 0 if op.startswith("v_mfma") else SETTLED if op == "s_barrier" else 1
        last = re.match(r"s_nop (\d+)$", block[-1]) if block[0].startswith("s_nop") and len(block) > 3 else None
        if last and int(last.group(1)) + 1 + sum(int(t.split()[1]) + 1 for t in block[-2:-1] if t.startswith("s_nop")) >= WAIT:
            flight = set()
    return problems, seen


def test_the_reading():
    asm = lambda *t: [";;#ASMSTART", *t, ";;#ASMEND"]
    read, wait = "ds_read_b128 v[20:23], v1 offset:64", "s_waitcnt lgkmcnt(0)"
    product = "v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], v[24:27], "
    last = asm("s_nop 1", product + "v[0:15]", product + "v[0:15]", "s_nop 15")
    accumulate = "v_mfma_f32_32x32x16_bf16 a[0:15], v[16:19], v[24:27], a[0:15]"
    factor = asm("v_accvgpr_read_b32 v40, a3", "v_mul_f32 v40, v40, v41", "v_accvgpr_write_b32 a3, v40")
    good = asm(read) + asm("ds_read_b32 v30, v1") + asm("s_waitcnt lgkmcnt(1)") + ["v_mov_b32_e32 v24, v20"] + asm("s_nop 1", product + "0") + \
        ["v_add_u32_e32 v31, v32, v33"] + last + ["v_mov_b32_e32 v50, v0", accumulate] + asm("s_waitcnt lgkmcnt(0)", "s_barrier") + factor
    assert check(good) == ([], dict(reads=2, products=3, factors=1))
    for bad in (asm(read) + ["v_mov_b32_e32 v24, v20"] + asm(wait),                      # read before the wait
                asm(read) + ["v_mov_b32_e32 v21, 0"] + asm(wait),                        # another use of its register
                asm(read) + asm("ds_read_b32 v30, v1") + asm("s_waitcnt lgkmcnt(2)") + ["v_mov_b32_e32 v24, v20"],
                ["v_mov_b32_e32 v24, v20"] + asm(product + "0") + last,                  # an operand right before
                asm(product + "0") + ["v_mov_b32_e32 v50, v3"] + last,
                asm(product + "0") + ["s_cbranch_vccnz .LBB0_1"] + last,
                asm("s_nop 1", product + "v[0:15]", product + "v[0:15]", "s_nop 7") + ["v_mov_b32_e32 v50, v3"],
                [accumulate] + factor):
        assert check(bad)[0], bad


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_nothing_touches_what_is_on_its_way(tmp_path):
    from paper_2609_03949_amd.csrc import build
    flags = [f for f in build.FLAGS if f != "-shared"]
    out = tmp_path / "k_chunk8.s"
    subprocess.run([HIPCC, *flags, "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S",
                    os.path.join(build.HERE, "k_chunk8.hip"), "-o", str(out)], check=True, capture_output=True)
    lines = out.read_text().split("\n")
    for rg in (1, 2, 4, 8):
        for kernel in ("run", "unit"):
            name = f"chunk8_{kernel}_kernel"
            start = next(i for i, l in enumerate(lines) if re.match(rf"_ZN3vkv\d+{name}ILi{rg}E\w*:", l))
            end = next(i for i in range(start, len(lines)) if lines[i].startswith(".Lfunc_end"))
            problems, seen = check(lines[start:end])
            assert not problems, (name, rg, len(problems), problems[:5])
            # 36 steps of 16 dims against two blocks of tile rows, for the first tile and in the loop; factors there and for the last tile
            assert seen["products"] == (2 * 2 * 36 if rg == 8 else 0), (name, rg, seen)
            assert seen["factors"] == {1: 8 * 4, 2: 4 * 16, 4: 4 * 2 * 16, 8: 2 * 4 * 4 * 16}[rg], (name, rg, seen)
            assert seen["reads"] >= 10 + 16          # a tile's keys and values
