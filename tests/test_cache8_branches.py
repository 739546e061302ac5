"""The LDS reads that the kernels of the 8-bit cache's attention write out, followed along every way through the compiled
code, branches and loops included: nothing names the result of a read before a wait that covers it on the way there, and none
is on its way where a function is called or returns (it may copy or save registers that it does not know to be late)."""
import os
import re
import subprocess

import pytest

from test_product_waits import HIPCC, ROOT, registers, statements


def follow(lines):
    """Problems on all ways from the first line on, and the number of LDS reads seen."""
    code = [text for block in filter(None, statements(lines)) for text in block]
    at = {text[:-1]: i for i, text in enumerate(code) if text.endswith(":")}
    ends = set(at.values())                          # where other ways come in
    steps = []                                      # per instruction: op, what it names, what it waits for, what it sends out
    for text in code:
        op, _, rest = text.partition(" ")
        wait = re.search(r"lgkmcnt\((\d+)\)", text) if op == "s_waitcnt" else None
        sent = None
        if op.startswith(("ds_", "s_load", "s_buffer_load")):
            sent = frozenset(registers(rest.split(",")[0])) if op.startswith(("ds_read", "ds_bpermute", "ds_swizzle")) else frozenset()
        steps.append((op, frozenset(registers(rest)), int(wait.group(1)) if wait else None, sent, rest.strip()))
    # before an instruction: each register that a read on its way writes, and the fewest LDS and scalar operations issued behind
    # that read on any way there (where ways meet, the fewest: the wait that covers that one covers the others)
    before, problems, todo = {0: {}}, {}, [0]
    while todo:
        i = todo.pop()
        late = dict(before[i])
        while True:
            op, named, wait, sent, rest = steps[i]
            if wait is not None:
                late = {r: n for r, n in late.items() if n < wait}
            if named & late.keys():
                problems[i] = f"{code[i]}: names what an LDS read on its way writes"
            if late and op in ("s_swappc_b64", "s_setpc_b64"):
                problems[i] = f"{code[i]}: LDS reads on their way over a call"
            if sent is not None:
                late = {r: n + 1 for r, n in late.items()}
                late.update(dict.fromkeys(sent, 0))
            if op in ("s_endpgm", "s_setpc_b64"):
                break
            goes = [at[rest]] if op.startswith(("s_cbranch", "s_branch")) else []
            if op != "s_branch":
                goes.append(i + 1)
            if goes == [i + 1] and i + 1 not in ends:
                i += 1
                continue
            for j in goes:
                old = before.get(j)
                new = late if old is None else {r: min(n, old.get(r, n)) for r, n in {**old, **late}.items()}
                new = {r: min(n, late.get(r, n)) for r, n in new.items()}
                if new != old:
                    before[j] = new
                    todo.append(j)
            break
    reads, i, reached = 0, 0, set()
    for i in before:
        while i < len(steps) and i not in reached:
            reached.add(i)
            if steps[i][0].startswith(("s_endpgm", "s_setpc", "s_branch")):
                break
            i += 1
    return list(problems.values()), sum(steps[i][0].startswith("ds_read") for i in reached)


def test_the_following():
    read, wait, use = "ds_read_b128 v[20:23], v1", "s_waitcnt lgkmcnt(0)", "v_mov_b32_e32 v24, v20"
    end = ["s_endpgm"]
    assert follow([read, wait, use, *end]) == ([], 1)
    # one way waits, the other does not; the waiting one is elsewhere in the text
    assert follow([read, "s_cbranch_scc1 .LBB0_2", wait, ".LBB0_1:", use, *end, ".LBB0_2:", wait, "s_branch .LBB0_1"]) == ([], 1)
    assert follow([read, "s_cbranch_scc1 .LBB0_2", wait, ".LBB0_1:", use, *end, ".LBB0_2:", "s_nop 0", "s_branch .LBB0_1"])[0]
    # a block out of line that copies what is on its way
    assert follow([read, "s_cbranch_scc1 .LBB0_2", ".LBB0_1:", wait, use, *end, ".LBB0_2:", use, "s_branch .LBB0_1"])[0]
    # around a loop: the read of one turn, named in the next
    loop = [".LBB0_1:", use, read, "ds_write_b32 v1, v2", "s_cbranch_scc1 .LBB0_1", *end]
    assert follow(["s_nop 0", *loop])[0]
    assert follow(["s_nop 0", loop[0], "s_waitcnt lgkmcnt(1)", *loop[1:]]) == ([], 1)
    # a call, and a return
    assert follow([read, "s_swappc_b64 s[30:31], s[0:1]", wait, *end])[0]
    assert follow([read, wait, "s_swappc_b64 s[30:31], s[0:1]", *end]) == ([], 1)
    assert follow([read, "s_setpc_b64 s[30:31]"])[0]


def tile_loops(lines):
    """The innermost loops with matrix products: [first line, last line)."""
    at = {m.group(1): i for i, l in enumerate(lines) for m in [re.match(r"(\.LBB\w+):", l)] if m}
    back = {(at[m.group(1)], i) for i, l in enumerate(lines) for m in [re.match(r"\s+s_c?branch\w*\s+(\.LBB\w+)", l)] if m and at[m.group(1)] < i}
    loops = [(a, b) for a, b in back if any("v_mfma" in l for l in lines[a:b])]
    return [(a, b) for a, b in loops if not any(a <= x and y <= b for x, y in loops if (x, y) != (a, b))]


@pytest.fixture(scope="module")
def functions(tmp_path_factory):
    """Name and lines of each device function of the compiled file."""
    from paper_2609_03949_amd.csrc import build
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    flags = [f for f in build.FLAGS if f != "-shared"]
    out = tmp_path_factory.mktemp("asm") / "k_chunk8.s"
    subprocess.run([HIPCC, *flags, "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S",
                    os.path.join(build.HERE, "k_chunk8.hip"), "-o", str(out)], check=True, capture_output=True)
    lines = out.read_text().split("\n")
    starts = [i for i, l in enumerate(lines) if re.match(r"_ZN3vkv\w+:", l)]
    return [(lines[s].split(":")[0], lines[s + 1:next(i for i in range(s, len(lines)) if lines[i].startswith(".Lfunc_end"))]) for s in starts]


def test_every_way_waits(functions):
    found = 0
    for name, lines in functions:
        problems, reads = follow(lines)
        assert not problems, (name, len(problems), problems[:5])
        if re.search(r"chunk8_(run|unit)_kernel", name):
            found += 1
            assert reads >= 26, name                 # a tile's keys and values
    assert found == 8


def test_no_register_is_kept_in_memory_across_a_tile(functions):
    """A register that the compiler fetches from memory in the tile loop comes back with a wait for every load before it, the
    next tiles' among them."""
    found = 0
    for name, lines in functions:
        if re.search(r"chunk8_(run|unit)_kernel", name):
            loops = tile_loops(lines)
            found += 1
            assert len(loops) >= (2 if re.search("ILi[24]E", name) else 1), name      # units of 32 and 64 rows: scores, outputs
            for a, b in loops:
                assert not [l for l in lines[a:b] if "scratch_" in l], name
    assert found == 8
