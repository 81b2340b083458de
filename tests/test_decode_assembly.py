"""What decode.hip has to be compiled to, read from the assembly that the compiler makes of it.

- No kernel keeps anything in scratch memory.  (With matrix results in ordinary registers this compiler has made wrong code of a
  kernel that used accumulation registers and spilled.)
- The pipeline's second product is inline assembly, which the compiler does not take for a matrix instruction: it inserts no waits.
  Between what writes an operand of it and the product there have to be 2 wait states, between the product and anything but
  another product that touches its result 18 (the longest that a product of 16 x 16 asks for)."""
import os
import re
import subprocess

import pytest

from paper_2505_24179_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "decode.s")
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, "decode.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    text = open(out).read()
    names = re.findall(r"^\s+\.name:\s+(_ZN4sale\S*kernel\S*)$", text, re.M)
    scratch = re.findall(r"^\s+\.private_segment_fixed_size:\s+(\d+)$", text, re.M)
    bodies = {n: text.split(f"\n{n}:", 1)[1].split("\n.Lfunc_end", 1)[0].splitlines() for n in names}
    return dict(zip(names, map(int, scratch))), bodies


def test_nothing_is_spilled(kernels):
    scratch, _ = kernels
    assert len(scratch) >= 16
    assert not {n: b for n, b in scratch.items() if b}


def _registers(text, kind):
    found = {int(n) for n in re.findall(rf"\b{kind}(\d+)\b", text)}
    for a, z in re.findall(rf"\b{kind}\[(\d+):(\d+)\]", text):
        found |= set(range(int(a), int(z) + 1))
    return found


def test_inline_products_have_their_waits(kernels):
    checked = 0
    for name, body in kernels[1].items():
        at, inline = 0, False
        result, written = {}, {}      # wait state at which an inline product wrote, and another vector instruction
        for line in body:
            if "#ASMSTART" in line:
                inline = True
            elif "#ASMEND" in line:
                inline = False
            code = line.split(";")[0].strip()
            if not code or code.startswith(".") or code.endswith(":"):
                continue
            op, _, rest = code.partition(" ")
            args = [x.strip() for x in rest.split(",")]
            at += 1 + (int(args[0]) if op == "s_nop" else 0)
            if op.startswith("v_mfma") and inline:
                checked += 1
                sources = [("v", r) for r in _registers(",".join(args[1:3]), "v")] + [("a", r) for r in _registers(args[0], "a")]
                near = [r for r in sources if at - written.get(r, -99) - 1 < 2]
                assert not near, f"{name}: {code}: {near} written too shortly before"
                for r in _registers(args[0], "a"):
                    result[r] = at
                    written.pop(("a", r), None)
                continue
            touched = _registers(rest, "a")
            near = [r for r in touched if at - result.get(r, -99) - 1 < 18]
            assert not near, f"{name}: {code}: {near} too shortly after an inline product"
            if op.startswith("v_"):
                for kind in "va":
                    for r in _registers(args[0], kind):
                        written[kind, r] = at
                        if kind == "a":
                            result.pop(r, None)
    assert checked == 2 * 2 * 96      # bf16 and 8-bit pages, steps in one page or two, the products of two phases and the last ones


def test_keys_in_lds_have_their_waits(kernels):
    """The pipeline's keys go to LDS by loads that write there (L); the reads of them (R), which follow, need all of a step to have
    arrived, and what comes next to a buffer, that its reads have.  w, W: at most 8, 16 of the loads (P: others) are outstanding.  K: no
    read is."""
    phases = prologues = 0
    for name, body in kernels[1].items():
        blocks = [[]]
        for line in body:
            if re.match(r"\.LBB\S+:", line) or line.lstrip().startswith("; %bb."):
                blocks.append([])
            blocks[-1].append(line.split(";")[0].strip())
        for block in blocks:
            events = ""
            for code in block:
                vm, lgkm = re.search(r"vmcnt\((\d+)\)", code), re.search(r"lgkmcnt\((\d+)\)", code)
                if code.startswith("s_waitcnt"):
                    events += "w" if vm and int(vm[1]) <= 8 else "W" if vm and int(vm[1]) <= 16 else ""
                    events += "K" if lgkm and int(lgkm[1]) == 0 else ""
                elif code.startswith(("buffer_load", "global_load")):
                    events += "L" if code.endswith(" lds") else "P"
                elif code.startswith("ds_read_b128"):
                    events += "R"
            if "L" not in events:
                continue
            if sum(code.startswith("v_mfma") for code in block) >= 60:
                phases += 1
                assert re.fullmatch(r"K+L{8}[wW]+[RP]{16}", events) and events.count("R") == 8, (name, events)
            else:
                prologues += 1
                assert re.match(r"K*L{16}w+(?:RK*){8}(?<=K)L{8}P{8}[wW]+(?:RK*){8}", events), (name, events)
    assert (phases, prologues) == (4, 2)


def test_keys_lie_below_64_kb_of_lds(kernels):
    """A load to LDS takes its place from m0, documented as 16 bits: 8 KB times the wave's number and a constant here."""
    checked = 0
    for name, body in kernels[1].items():
        place = {}      # registers that hold 8 KB * wave and a constant
        for line in body:
            op, _, rest = line.split(";")[0].strip().partition(" ")
            args = [x.strip() for x in rest.split(",")]
            if op == "s_lshl_b32" and args[2] == "13":
                at = 0
            elif op in ("s_or_b32", "s_add_i32", "s_add_u32", "s_addk_i32") and args[-2] in place and re.fullmatch(r"0x[0-9a-f]+|\d+", args[-1]):
                at = place[args[-2]] + int(args[-1], 0)
            elif op == "s_mov_b32":
                at = place.get(args[1])
            else:
                at = None
            if op.startswith("s_"):
                if args[0] == "m0":
                    checked += 1
                    assert at is not None and 3 * 8192 + at + 1024 <= 65536, (name, line)
                for r in _registers(args[0], "s"):
                    place.pop(f"s{r}", None)
                if at is not None:
                    place[args[0]] = at
    assert checked == 2 * (16 + 8 + 16)      # a step in one page or two: before the loop 16 and 8, its two phases 8 each
