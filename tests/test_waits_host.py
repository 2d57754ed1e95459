"""Between a matrix instruction and the first use of what it writes lie as many wait states as gfx950 wants, over every way through the code of
every kernel of the built library.

The compiler sets these waits, but where two ways of different length meet between the two instructions it has been seen to count the longer one;
the kernels that have such places wait by hand.  This walks the disassembled kernels, so that a kernel without that, or another compiler's
code, does not bring the fault back.
"""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import paper_2407_09453_amd as bsp
from test_resources_host import _code_objects

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# wait states before another instruction touches the result: two more than its passes of four clocks in fp32, four more otherwise
KINDS = {"16x16x32_bf16": 4 + 4, "32x32x16_bf16": 8 + 4, "16x16x64_i8": 4 + 4, "16x16x32_i8": 4 + 4, "16x16x128_f8f6f4": 8 + 4, "32x32x64_f8f6f4": 16 + 4,
         "4x4x1_16b_f32": 2 + 2, "16x16x4_f32": 8 + 2}


def _registers(operands):
    out = set()
    for kind, a, b, c in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operands):
        out.update((kind, i) for i in (range(int(a), int(b) + 1) if a else [int(c)]))
    return out


def _kernels(text):
    """(name, [(address, operation, operands, where it branches to)]) of a disassembly."""
    name, body = None, []
    for line in text.splitlines():
        m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if m:
            if body:
                yield name, body
            name, body = m.group(1), []
            continue
        m = re.match(r"^\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):.*?(?:<\S+?\+0x([0-9a-f]+)>)?$", line)
        if m:
            body.append((int(m.group(3), 16), m.group(1), m.group(2), int(m.group(4), 16) if m.group(4) else None))
    if body:
        yield name, body


def _near(body, most=24):
    """{operation: (fewest states before its result is touched, by what)} of one kernel."""
    base = body[0][0]
    at = {address: i for i, (address, _, _, _) in enumerate(body)}
    touched, worst = {}, {}

    def touches(i):
        if i not in touched:
            touched[i] = _registers(body[i][2])
        return touched[i]
    for i, (_, op, operands, _) in enumerate(body):
        if not op.startswith("v_mfma"):
            continue
        kind = next((k for k in KINDS if k in op), op)
        best, ways = {}, [(i + 1, 0, frozenset(_registers(operands.split(",")[0])))]
        while ways:
            p, states, result = ways.pop()
            while p < len(body) and result and states < most and best.get((p, result), most) > states:
                best[p, result] = states
                _, o, args, to = body[p]
                used, after = touches(p) & result, result
                if used and o.startswith("v_mfma"):
                    onto, *factors, sums = [_registers(a) for a in re.split(r",(?![^\[]*\])", args)[:4]]
                    if sums == result or onto == result:  # a sum that goes on as one is the matrix unit's own affair, from there on with a walk of its own
                        used, after = set().union(*factors) & result, result - onto
                if used:
                    worst[kind] = min(worst.get(kind, (most, "")), (states, o + " " + args))
                    break
                result = after
                if o in ("s_endpgm", "s_setpc_b64", "s_swappc_b64"):
                    break
                states += int(args, 0) + 1 if o == "s_nop" else 1
                if o == "s_branch":
                    p = at[base + (to or 0)]
                    continue
                if o.startswith("s_cbranch"):
                    ways.append((at[base + (to or 0)], states, result))
                p += 1
    return worst


def test_the_walk_sees_what_it_is_for():
    """Straight code with its wait, a branch around the wait, a loop that comes back to a use, and an operand that is the result."""
    def body(*lines):
        return [(4 * i, *line) for i, line in enumerate(lines)]
    mfma = ("v_mfma_f32_32x32x16_bf16", "v[0:15], v[20:23], v[24:27], 0", None)
    use, end, other = ("v_add_f32_e32", "v40, v3, v41", None), ("s_endpgm", "", None), ("v_mov_b32_e32", "v50, v51", None)
    assert _near(body(mfma, ("s_nop", "11", None), use, end)) == {"32x32x16_bf16": (12, "v_add_f32_e32 v40, v3, v41")}
    assert _near(body(mfma, ("s_cbranch_scc1", "1", 12), ("s_nop", "15", None), use, end))["32x32x16_bf16"][0] == 1
    assert _near(body(mfma, ("s_nop", "7", None), ("s_branch", "", 20), use, end, other, ("s_branch", "", 12)))["32x32x16_bf16"][0] == 11
    assert _near(body(mfma, mfma, end)) == {}
    onward = ("v_mfma_f32_32x32x16_bf16", "v[2:17], v[20:23], v[24:27], v[0:15]", None)
    assert _near(body(mfma, onward, ("s_nop", "15", None), use, end)) == {"32x32x16_bf16": (16, "v_add_f32_e32 v40, v3, v41")}
    assert _near(body(mfma, onward, ("v_add_f32_e32", "v40, v1, v41", None), ("s_nop", "15", None), use, end))["32x32x16_bf16"][0] == 1
    assert _near(body(mfma, ("v_mfma_f32_32x32x16_bf16", "v[0:15], v[4:7], v[24:27], 0", None), end))["32x32x16_bf16"][0] == 0


@pytest.mark.skipif(not os.path.exists(OBJDUMP) or not shutil.which("hipcc"), reason="no ROCm toolchain")
def test_results_of_matrix_instructions_are_waited_for(tmp_path):
    def of(n, co):
        f = tmp_path / ("%d.co" % n)
        f.write_bytes(co)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(f)], capture_output=True, text=True, check=True).stdout
        return [(name, body) for name, body in _kernels(text) if any(op.startswith("v_mfma") for _, op, _, _ in body)]
    with ThreadPoolExecutor(4) as pool:
        kernels = sum(pool.map(lambda a: of(*a), enumerate(_code_objects(open(bsp.binding.lib_path(), "rb").read()))), [])
    assert len(kernels) > 100, len(kernels)
    assert any("f8_wide_low" in name for name, _ in kernels) and any("adapt_grad" in name for name, _ in kernels)
    for name, body in kernels:
        for kind, (states, use) in _near(body).items():
            assert states >= KINDS[kind], (name, kind, states, use)
