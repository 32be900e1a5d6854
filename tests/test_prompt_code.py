"""What the prompts' attention was compiled to, read from the library that was built here: the waits around its assembly."""
import re

from test_qgemm_code import _instructions, code_objects  # noqa: F401  (a fixture)


def _registers(text):
    out = set()
    for lo, hi, one in re.findall(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", text):
        out |= set(range(int(lo), int(hi) + 1)) if lo else {int(one)}
    return out


def _within(code, i, reach):
    """Instructions that may follow the i-th within `reach`, path by path: the caller sends whether to go on."""
    index = {at: n for n, (at, _, _) in enumerate(code)}
    todo, seen = [(i, 0)], set()
    while todo:
        n, depth = todo.pop()
        for nxt in ([index[code[n][2]]] if code[n][2] is not None else []) + ([] if code[n][1].startswith(("s_branch", "s_endpgm")) else [n + 1]):
            if nxt in seen or nxt >= len(code) or depth >= reach:
                continue
            seen.add(nxt)
            if (yield code[nxt][1]):
                todo.append((nxt, depth + 1))
            yield


def test_waits_around_the_maxima_are_stated(code_objects):
    """The maxima are assembly, which the compiler's hazard pass does not look into.  Between a matrix step of four passes and a
    maximum that reads its result stand eight states of s_nop; between a maximum and a swap of lanes two."""
    kernels, read, bare = 0, 0, []
    for elf, path in code_objects:
        if b"kv_prompt_k" not in elf:
            continue
        for name, code in _instructions(path):
            if "kv_prompt_k" not in name:
                continue
            kernels += 1
            for i, (_, op, _) in enumerate(code):
                matrix, maximum = op.startswith("v_mfma"), re.match("v_max3?_f32", op)
                if not matrix and not maximum:
                    continue
                result, walk = _registers(op.split(",")[0]), _within(code, i, 40)
                for then in walk:
                    nop = re.match(r"s_nop (\d+)", then)
                    what, _, operands = then.partition(" ")
                    dest, _, sources = operands.partition(",")
                    reads = result & (_registers(operands) if "permlane" in what else _registers(sources))
                    on = not (nop and int(nop.group(1)) >= (7 if matrix else 1))
                    if on and reads and re.match("v_max3?_f32" if matrix else "v_permlane", what):
                        bare.append((name, op, then))
                    walk.send(on and not result & _registers(dest))
                read += matrix
    assert kernels == 28 and read and not bare, (kernels, bare[:3])
