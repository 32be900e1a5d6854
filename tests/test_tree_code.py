"""What the wide tree's attention was compiled to, read from the library that was built here: the waits around its assembly, as
test_prompt_code.py states them of the prompts', whose code it shares."""
import re

from test_prompt_code import _registers, _within
from test_qgemm_code import _instructions, code_objects  # noqa: F401  (a fixture)


def test_waits_around_the_maxima_are_stated(code_objects):
    kernels, read, bare = 0, 0, []
    for elf, path in code_objects:
        if b"kv_tree_wide_k" not in elf:
            continue
        for name, code in _instructions(path):
            if "kv_tree_wide_k" not in name:
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
