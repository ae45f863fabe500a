"""Loads in assembly: the compiler does not look inside, so the wait states that the hardware asks for stand in the assembly itself.  Between a vector instruction that writes a scalar register (a lane
read, which is how a spilled descriptor comes back) and a load that takes it: five; between a write of m0 and a load past the registers: one.  Whether the compiler puts such an instruction there
depends on the registers that it has left, so it is the text that is held to it."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_06003_amd", "csrc")
SOURCES = sorted(x for x in os.listdir(CSRC) if x.endswith((".hip", ".hpp", ".cpp")))


def statements(text):
    for m in re.finditer(r"\basm\s+volatile\s*\(|\basm\s*\(", text):
        end, depth = m.end(), 1
        while depth:
            depth += {"(": 1, ")": -1}.get(text[end], 0)
            end += 1
        yield text[m.end():end - 1]


@pytest.mark.parametrize("source", SOURCES)
def test_loads_wait_for_their_scalar_operands(source):
    with open(os.path.join(CSRC, source)) as f:
        for body in statements(f.read()):
            if not re.search(r"(buffer|global|flat|scratch)_(load|store|atomic)", body) or not re.search(r'"s"\s*\(|"\{s', body):
                continue
            states, lines = 0, "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', body.split(":")[0])).split(r"\n\t")
            for line in lines:
                if re.match(r"(buffer|global|flat|scratch)_", line):
                    break
                nop = re.match(r"s_nop (\d+)$", line)
                states += int(nop[1]) + 1 if nop else 1
            assert states >= 5, body


def test_there_are_such_loads():
    assert {"gated.hip", "attn.hpp"} <= {os.path.basename(x) for x in glob.glob(os.path.join(CSRC, "*")) if "buffer_load_dwordx4" in open(x).read()}
