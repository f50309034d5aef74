"""The waits that the memory-to-LDS loads of the adapters' kernels owe to their source alone (see test_linear_waits_host.py): a wavefront waits for
its own LDS reads before a barrier behind which other wavefronts' loads overwrite what they read.  Device code before any optimisation."""
import os
import re
import subprocess

import pytest

from paper_2506_01206_amd import build
from test_linear_waits_host import counters

LIST = re.compile(r"@llvm\.amdgcn\.s\.waitcnt\(i32 (\d+)\)|call void @\S*(lds_barrier)\S*\(|call void @(\S*down_kernel\S*UliE_clEi)\(")


def functions(source, tmp_path):
    """name -> the function's waits (their immediates), barriers ("barrier") and calls of lambdas of one int ("wait"), in order"""
    out = tmp_path / (source + ".ll")
    flags = [f for f in build.FLAGS if f not in ("-O3", "-fPIC", "-Wall")]
    flags = flags[:flags.index("-mllvm")] + flags[flags.index("-mllvm") + 2:]      # (an option of the code generator)
    subprocess.check_call([build.HIPCC] + flags + ["-O3", "--cuda-device-only", "-S", "-emit-llvm", "-Xclang", "-disable-llvm-passes", "-w",
                                                   os.path.join(build.CSRC, source), "-o", str(out)])
    found = {}
    for body in re.findall(r"^define [^\n]*\n.*?^}", out.read_text(), re.S | re.M):
        name = re.search(r'@"?([\w.$]+)"?\(', body).group(1)
        found[name] = [int(a) if a else "barrier" if b else "wait" for a, b, c in LIST.findall(body.split("\n", 1)[1])]
    return found


def test_slabs_beside_a_product(tmp_path):
    """A stage is requested anew behind the second barrier of a turn."""
    multiply = {n: l for n, l in functions("linear.hip", tmp_path).items() if "AdapterSlabs" in n and "multiply" in n}
    assert len(multiply) >= 5
    for name, l in multiply.items():
        assert [x for x in l if x == "barrier"] == ["barrier"] * 2 and l[-1] == "barrier", (name, l)
        assert l[-2] != "barrier" and counters(l[-2])[1] == 0, (name, l)


def test_the_way_into_the_adapters(tmp_path):
    """Stages are requested behind the first barrier of an adapter, where the last one's sums have been read, and behind a slab's."""
    found = functions("adapters.hip", tmp_path)
    kernels = {n: l for n, l in found.items() if "down_kernel" in n and n.startswith("_ZN")}
    assert len(kernels) >= 5
    for name, l in kernels.items():
        assert l[1] == "barrier" and l[0] != "barrier" and counters(l[0])[1] == 0, (name, l)
        assert l[2:4] == ["wait", "barrier"] and l.count("wait") == 1, (name, l)
    waits = {n: [x for x in l if x != "barrier"] for n, l in found.items() if "down_kernel" in n and n.endswith("UliE_clEi")}
    assert len(waits) == len(kernels)
    for name, l in waits.items():
        assert len(l) == 3 and all(counters(x)[1] == 0 for x in l), (name, l)
