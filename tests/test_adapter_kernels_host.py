"""Kernels of one adapted row: every compiled one is one that some call takes."""
import re
import subprocess

from paper_2506_01206_amd import build


def test_no_kernel_for_columns_that_take_two_launches():
    """Two tiles of ranks beside the columns of one row go up to 6144 of them (768 workgroups and tiles); the streaming kernel starts at 8192."""
    names = subprocess.check_output(["nm", "-C", build.LIB], text=True)
    kernels = set(re.findall(r"linear_few_kernel<([^<>]*), [^<>,]*OneRowTail<(\d)>", names))
    assert {r for _, r in kernels} == {"1", "2"}
    stream = {r for args, r in kernels if args.endswith("true")}
    assert stream == {"1"}, kernels
