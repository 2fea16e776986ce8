"""Operators of a conditioned predictor block, without a GPU: what the compiler is told of addresses, limits of launches, what is refused at the
ends of the ranges."""
import os
import re
import subprocess

from paper_2505_14741_amd import build


def test_group_norm_accesses_promise_no_alignment_beyond_an_element():
    """x, out, gamma and beta may lie at any element's address: wide loads and stores of them, kept in L2 or not, must say so to the compiler."""
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", "-emit-llvm", os.path.join(build.CSRC, "group_norm.hip"), "-o", "-"],
                       capture_output=True, text=True, check=True)
    size = {"bfloat": 2, "float": 4}
    seen = set()
    for line in r.stdout.splitlines():
        for kind, pattern in (("store", r"store <(\d+) x (\w+)> [^,]*, (?:ptr|ptr addrspace\(1\)) \S+, align (\d+)"),
                              ("load", r"load <(\d+) x (\w+)>, (?:ptr|ptr addrspace\(1\)) \S+, align (\d+)")):
            m = re.search(pattern, line)
            if m and m.group(2) in size:
                assert int(m.group(3)) == size[m.group(2)], line
                seen.add((kind, m.group(1), m.group(2), "nontemporal" in line))
    for kind, count, elem, streamed in [(k, n, e, s) for n, e in (("8", "bfloat"), ("4", "bfloat"), ("4", "float"))
                                        for k, s in (("load", False), ("store", False), ("store", True))]:
        assert (kind, count, elem, streamed) in seen
