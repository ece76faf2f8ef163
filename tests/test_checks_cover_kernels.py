"""Every kernel of the KV cache checks its global accesses in the -DESTP_CHECKS build (CPU, by the sources):
its body calls in_bounds, or a helper of the shared headers that does."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_15592_gb300", "csrc")


def _body(text, at):
    """The braces that follow position `at`, outside of parentheses."""
    depth = 0
    while text[at] != "{" or depth:
        depth += {"(": 1, ")": -1}.get(text[at], 0)
        at += 1
    end, open_ = at, 0
    while True:
        open_ += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
        if open_ == 0:
            return text[at:end]


def _read(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def _helpers():
    """in_bounds and the functions of cache.cuh that return what it says."""
    text, found = _read("cache.cuh"), {"in_bounds"}
    for m in re.finditer(r"__device__ __forceinline__ bool (\w+)\(", text):
        if re.search(r"return in_bounds\(", _body(text, m.start())):
            found.add(m.group(1))
    return found


KERNELS = [(os.path.basename(p), m.group(1)) for p in sorted(glob.glob(os.path.join(CSRC, "cache_*.cu")))
           for m in re.finditer(r"__global__ void __launch_bounds__\((?:[^()]|\([^()]*\))*\)\s+(\w+)\(", _read(os.path.basename(p)))]


def test_all_kernels_are_found():
    assert len(KERNELS) == sum(_read(os.path.basename(p)).count("__global__") for p in glob.glob(os.path.join(CSRC, "cache_*.cu"))) == 8


@pytest.mark.parametrize("name,kernel", KERNELS, ids=[k for _, k in KERNELS])
def test_kernel_checks_its_accesses(name, kernel):
    text = _read(name)
    body = _body(text, re.search(r"\b%s\(const|\b%s\(\s*const" % (kernel, kernel), text).start())
    assert re.search(r"\b(?:%s)\(" % "|".join(sorted(_helpers())), body), f"{kernel} makes no bounds check"
