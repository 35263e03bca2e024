"""Rules that the kernels' sources have to keep and that no run can show, checked on the text."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2006_02924_b200", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")))


def _code(path):
    with open(path) as f:
        text = f.read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _body(text, at):
    """The braces that open behind `at`, with what is in them."""
    begin = text.index("{", at)
    depth = 0
    for i in range(begin, len(text)):
        depth += (text[i] == "{") - (text[i] == "}")
        if depth == 0:
            return text[begin:i + 1]
    raise AssertionError("unbalanced braces")


def _kernels():
    for path in SOURCES:
        text = _code(path)
        for m in re.finditer(r"__global__\b", text):
            body = _body(text, m.end())
            name = re.findall(r"(\w+)\s*\(", text[m.end():text.index("{", m.end())])
            yield os.path.basename(path), next(n for n in name if n.endswith("_kernel")), body


EARLY = [k for k in _kernels() if "wait_for_previous_kernel" in k[2]]


def test_the_kernels_that_start_early_are_found():
    names = {name for _, name, _ in EARLY}
    assert {"dropout_kernel", "residual_norm_kernel", "residual_norm_grad_kernel", "residual_norm_join_kernel", "fp8_pack_kernel",
            "fp8_pack_weight_kernel", "fp8_linear_kernel", "fp8_join_kernel", "embedding_sum_kernel"} <= names


@pytest.mark.parametrize("name", [k[1] for k in EARLY])
def test_kernels_that_start_early_read_what_is_written_meanwhile_coherently(name):
    """A kernel that may be resident while its predecessor still writes must not read through the non-coherent path:
    that is defined for memory which nobody writes in the kernel's whole life, the time before its wait included."""
    file, body = next((file, body) for file, n, body in EARLY if n == name)
    found = re.findall(r"__ldg\b|ld\.global\.nc", body)
    assert not found, f"{name} in {file}"


@pytest.mark.parametrize("file", ["adasum_random.cuh", "adasum_vectors.cuh", "adasum_operators.cuh", "adasum_residual_norm.cuh",
                                  "adasum_fp8.cuh", "adasum_tensor.cuh"])
def test_what_those_kernels_share_reads_coherently(file):
    assert not re.findall(r"__ldg\b|ld\.global\.nc", _code(os.path.join(CSRC, file)))


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_what_calls_keep_for_one_another_is_atomic(path):
    """Threads may make their first calls at once: a function's static that is written is an atomic.  (Namespaces hold
    mutable objects behind a mutex.)"""
    statics = re.findall(r"^[ \t]+static\s+(?!constexpr\b|const\b|inline\b|__)([^;={(]*[\w\]])\s*[;={]", _code(path), flags=re.M)
    assert not [s for s in statics if not s.startswith("std::atomic<")]
