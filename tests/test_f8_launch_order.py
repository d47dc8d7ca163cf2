"""The kernels of the 8-bit path are launched while the kernel before them in the stream may still run: what they do before
their wait for it (cudaGridDependencySynchronize) must not touch device memory.  Read from the sources, because a violation
is a race whose outcome a run cannot be relied on to show."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_14985_b200", "csrc")
FILES = ("quantize.cuh", "gemm_f8.cuh", "append.cuh", "paged_f8.cuh")
WAIT = re.compile(r"\bpdl_begin\(\)|\bcudaGridDependencySynchronize\(\)")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def block(text, at):
    """The text of the braces that open at or after `at`."""
    at = text.index("{", at)
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at + 1:i]
    raise AssertionError("unbalanced braces")


def kernels():
    for name in FILES:
        text = source(name)
        for m in re.finditer(r"__global__[^;{]*?(\w+_kernel)\s*\(", text):
            yield name, m.group(1), block(text, m.end())


KERNELS = list(kernels())


def pointer_fields(name):
    fields = set()
    for m in re.finditer(r"\bstruct \w+Params\b", source(name)):
        for decl in block(source(name), m.end()).split(";"):
            if "*" in decl:
                fields |= {w for w in re.findall(r"\w+", decl.split("*", 1)[1])}
    return fields


def test_every_kernel_is_seen():
    assert {k for _, k, _ in KERNELS} == {"quantize_rows_kernel", "quantize_blocks_kernel", "gemm_f8_split_kernel", "gemm_f8_big_kernel",
                                          "kv_append_kernel", "paged_f8_decode_kernel", "paged_f8_combine_kernel"}
    assert {"seq_lens", "block_table", "splits", "ks", "vs"} <= pointer_fields("paged_f8.cuh") and "sa" in pointer_fields("gemm_f8.cuh")


@pytest.mark.parametrize("name,kernel,body", KERNELS, ids=[k for _, k, _ in KERNELS])
def test_nothing_is_read_before_the_wait(name, kernel, body):
    wait = WAIT.search(body)
    assert wait, "the kernel does not wait"
    before = body[:wait.start()]
    assert not re.search(r"\bp\.(%s)\b" % "|".join(sorted(pointer_fields(name))), before), "a pointer of the parameters is used before the wait"
    assert not re.search(r"[(,]\s*p\s*[,)]", before), "the parameters go to a function before the wait"


@pytest.mark.parametrize("name", FILES + ("f8.cuh",))
def test_no_non_coherent_loads(name):
    # such a load may only meet memory that nothing writes while the kernel is there, and these kernels are there while the one before
    # them may still write their inputs (scales that the quantiser or the cache append has just made, say)
    assert not re.search(r"\b__ldg\b|\bld\.global\.nc\b|\b__restrict__\b", source(name))


@pytest.mark.parametrize("name,kernel,body", KERNELS, ids=[k for _, k, _ in KERNELS])
def test_nothing_is_written_before_the_wait(name, kernel, body):
    # the clock stamps in particular: taken before the wait they would count the predecessor's time as the kernel's
    before = body[:WAIT.search(body).start()]
    assert not re.search(r"\bclock_probe\b|\bg_status\b|\bappend_report\b|\bst\.global\b", before)
