"""Orders in the adapters', layer norm's and AdamW's kernels that no run can show
to be wrong, checked in their source.

Each is launched as a programmatic dependent of the kernel before it, so nothing
of that kernel may be read in front of griddepcontrol.wait, and dependents may
start behind it only: a dependent that started earlier could write over what the
kernel before still reads.  Kernels with tensor memory take it before the wait: a
dependent that took it first would wait for a kernel that waits for tensor memory."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_1701_00485_gb300", "csrc")
READS = re.compile(r"__ld\w*\(|bulk_load\w*\(|cp_async16\(|a\.route\.|perm\[|ids\[|\bload\w*\(|a\.ad\.|word_at\(")


def _kernels():
    for name in ("tbn_adapter.cu", "tbn_adapter_small.cu", "tbn_layernorm.cu", "tbn_adamw.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for m in re.finditer(r"__global__ void[^{;]*?(\w+_kernel)\(", text):
            begin = text.index("{", text.index(")", m.end()))
            yield name, m.group(1), text[begin:text.index("\n}\n", begin)]


KERNELS = list(_kernels())


def test_the_kernels_are_found():
    names = [k for _, k, _ in KERNELS]
    sources = "".join(open(os.path.join(CSRC, name)).read() for name in dict.fromkeys(n for n, _, _ in KERNELS))
    assert len(names) == len(set(names)) == sources.count("__global__ void") > 0
    assert len(set(n for n, _, _ in KERNELS)) == 4


@pytest.mark.parametrize("name,kernel,body", KERNELS, ids=[k for _, k, _ in KERNELS])
def test_wait_comes_before_reads_and_dependents(name, kernel, body):
    wait = body.find("grid_dependency_wait();")
    launch = body.find("grid_dependents_launch();")
    first = READS.search(body)
    assert 0 <= wait < launch, "%s: dependents start before the wait" % kernel
    assert body.count("grid_dependency_wait();") == body.count("grid_dependents_launch();") == 1
    if first is not None:
        assert wait < first.start(), "%s reads before its wait" % kernel
    else:   # plain reads: nothing but declarations of shared memory stands before the wait
        lines = [line.strip() for line in body[1:wait].splitlines()]
        assert all(line.startswith(("__shared__", "extern __shared__")) for line in lines if line), kernel


@pytest.mark.parametrize("kernel", ["shrink_tc_kernel", "expand_tc_kernel", "grad_tc_kernel"])
def test_tensor_memory_is_taken_before_the_wait(kernel):
    body = next(b for _, k, b in KERNELS if k == kernel)
    begin = body.find("tc_begin<")
    assert 0 <= begin < body.find("grid_dependency_wait();")
    # and given back on every way out
    after = body[begin:]
    assert not re.search(r"return;", after)
    assert "tc_end<" in after[-60:]
