"""Shared memory of another CTA of a cluster may be accessed only when that CTA
is known to have started: in each kernel that does so, a barrier of the whole
cluster stands before the first access.  Read from the source, as no run can show
it: the CTAs of a cluster mostly start together."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2608_06690_gb300" / "csrc"
# what reaches another CTA's shared memory, by itself or in a function of the same file, and what waits for all CTAs
REMOTE = r"map_shared_rank\(|dsmem_addr\(|mapa\."
BARRIER = r"\bcluster_sync_all\(\)|\bcluster\.sync\(\)|\bcluster_wait\(\)"


def stripped(path):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", path.read_text(), flags=re.S)


def body(text, at):
    """The block that opens behind `at`."""
    start = text.index("{", at)
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[start:i + 1]
    raise ValueError("unbalanced")


def functions(text):
    """Names and bodies of a file's device functions, kernels apart."""
    kernels, others = {}, {}
    for m in re.finditer(r"__(global|device)__[^;{}=]*?\b(\w+)\((?=[^;{]*\)[^;{]*\{)", text):
        name = m.group(2)
        if name == "__launch_bounds__":
            name = re.search(r"\b(\w+)\((?!\()", text[m.end():]).group(1)
        (kernels if m.group(1) == "global" else others).setdefault(name, body(text, m.end()))
    return kernels, others


def without_lambdas(text, calls):
    """A kernel's text without what its named lambdas hold, and `calls` with the names of those that match it."""
    while True:
        m = re.search(r"\bauto (\w+) = \[[^\]]*\](?:\([^{};]*\))?[^{};]*(?=\{)", text)
        if not m:
            return text, calls
        inner = body(text, m.start())
        if re.search(calls, inner):
            calls += r"|\b%s\(" % m.group(1)
        text = text[:m.start()] + text[m.end() + len(inner):]


def cluster_files():
    return [p for p in sorted(CSRC.glob("*.cu")) if re.search(REMOTE, stripped(p))]


def test_there_are_such_files():
    assert {"k_sample.cu", "k_route.cu"} <= {p.name for p in cluster_files()}


@pytest.mark.parametrize("path", cluster_files(), ids=lambda p: p.name)
def test_a_barrier_stands_before_the_first_access(path):
    kernels, others = functions(stripped(path))
    # functions that access another CTA's memory before they wait for all of them, and ones that call such
    remote = set()
    while True:
        calls = "|".join([REMOTE] + [r"\b%s(?:<[^<>]*>)?\(" % n for n in sorted(remote)])
        more = set()
        for name, text in others.items():
            access, barrier = re.search(calls, text), re.search(BARRIER, text)
            if access and not (barrier and barrier.start() < access.start()):
                more.add(name)
        if more <= remote:
            break
        remote |= more
    checked = 0
    for name, text in kernels.items():
        text, calls_here = without_lambdas(text, calls)
        access, barrier = re.search(calls_here, text), re.search(BARRIER, text)
        if access:
            checked += 1
            assert barrier and barrier.start() < access.start(), "%s: %s reaches another CTA's shared memory before a barrier: %s" % (path.name, name, access.group(0))
    assert checked
