"""Rules that the kernels' sources keep and that no run on one GPU can be relied on to show when they are broken."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34162_b200", "csrc")
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".cpp", ".h")))


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"/\*.*?\*/", " ", re.sub(r"//[^\n]*", "", text), flags=re.S)


def closing(text, at, brackets="{}"):
    """Behind the bracket that closes the one at `at`."""
    depth = 0
    while True:
        depth += (text[at] == brackets[0]) - (text[at] == brackets[1])
        at += 1
        if depth == 0:
            return at


def functions(text, kind):
    """Name and body of each function that is declared with `kind`."""
    for m in re.finditer(kind + r"\b", text):
        at = m.end()
        while True:
            name = re.compile(r"(\w+)\s*\(").search(text, at)
            if not name:
                return
            end = closing(text, name.end() - 1, "()")
            if name.group(1) not in ("__launch_bounds__", "alignas"):
                break
            at = end
        body = re.compile(r"[\s\w]*{").match(text, end)
        if body:                                       # else a declaration
            yield name.group(1), text[body.end() - 1:closing(text, body.end() - 1)]


def without_cluster_blocks(body):
    """Blocks of code for clusters are taken for code that every access, for clusters too, has behind it."""
    while m := re.search(r"if \(cluster > 1\) {", body):
        end = closing(body, m.end() - 1)
        body = body[:m.start()] + body[m.end():end - 1] + body[end:]
    return body


def comes_before(body, barrier, access):
    """Whether whoever comes to `access` has passed `barrier`: no block that holds it ends in between."""
    depth = 0
    for c in body[barrier:access]:
        depth += (c == "{") - (c == "}")
        if depth < 0:
            return False
    return True


def test_the_parser_sees_the_kernels():
    names = {n for f in SOURCES for n, _ in functions(source(f), "__global__")}
    assert {"policy_row_kernel", "policy_ring_kernel", "sort_tokens_kernel", "distill_row_kernel", "attention_dkv_mma_kernel"} <= names


@pytest.mark.parametrize("name", [f for f in SOURCES if f.endswith(".cu")])
def test_no_block_is_written_to_before_its_cluster_has_met(name):
    """Shared memory of another block may be accessed once that block is known to have started: a barrier of the cluster stands before
    every such access of every kernel."""
    text = source(name)
    remote = {"peer_addr"} | {n for n, body in functions(text, "__device__") if "peer_addr(" in body}
    access = re.compile(r"\b(?:" + "|".join(remote) + r")\s*(?:<[^;()]*>)?\(")
    for kernel, body in functions(text, "__global__"):
        body = without_cluster_blocks(body)
        barriers = [m.start() for m in re.finditer(r"\bcluster_(?:sync|wait)\(\)", body)]
        for m in access.finditer(body):
            assert any(b < m.start() and comes_before(body, b, m.start()) for b in barriers), (kernel, body[m.start() - 60:m.end() + 60])


@pytest.mark.parametrize("name", [f for f in SOURCES if f.endswith(".cu")])
def test_what_a_device_answers_is_not_kept_for_another(name):
    """A function that asks the device how much of something fits keeps the answer with its context, not in a static of its own."""
    for kind in ("cudaError_t", "int", "void", "bool"):
        for function, body in functions(source(name), r"\b" + kind):
            if re.search(r"\bcuda(Occupancy|DeviceGetAttribute|GetDeviceProperties)", body):
                assert not re.search(r"\bstatic\b(?!\s+(?:constexpr|_assert))(?!_assert)", body), function
