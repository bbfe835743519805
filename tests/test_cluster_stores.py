"""Stores into another CTA's shared memory, read in the sources: a kernel makes the first one behind a wait for the whole cluster, on
every way there, since a CTA that has not begun has no shared memory to be written to.  (How the CTAs of a cluster begin cannot be
set from a test, so the order itself is looked at.)"""
import os
import re

import pytest

from paper_2505_02351_b200 import build

# what stores into other CTAs, and what waits until all have begun; none of either is conditional but on the kernel's own form
STORES = re.compile(r"\b(tell_all<|send_columns<|st_cluster_float2\()")
WAITS = re.compile(r"\b(wait_begun<kCtas>\(\)|cluster_wait\(\))")
ARRIVES = re.compile(r"\b(arrive_begun<kCtas>\(\)|cluster_arrive(_relaxed)?\(\))")


def kernels(source):
    """(name, body) of every kernel of a source file."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, source)).read())
    for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\([^)]*\)\s*)?(\w+)\s*\([^{;]*?\)\s*\{", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield m.group(1), text[m.end():at - 1]


@pytest.mark.parametrize("source,name", [("pages.cu", "give_pages_kernel"), ("pages.cu", "compact_plan_kernel"), ("chunk.cu", "chunk_kernel"),
                                         ("qkv_int4.cu", "qkv_int4_kernel")])
def test_the_first_store_waits_until_the_cluster_has_begun(source, name):
    body = dict(kernels(source))[name]
    store, wait, arrive = (r.search(body) for r in (STORES, WAITS, ARRIVES))
    assert store and wait and arrive and arrive.start() < wait.start() < store.start()


def test_no_other_kernel_stores_into_other_ctas():
    known = {"give_pages_kernel", "compact_plan_kernel", "chunk_kernel", "qkv_int4_kernel"}
    assert {n for s in build.SOURCES for n, body in kernels(s) if STORES.search(body)} == known
