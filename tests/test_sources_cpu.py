"""Rules that the library's sources keep and no result shows."""
import os
import re

import pytest

from paper_2410_18517_b200 import build as kbuild


def kernel(source, name):
    """The text of a kernel, up to the next one."""
    with open(os.path.join(kbuild.CSRC, source)) as f:
        parts = f.read().split("__global__")
    found = [p for p in parts[1:] if re.match(r"[^{;]*\b%s\(" % name, p)]
    assert len(found) == 1, (source, name)
    return found[0]


@pytest.mark.parametrize("source,name", [
    ("kvs_kernels.cu", "decode_splitk_scalar"), ("kvs_mma.cu", "decode_splitk_mma"), ("kvs_pack4_mma.cu", "decode_pack4_mma"),
    ("kvs_pack4.cu", "decode_pack4_f32"), ("kvs_tree.cu", "tree_attention_fma"), ("kvs_tree_tc.cu", "tree_attention_tc"),
])
def test_attention_kernels_wait_before_they_let_the_next_launch_start(source, name):
    """What a later launch may fetch early (safe_rows_of) rests on it: once such a kernel has let its successor start,
    everything before the kernel is complete."""
    text = kernel(source, name)
    releases = [m.start() for m in re.finditer(r"pdl_launch_dependents\(\);", text)]
    waits = [m.start() for m in re.finditer(r"pdl_wait\(\);", text)]
    assert releases and len(waits) >= len(releases)
    for n, at in enumerate(releases):        # every role of the kernel waits, then releases
        assert sum(w < at for w in waits) > n, (source, text[at - 200:at])


def header_before(declaration):
    """The comment in front of a declaration of the C interface, as one line of words."""
    with open(os.path.join(kbuild.CSRC, "..", "..", "include", "kvs.h")) as f:
        text = f.read()
    text = text[:text.index(declaration)]
    return " ".join(text[text.rindex("/*"):].replace("\n *", " ").split())


def test_static_attention_names_the_calls_that_must_wait_for_it():
    """Every call that may move rows (rows_moved in its body)."""
    with open(os.path.join(kbuild.CSRC, "kvs_api.cu")) as f:
        parts = re.split(r"\nkvs_status (kvs_\w+)\(", f.read())
    movers = {name for name, body in zip(parts[1::2], parts[2::2]) if "rows_moved(" in body}
    assert {"kvs_evict", "kvs_accept_draft", "kvs_reorder"} <= movers
    words = header_before("kvs_status kvs_decode_attention_static(")
    waits = words[words.index("move or overwrite rows it reads"):]
    assert all(name in waits for name in movers)


def test_header_states_the_rows_that_selection_takes():
    words = header_before("kvs_status kvs_beam_select(")
    with open(os.path.join(kbuild.CSRC, "kvs_api.cu")) as f:
        body = re.split(r"\nkvs_status (?=kvs_\w+\()", f.read())
    limit = re.search(r"n_requests \* n_beams > (\d+)\)", next(b for b in body if b.startswith("kvs_beam_select("))).group(1)
    assert f"n_requests * n_beams at most max_batch and {limit}" in words


def test_no_function_that_nothing_calls():
    text = ""
    for source in kbuild.SOURCES + kbuild.HEADERS:
        with open(os.path.join(kbuild.CSRC, source)) as f:
            text += re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"__(?:device|host)__ (?:__forceinline__|__noinline__|constexpr|__host__|__device__| )*[\w:&* ]*?\b(\w+)\(", text))
    assert len(names) > 40
    assert not [n for n in sorted(names) if len(re.findall(r"\b%s\b" % n, text)) < 2]


def test_trace_and_kernel_choice_of_4bit_caches_are_as_the_header_says():
    assert "Over a 4-bit cache of fp32 storage only rows 150 and 151" in header_before("kvs_status kvs_trace_begin(")
    assert "KVS_TRACE_STAMP" not in kernel("kvs_pack4.cu", "decode_pack4_f32") and "KVS_TRACE_STAMP" in kernel("kvs_pack4_mma.cu", "decode_pack4_mma")
    with open(os.path.join(kbuild.CSRC, "kvs_api.cu")) as f:
        text = f.read()
    plan = text[text.index("bool choose_plan("):]
    assert plan.index("KVS_CACHE_4BIT") < plan.index("return false;") < plan.index("opt_kernel")
