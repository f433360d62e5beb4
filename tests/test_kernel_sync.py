"""Synchronisation that no run shows reliably when it is missing, read from the kernels' sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_13804_gb300", "csrc")


def _source(name):
    """A source file without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _top_level(text, kernel, until):
    """The kernel's statements outside any inner braces, up to `until`."""
    text = text[re.search(r"\b%s\(const BatchDesc" % kernel, text).start():]
    text = text[text.index("{") + 1:]
    depth, out = 0, []
    for i, ch in enumerate(text):
        if depth == 0 and text.startswith(until, i):
            return "".join(out)
        if ch == "}":
            depth -= 1
        if depth == 0:
            out.append(ch)
        if ch == "{":
            depth += 1
    raise AssertionError("no round loop in " + kernel)


@pytest.mark.parametrize("name,kernel", [("select.cu", "select_kernel"), ("select_gram.cu", "select_gram_kernel")])
def test_cluster_barrier_before_the_first_round(name, kernel):
    """Kernels that write into other CTAs' shared memory wait for the whole cluster to have started first: a
    cluster barrier on every path before the first round."""
    statements = _top_level(_source(name), kernel, "while (nsel < k_max)")
    assert re.search(r"(^|;|\})\s*(cluster\.sync|cluster_sync_all)\(\);", statements), "a CTA may write to a peer that has not started"


def test_warp_waits_order_the_other_lanes():
    """A wait that lane 0 makes for its warp: a shuffle hands its outcome to the other lanes, but orders no memory;
    what they read afterwards is ordered by a __syncwarp()."""
    found = []
    for name in sorted(os.listdir(CSRC)):
        for m in re.finditer(r"SP_DEVINL bool (mbar_\w*_warp)\(.*?\n\}", _source(name), re.S):
            found.append(m.group(1))
            assert re.search(r"__syncwarp\(\);\s*return __shfl_sync\([^;]*;\s*\}$", m.group(0)), m.group(1)
    assert "mbar_wait_warp" in found and "mbar_poll_cluster_warp" in found


def _kernel(text, kernel):
    """The text of a kernel's body."""
    text = text[re.search(r"\b%s\([^;]*?\)\s*\{" % kernel, text).end():]
    depth = 1
    for i, ch in enumerate(text):
        depth += (ch == "{") - (ch == "}")
        if depth == 0:
            return text[:i]
    raise AssertionError("no end of " + kernel)


def _waits_first(body):
    """Whether every thread waits for the kernel before this one, outside any condition, before the first trigger."""
    wait = re.search(r"(?:^|[;{}])\s*pdl_wait\(\);", body)
    trigger = re.search(r"\bpdl_trigger\(\);", body)
    if wait is None or (trigger is not None and trigger.start() < wait.end() - 1):
        return False
    return body[:wait.end()].count("{") == body[:wait.end()].count("}")


def test_what_runs_beside_the_tensor_kernel_finds_its_inputs_complete():
    """prefix_warp_kernel behind prefix_tc_kernel (`late`) reads queries, lengths, tables and pages before any wait of its
    own.  What wrote them is complete because the tensor kernel waits before it lets the next kernel start; the warp
    kernel's own end waits for the tensor kernel, so that the merge finds both complete."""
    tc, warp = _kernel(_source("prefix_attn_tc.cu"), "prefix_tc_kernel"), _kernel(_source("prefix_attn.cu"), "prefix_warp_kernel")
    assert _waits_first(tc), "the tensor kernel lets the warp kernel start before what came before is complete"
    assert not _waits_first(re.sub(r"pdl_wait\(\);\s*pdl_trigger\(\);", "pdl_trigger(); pdl_wait();", tc))
    assert not _waits_first(tc.replace("pdl_wait();", "if (warp == 0) pdl_wait();"))
    first = re.search(r"pdl_\w+\(\);", warp)
    assert warp[:first.end()].rstrip().endswith("if (!late) pdl_wait();")
    assert re.search(r"if \(late\) pdl_wait\(\);\s*$", warp), "the merge would not wait for the tensor kernel"
    calls = _source("prefix_attn.cu")
    calls = calls[calls.index("prefix_attention_launch("):]
    assert calls.index("prefix_tc_launch(") < calls.index("prefix_warp_kernel<128>") and "L.tc.workers ? 1 : 0)" in calls
    assert _waits_first(_kernel(_source("prefix_attn.cu"), "prefix_merge_kernel"))


@pytest.mark.parametrize("name,kernel", [("prefix_attn.cu", "prefix_row_kernel"), ("paged.cu", "paged_append_kernel"),
                                         ("beam.cu", "beam_scan_kernel"), ("beam.cu", "beam_join_kernel"),
                                         ("beam.cu", "beam_reorder_kernel")])
def test_paged_kernels_wait_before_they_let_the_next_start(name, kernel):
    assert _waits_first(_kernel(_source(name), kernel))
