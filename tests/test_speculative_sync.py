"""Synchronisation of the kernels for drafted tokens that no run shows reliably when it is missing, read from their sources."""
import re

from test_kernel_sync import _kernel, _source


def _ends_uniformly(body):
    """Whether what other CTAs change while the kernel runs ends a CTA only as a whole: what a thread has read of work.end is
    used in a vote of the CTA and nowhere else."""
    head = body[:body.index("sum_slice")]
    if len(re.findall(r"\bwork\.end\b", head)) != 1:
        return False
    name = re.search(r"\bint (\w+) = [^;]*\bwork\.end\b[^;]*;", head)
    uses = [m.start() for m in re.finditer(r"\b%s\b" % name.group(1), body) if m.start() > name.end()]
    return bool(uses) and all(re.search(r"__syncthreads_or\([^()]*$", body[:at]) for at in uses)


def test_rows_that_are_passed_over_end_whole_ctas():
    """Rows in order: the sequence's end moves while a CTA looks at it.  Warps that saw different ends would part before the
    barriers of the sums."""
    body = _kernel(_source("verify.cu"), "verify_sums_kernel")
    assert _ends_uniformly(body)
    assert not _ends_uniformly(re.sub(r"__syncthreads_or", "", body))


def _count_is_acquired(body):
    """Whether the thread that counts a slice puts a fence on both sides of the count, ahead of the barrier that hands what
    other CTAs wrote on to its warp."""
    return re.search(r"__threadfence\(\);[^}]*\bconst bool (\w+) = atomicAdd\(work\.count\b[^;]*;\s*if \(\1\) __threadfence\(\);[^}]*\}"
                     r"\s*__syncthreads\(\);", body) is not None


def test_the_last_slice_of_a_row_sees_the_others():
    body = _kernel(_source("verify.cu"), "verify_sums_kernel")
    assert _count_is_acquired(body)
    assert not _count_is_acquired(re.sub(r"if \(\w+\) __threadfence\(\);", "", body))


def _lengths_are_read_before_they_change(body):
    """Whether every CTA's reads of the lengths are released by its arrival at the cluster's barrier and the writes lie behind
    a wait that acquires them."""
    arrive, wait = body.find("barrier.cluster.arrive.release"), body.find("barrier.cluster.wait.acquire")
    reads = [m.start() for m in re.finditer(r"= a\.lens\[", body)]
    writes = [m.start() for m in re.finditer(r"\ba\.lens\[[^;]*\]\s*= ", body)]
    return bool(reads and writes) and max(reads) < arrive < wait < min(writes) and "arrive.relaxed" not in body


def test_forks_read_all_lengths_before_one_changes():
    body = _kernel(_source("pages.cu"), "pages_fork_kernel")
    assert _lengths_are_read_before_they_change(body)
    assert not _lengths_are_read_before_they_change(body.replace("arrive.release", "arrive.relaxed"))
    assert not _lengths_are_read_before_they_change(body.replace("wait.acquire", "wait"))
