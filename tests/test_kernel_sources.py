"""Rules of the kernels launched as programmatic dependents that no run can be
trusted to show (a breach would hang now and then, or read stale memory), held
to the sources themselves."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2408_00539_gb300", "csrc")


def _body(text, at):
    """The block that opens at or after `at`."""
    start = text.index("{", at)
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[start:i]
    raise ValueError("unbalanced braces")


def _kernels():
    """(name, parameters, body) of every kernel, comments taken out."""
    out = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s+)?(\w+)\s*\(", text):
            depth, end = 1, m.end()
            while depth:
                depth += {"(": 1, ")": -1}.get(text[end], 0)
                end += 1
            out.append((m.group(1), text[m.end():end], _body(text, end)))
    return out


KERNELS = _kernels()
TRIGGER = re.compile(r"pdl_wait\(\)|pdl_trigger\(\)|griddepcontrol\.launch_dependents")


def test_kernels_found():
    names = {n for n, _, _ in KERNELS}
    assert {"fwd_pair_kernel", "fwd_kernel", "dq_kernel", "dkdv_kernel", "dq_gemm_kernel", "decode_tc_kernel"} <= names


@pytest.mark.parametrize("name", [n for n, _, b in KERNELS if "tmem_alloc" in b])
def test_trigger_follows_the_allocation(name):
    """A kernel that holds tensor memory lets its successor start only after
    the block-wide barrier behind its own allocation: the successor may allocate
    before it waits, and each would wait for the other."""
    body = next(b for n, _, b in KERNELS if n == name)
    allocated = body.index("__syncthreads()", body.index("tmem_alloc"))
    for m in TRIGGER.finditer(body):
        # a block that leaves before the allocation needs none
        leaves = re.match(r"[^{}]*\breturn;", body[m.end():])
        assert m.start() > allocated or leaves, name


@pytest.mark.parametrize("name", [n for n, _, b in KERNELS if "pdl_" in b])
def test_nothing_counts_as_constant(name):
    """Loads of a dependent kernel that the compiler may take for constant may
    be moved before its wait: no __restrict__ parameters, no __ldg."""
    params, body = next((p, b) for n, p, b in KERNELS if n == name)
    assert "__restrict__" not in params and "__ldg" not in body


def test_page_table_and_offsets_are_plain_loads():
    for name, function in (("ism_internal.cuh", "paged_row"), ("ism_rope.cu", "seq_of")):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        at = text.index(function + "(")
        assert "__restrict__" not in text[at:text.index(")", at)] and "__ldg" not in _body(text, at)


def test_early_reads_go_to_l2():
    """What is read before the kernel's own wait comes from L2: the lengths and
    the page table of the decode, O and dO of the dependent Delta."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "ism_decode_tc.cu")).read())
    assert re.findall(r"[^\n]*\bcache_len\b[^\n]*", text) == [
        "__device__ __forceinline__ int32_t cached(const DecodeArgs& a, int b) { return ld_gpu(a.cache_len + b); }"]
    assert "ld_gpu(page_entry(" in text and "paged_row(" not in text
    body = next(b for n, _, b in KERNELS if n == "delta_kernel")
    loads = re.findall(r"=([^;]*(?:\bO\b|\bdO\b)[^;]*);", body)
    assert len(loads) == 2 and all("__ldcg" in x for x in loads)


def test_split_forward_triggers_behind_its_last_barrier():
    """The merge behind a split forward starts when every warp is done: the
    first thread of a block to trigger does so for the block."""
    body = next(b for n, _, b in KERNELS if n == "fwd_pair_kernel")
    assert body.rindex("pdl_trigger()") > body.rindex("__syncthreads()")


def test_metadata_is_read_as_it_was_written():
    """The metadata kernels read tiles and bounds that they wrote themselves:
    nothing of theirs counts as constant."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "ism_meta.cu")).read())
    assert "__restrict__" not in text and "__ldg" not in text


def _source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_lengths_and_pages_on_the_device_are_bounded():
    """What an append reads on the device (cache lengths, page entries) is not what
    the host has checked: every use of it goes through a bound, and rows that do
    not fit are not written."""
    meta, tc, common = _source("ism_meta.cu"), _source("ism_decode_tc.cu"), _source("ism_internal.cuh")
    assert not re.search(r"c_snap\s*\[|cache_len\s*\[", meta)
    assert sorted(re.findall(r"[^\n]*lens\.len\[[^\n]*", meta)) == [
        "    const int32_t len = lens.len[b];"] * 3 + [
        "__device__ __forceinline__ int32_t cached_len(const CacheLens& lens, int b) "
        "{ return bounded_len(lens.len[b], lens.most); }"]
    row = _body(meta, meta.index("write_row("))
    assert "lens.most) return -1" in row and "page_held(pages, entry) ? row : -1" in row
    for name in ("cache_write_kernel", "rope_cache_write_kernel"):
        body = next(b for n, _, b in KERNELS if n == name)
        assert "write_row(lens" in body and "bounded_len(len, lens.most)" in body and "paged_row(" not in body
    assert "bounded_len(len, lens.most)" in _body(meta, meta.index("void zero_value_tail("))
    assert "write_row(lens" in _body(meta, meta.index("void zero_value_tail("))
    assert len(re.findall(r"\bcached\(", tc)) == 2 and "bounded_len(cached(a, b), a.len_most)" in tc
    assert "bounded_len(" in _body(common, common.index("advance_cache_len("))
    assert "num_pages" in _body(common, common.index("page_row("))
    assert "num_pages" in _body(_source("ism_decode_win.cu"), _source("ism_decode_win.cu").index("auto row_of"))


def test_what_is_asked_of_a_device_is_kept_a_device():
    """The number of resident clusters sets the one-launch step's shape; it is the current device's."""
    text = _source("ism_decode_win.cu")
    body = _body(text, text.index("int active_clusters("))
    assert "cudaGetDevice(&dev)" in body and re.findall(r"\bknown\[[^;]*\]\.(?:load|store)", body)
    assert all(x.startswith("dev") for x in re.findall(r"\bknown\[(\w+)", body[body.index("cudaGetDevice"):]))


def test_timers_cover_every_launch_of_their_kind():
    """The sums of the sinks' parts are part of dK/dV: no launch of the backward lies outside a timer."""
    text = _source("ism_bwd_tc.cu")
    body = _body(text, text.index("cudaError_t launch_bwd_t("))
    within, launches = 0, 0
    for m in re.finditer(r"timer_(begin|end)\(|\b(?:launch|launch_dkdv_pair|launch_dq_gemm)\(", body):
        if m.group(1):
            within += 1 if m.group(1) == "begin" else -1
            assert within in (0, 1)
        else:
            launches += 1
            assert within == 1, body[m.start():m.start() + 80]
    assert launches == 6 and within == 0


def test_plain_metadata_knows_no_window():
    """The metadata kernels of plain calls are instantiations without the window's arithmetic (0.7 us a pass)."""
    text = _source("ism_meta.cu")
    for name in ("pass_meta_kernel", "pass_meta_small_kernel"):
        at = text.index(name + "(")
        assert re.search(r"template <bool kWin>\s+__global__[^;{]*$", text[:at]), name
        body = next(b for n, _, b in KERNELS if n == name)
        assert "kWin ? window : Window{0, 0}" in body and "if (kWin && parts.n > 0)" in body
        assert re.search(name + r"<true>\s*:\s*" + name + "<false>", text)
