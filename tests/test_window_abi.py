"""Host-side checks of the windowed calls and the page operations (no GPU):
layouts of the packed structs, sizes, and refusals before anything is launched."""
import ctypes as C
import os
import re
import subprocess
import sysconfig

import numpy as np
import pytest
import torch

from paper_2408_00539_gb300 import ism

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where no GPU is visible")
FAKE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return ism.load(build_if_missing=True)


def _segs():
    return ism.Segments.from_numpy([0, 300, 430], [0, 2, 3], [100, 300, 130], [0, 1, 0], device="cpu")


def _head(form=0, hq=4, hkv=2, d=128, dtype=0, scale=0.1):
    return (*_segs().fields(), hq, hkv, d, dtype, form, scale, 1.0, 1.0, 1.0)


def test_struct_sizes(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include "ism.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) { printf("%zu %zu %zu %zu", '
                   'sizeof(ism_window_t), sizeof(ism_pages_t), offsetof(ism_pages_t, num_pages), '
                   'offsetof(ism_pages_t, block_table)); return 0; }\n')
    exe = str(tmp_path / "s")
    cc = (sysconfig.get_config_var("CC") or "gcc").split()[0]
    try:
        subprocess.run([cc, "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    except FileNotFoundError:
        pytest.skip("no C compiler")
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in re.findall(r"\d+", out)] == [ism._WINDOW.size, ism._PAGES.size, 24, 40]


def test_backward_sizes(lib):
    full, low = ism._pass_sizes(_head(), True, ism._window(50, 4))
    plain_full, plain_low = ism._pass_sizes(_head(), True)
    assert low == plain_low <= full <= plain_full
    assert ism._pass_sizes(_head(), True, ism._window(300, 0)) == (plain_full, plain_low)


@host_only
def test_windows_are_refused(lib):
    def fwd(window=(50, 4), plan=(0, 0, 0), **head):
        code = lib.ism_call_fwd_window(ism._PASS.pack(*_head(**head), 0, 0, 0, *plan, *(0,) * 14),
                                       None if window is None else ism._WINDOW.pack(*window))
        return code, lib.ism_last_error().decode()

    assert fwd(None) == (1, "window is NULL")
    assert fwd((0, 0)) == (1, "window 0 must be at least 1")
    assert fwd((5, -2)) == (1, "sinks -2 must be at least 0")
    assert fwd(dtype=2) == (2, "windowed attention needs bf16 or fp32 inputs")
    assert fwd(form=1) == (2, "windowed attention needs bf16 or fp32 inputs")
    assert fwd(plan=(256, 0, 0)) == (2, "the windowed calls take no plan")
    assert "rope tables" in fwd(form=2)[1]
    assert fwd(d=96)[0] == 2 and fwd(hq=3)[0] == 1
    assert "must be non-NULL" in fwd()[1]
    call = ism._PASS.pack(*_head(), *(0,) * 20)
    assert lib.ism_call_bwd_window(call, ism._WINDOW.pack(0, 0)) == 1
    assert lib.ism_call_bwd_window(call, ism._WINDOW.pack(4, 0)) == 1 and "non-NULL" in lib.ism_last_error().decode()
    assert lib.ism_call_fwd_window(None, None) == lib.ism_call_append_window(None, None) == 1
    n = C.c_size_t()
    assert lib.ism_attn_bwd_window_workspace_size(None, None, ism._WINDOW.pack(4, 0), C.byref(n)) == 1


@host_only
def test_appends_are_refused(lib):
    lens, table = np.array([500], np.int32), np.array([[-1, 1, 2, 3, 4]], np.int32)
    end, typ = np.array([1], np.int32), np.array([1], np.uint8)

    def append(window, form=4, dtype=0, scale=0.1, d=128):
        call = ism._APPEND.pack(4, 2, d, dtype, form, scale, 1.0, 1.0, 1.0, 0, 0, 0, 1, 1, 1, 5, 128, 5,
                                ism._addr(end), ism._addr(typ), FAKE, FAKE, FAKE, FAKE, FAKE, 640, FAKE,
                                ism._addr(table), FAKE, ism._addr(lens), FAKE, 0, 0, 0, 0)
        return lib.ism_call_append_window(call, ism._WINDOW.pack(*window)), lib.ism_last_error().decode()

    # the first page may be missing only where no row and no sink needs it: then the workspace is what is wrong
    for window, needed in (((373, 0), False), ((374, 0), True), ((200, 1), True), ((1, 0), False), ((1000, 0), True)):
        code, text = append(window)
        assert code == (1 if needed else 5), (window, text)
        assert ("page 0 of the block table is -1" in text) == needed
    assert append((0, 0))[0] == 1 and append((4, 0), dtype=2)[0] == 2 and append((4, 0), d=80)[0] == 2
    assert "needs ISM_BF16" in append((4, 0), form=6, dtype=1)[1]
    assert "rope tables" in append((4, 0), form=2)[1]


@host_only
def test_pools_are_refused(lib):
    table, lens, refs = np.full((2, 3), -1, np.int32), np.zeros(2, np.int32), np.zeros(4, np.int32)

    def free(row_bytes=64, pages=4, page=128, slots=2, most=3, pool=FAKE, seqs=(0,)):
        s = ism._PAGES.pack(pool, pool, row_bytes, pages, page, slots, most, FAKE, ism._addr(table), FAKE,
                            ism._addr(lens), ism._addr(refs))
        at = np.array(seqs, np.int32)
        return lib.ism_pages_free(s, ism._addr(at), len(seqs), None), lib.ism_last_error().decode()

    assert free()[0] == 0  # nothing is held: nothing is launched
    assert "row_bytes 40" in free(row_bytes=40)[1] and "page_size 100" in free(page=100)[1]
    assert "num_pages" in free(pages=0)[1] and "num_seqs" in free(slots=0)[1] and "num_seqs" in free(most=0)[1]
    assert "num_pages" in free(pages=1 << 24)[1] and "16-byte aligned" in free(pool=FAKE + 8)[1]
    assert "non-NULL" in free(pool=0)[1]
    assert free(seqs=(0, 0))[0] == 1 and free(seqs=(2,))[0] == 1
    assert lib.ism_pages_compact(None, None, None) == 1 and lib.ism_last_error() == b"pages is NULL"
    lens[1] = 500
    assert "does not fit" in free(seqs=(1,))[1]


def test_python_arguments():
    pool, i32 = torch.zeros((256, 2, 8), dtype=torch.bfloat16), torch.int32
    table, lens = torch.full((2, 3), -1, dtype=i32), torch.zeros(2, dtype=i32)
    host = (np.full((2, 3), -1, np.int32), np.zeros(2, np.int32), np.zeros(2, np.int32))

    def make(pool2=pool, page=128, t=table, n=lens, h=host):
        return ism.PagedCache(pool, pool2, page, t, h[0], n, h[1], h[2])

    assert make().free_pages == 2
    with pytest.raises(ValueError):
        make(page=100)
    with pytest.raises(ValueError):
        make(pool2=pool[:128])
    with pytest.raises(ValueError):
        make(t=torch.full((3, 2), -1, dtype=i32).T)
    for i in range(3):
        for bad in (host[i].astype(np.int64), host[i].tolist(), host[i][:1]):
            with pytest.raises(TypeError):
                make(h=host[:i] + (bad,) + host[i + 1:])
    with pytest.raises(TypeError):
        make(n=lens.long())
    with pytest.raises(ValueError, match="32-bit"):
        ism._window(2 ** 31, 0)


@host_only
def test_forks_from_pages_given_up_are_refused(lib):
    """At fewer keys than the source holds, also where they end with a page: what the
    window ending there needs has been given up.  At all of its keys a fork is as
    good as the source."""
    def fork(length, table, keys, page=128):
        held = sorted(p for p in table if p >= 0)
        table = np.array([table, [-1] * len(table)], np.int32)
        lens, refs = np.array([length, 0], np.int32), np.zeros(8, np.int32)
        refs[held] = 1
        s = ism._PAGES.pack(FAKE, FAKE, 64, 8, page, 2, table.shape[1], FAKE, ism._addr(table), FAKE, ism._addr(lens),
                            ism._addr(refs))
        src, dst, n = np.array([0], np.int32), np.array([1], np.int32), np.array([keys], np.int32)
        before = table.copy(), lens.copy(), refs.copy()
        code = lib.ism_pages_fork(s, ism._addr(src), ism._addr(dst), ism._addr(n), 1, None)
        if code == 1:
            assert all((a == b).all() for a, b in zip(before, (table, lens, refs)))
        return code, lib.ism_last_error().decode()

    passed = 3  # past the checks, at the launch: there is no device
    for keys in (1, 127, 128, 129, 255, 256):
        assert fork(500, [-1, -1, 4, 5], keys) == (1, f"sequence 0: the page of key {keys - 1} has been freed")
    for keys in (257, 384, 385, 500):
        assert fork(500, [-1, -1, 4, 5], keys)[0] == passed
    for keys in (128, 100, 385, 512):  # with a page of sinks
        assert fork(512, [0, -1, -1, 5], keys)[0] == passed
    for keys in (129, 256, 384):
        assert fork(512, [0, -1, -1, 5], keys)[0] == 1
    assert fork(512, [-1, -1, -1, -1], 512)[0] == passed  # (a window of one key)
    assert fork(512, [-1, -1, -1, -1], 511)[0] == fork(512, [-1, -1, -1, -1], 384)[0] == 1


@host_only
def test_appends_that_do_not_fit_the_pools_are_refused():
    """Types and heads of the new rows against the pools', before a page is taken."""
    pool = torch.zeros((256, 2, 64), dtype=torch.bfloat16)
    refs = np.zeros(2, np.int32)
    cache = ism.PagedCache(pool, pool.clone(), 128, torch.full((2, 3), -1, dtype=torch.int32),
                           np.full((2, 3), -1, np.int32), torch.zeros(2, dtype=torch.int32), np.zeros(2, np.int32), refs)

    def rows(hq=4, hk=2, hv=2, d=64, n=1, nk=None, b=1, dtype=torch.bfloat16, kd=None, vd=None):
        return (torch.zeros((b, n, hq, d), dtype=dtype), torch.zeros((b, nk or n, hk, d), dtype=kd or dtype),
                torch.zeros((b, nk or n, hv, d), dtype=vd or dtype))

    f32, f8 = torch.float32, torch.float8_e4m3fn
    for bad in (rows(dtype=f32), rows(dtype=f8), rows(kd=f32), rows(vd=f32)):
        with pytest.raises(TypeError, match="pools"):
            cache.append(*bad, [1], [1], 0.1)
    for bad in (rows(hk=4, hv=4), rows(hk=1, hv=1), rows(hv=4), rows(d=128), rows(nk=2)):
        with pytest.raises(ValueError, match="pools"):
            cache.append(*bad, [1], [1], 0.1, window=20)
    with pytest.raises(ValueError):
        cache.append(*(x[0] for x in rows()), [1], [1], 0.1)
    assert not refs.any() and (cache.block_table_host == -1).all() and not cache.cache_len_host.any()


def test_the_header_names_what_differs_from_the_plain_calls():
    """A window that hides nothing runs the plain calls' kernels but in two forms; both stand there."""
    text = open(os.path.join(ROOT, "include", "ism.h")).read()
    said = re.search(r"it is the plain operation(.*?)\n \*   window >= 1", text, re.S).group(1)
    said = re.sub(r"\s*\n \*\s*", " ", said)
    assert "bf16 backward at head_dim 128" in said and "single tokens" in said
