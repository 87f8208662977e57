"""Appends whose device lengths or page table are not what the host's mirrors
hold (a broken contract): nothing outside the caches is touched, nothing is
written for the sequence concerned, the other one comes out as ever, and
ism_check_status says so."""
import numpy as np
import pytest
import torch

from paper_2408_00539_gb300 import ism
from paper_2408_00539_gb300 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GUARD, MARK = 1024, 7.0  # rows in front of and behind a cache, and what they hold


def _guarded(rows, hkv, D, dtype):
    """(whole, the rows in its middle)."""
    whole = torch.full((rows + 2 * GUARD, hkv, D), MARK, dtype=dtype, device=DEV)
    return whole, whole[GUARD:GUARD + rows]


def _touched(whole, rows):
    return bool((whole[:GUARD] != MARK).any() or (whole[GUARD + rows:] != MARK).any())


@pytest.fixture
def form(knobs):
    """Windowed single tokens in three launches: the form that goes by the device's lengths."""
    knobs("ISM_DECODE_WINDOW", 0)


FORMS = [(128, torch.bfloat16, 4, 2), (64, torch.bfloat16, 4, 2), (128, torch.bfloat16, 3, 3),
         (64, torch.float32, 2, 2)]


@pytest.mark.parametrize("window", [None, 60])
@pytest.mark.parametrize("n", [1, 5, 140])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("D,dtype,hq,hkv", FORMS)
@pytest.mark.parametrize("length", [300, 299, -5, 2 ** 31 - 1])
def test_lengths_past_the_cache(form, D, dtype, hq, hkv, length, rope, n, window):
    if rope and dtype != torch.bfloat16:
        pytest.skip("rotary appends take bf16")
    B, cap = 2, 300
    if length == 299 and n == 1:
        length = 300
    gen = torch.Generator(device=DEV).manual_seed(n)
    old = [torch.randn((B * cap, hkv, D), generator=gen, device=DEV).to(dtype) for _ in range(2)]
    x = [torch.randn((B, n, h, D), generator=gen, device=DEV).to(dtype) for h in (hq, hkv, hkv)]
    tables = tuple(torch.from_numpy(t).to(DEV) for t in wl.rope_tables(cap, D)) if rope else None

    def run(first):
        pairs = [_guarded(B * cap, hkv, D, dtype) for _ in range(2)]
        for (_, c), o in zip(pairs, old):
            c.copy_(o)
        k, v = (c.view(B, cap, hkv, D) for _, c in pairs)
        dev, host = torch.tensor([first, 40], dtype=torch.int32, device=DEV), np.array([100, 40], np.int32)
        args = (*x, k, v, dev, host, [n], [1])
        if window:
            o, lse = ism.prefill_append_window(*args, D ** -0.5, window, 3, rope=tables)
        elif rope:
            o, lse = ism.prefill_append_rope(*args, *tables, D ** -0.5)
        else:
            o, lse = ism.prefill_append(*args, D ** -0.5)
        return o, lse, k, v, dev, [w for w, _ in pairs]

    ism.check_status(DEV)
    want = run(100)
    ism.check_status(DEV)
    got = run(length)
    with pytest.raises(ism.IsmError, match="the host's mirrors do not have") as info:
        ism.check_status(DEV)
    assert info.value.code == 1
    ism.check_status(DEV)
    assert not any(_touched(w, B * cap) for w in got[5])
    for c, o in zip(got[2:4], old):
        assert torch.equal(c[0], o.view(B, cap, hkv, D)[0])
    assert got[4].tolist() == [min(max(length, 0), cap - n) + n, 40 + n]
    for a, b in zip(got[2:4], want[2:4]):
        assert torch.equal(a[1], b[1])
    # (the other sequence's keys may be shared out otherwise: two roundings of the output)
    far = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -18
    a, b = got[0][1].double(), want[0][1].double()
    assert torch.isfinite(a).all() and ((a - b).abs() <= far * (b.abs() + 1)).all()


@pytest.mark.parametrize("window", [None, 60])
@pytest.mark.parametrize("one_launch", [0, 1])
@pytest.mark.parametrize("n", [1, 5])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("D,dtype,hq,hkv", FORMS)
@pytest.mark.parametrize("entry", [-1, 5, 2 ** 31 - 1, -2 ** 31])
def test_pages_outside_the_pool(knobs, D, dtype, hq, hkv, entry, rope, n, one_launch, window):
    """The device's table names no page of the pool for the new rows."""
    if rope and dtype != torch.bfloat16:
        pytest.skip("rotary appends take bf16")
    knobs("ISM_DECODE_WINDOW", one_launch)
    page, pages = 128, 5
    gen = torch.Generator(device=DEV).manual_seed(n)
    pairs = [_guarded(pages * page, hkv, D, dtype) for _ in range(2)]
    for _, c in pairs:
        c.copy_(torch.randn(c.shape, generator=gen, device=DEV))
    old = [c.clone() for _, c in pairs]
    x = [torch.randn((2, n, h, D), generator=gen, device=DEV).to(dtype) for h in (hq, hkv, hkv)]
    host = np.array([[0, 1], [3, 2]], np.int32)
    table = torch.tensor([[0, entry], [3, 2]], dtype=torch.int32, device=DEV)
    lens = np.array([130, 140], np.int32)
    dev = torch.from_numpy(lens.copy()).to(DEV)
    tables = tuple(torch.from_numpy(t).to(DEV) for t in wl.rope_tables(2 * page, D)) if rope else None
    args = (*x, *(c for _, c in pairs), page, table, host, dev, lens, [n], [1])
    ism.check_status(DEV)
    if window:
        o, _ = ism.prefill_append_paged_window(*args, D ** -0.5, window, 3, rope=tables)
    elif rope:
        o, _ = ism.prefill_append_paged_rope(*args, *tables, D ** -0.5)
    else:
        o, _ = ism.prefill_append_paged(*args, D ** -0.5)
    with pytest.raises(ism.IsmError, match="the host's mirrors do not have"):
        ism.check_status(DEV)
    assert not any(_touched(w, pages * page) for w, _ in pairs)
    for (_, c), before, new in zip(pairs, old, x[1:]):
        kept = torch.ones(pages * page, dtype=torch.bool, device=DEV)
        kept[2 * page + 12:3 * page] = False  # the second sequence's new rows, and zeros behind its values
        assert torch.equal(c[kept], before[kept])
    assert torch.equal(pairs[1][1][2 * page + 12:2 * page + 12 + n], x[2][1])
    assert torch.isfinite(o[1].float()).all()


@pytest.mark.parametrize("one_launch", [0, 1])
@pytest.mark.parametrize("n", [1, 5])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("page", [0, 128])
@pytest.mark.parametrize("D,dtype,hq,hkv", FORMS)
def test_a_mirror_that_is_not_the_devices_is_reported(knobs, D, dtype, hq, hkv, page, rope, n, one_launch):
    """Under a window, whichever form runs: both lengths fit the caches, so nothing else would show it."""
    if rope and dtype != torch.bfloat16:
        pytest.skip("rotary appends take bf16")
    knobs("ISM_DECODE_WINDOW", one_launch)
    B, cap = 40, 256
    caches = [torch.zeros((B * cap, hkv, D), dtype=dtype, device=DEV) for _ in range(2)]
    x = [torch.ones((B, n, h, D), dtype=dtype, device=DEV) for h in (hq, hkv, hkv)]
    tables = tuple(torch.from_numpy(t).to(DEV) for t in wl.rope_tables(cap, D)) if rope else None
    table = np.arange(2 * B, dtype=np.int32).reshape(B, 2)

    def step(device, host):
        dev = torch.from_numpy(device.copy()).to(DEV)
        args = (dev, host, [n], [1], D ** -0.5, 60, 3)
        if page:
            ism.prefill_append_paged_window(*x, *caches, page, torch.from_numpy(table).to(DEV), table, *args, rope=tables)
        else:
            ism.prefill_append_window(*x, *(c.view(B, cap, hkv, D) for c in caches), *args, rope=tables)

    lens = np.random.default_rng(n).integers(0, cap - n, B).astype(np.int32)
    lens[:3] = 0, 100, cap - n - 1
    ism.check_status(DEV)
    step(lens, lens)
    ism.check_status(DEV)
    one, swapped = lens.copy(), lens.copy()
    one[1] -= 1
    swapped[1:3] = lens[2], lens[1]
    for other in (one, np.maximum(lens - 1, 0), swapped):
        step(lens, other)
        with pytest.raises(ism.IsmError, match="the host's mirrors do not have") as info:
            ism.check_status(DEV)
        assert info.value.code == 1
    step(lens, lens)
    ism.check_status(DEV)
