"""The operators of include/switchsd_target.h at the edges of what their header takes: counts of pages that no map wrote,
against the plain implementations in 64 bits (target_ref.py)."""
import numpy as np
import pytest

from tests import target_ref as ref

pytestmark = pytest.mark.gpu


def _fw():
    import paper_2609_20186_gb300 as fw
    return fw


def _i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


# --- block tables and slot maps -----------------------------------------------------------------------------------
@pytest.mark.parametrize("B", [4, 70, 130, 170, 200, 300, 1100])
@pytest.mark.parametrize("bad", [-1, -2, -5, -2**31, 9, 2**31 - 1])
def test_map_leaves_rows_with_a_bad_count_of_pages_alone(B, bad):
    """A row whose held lies outside [0, blocks] keeps it, gets no slots, and moves no page: the pool's count, list and
    tables are those of a step that skips the row.  B: clusters of 1, 3, 5, 6, 7 and 8 CTAs."""
    import torch
    fw = _fw()
    T, page, blocks = 3, 16, 8
    rng = np.random.default_rng(B)
    pages = B * blocks
    free = rng.permutation(pages).astype(np.int32)
    st = ref.MapState(B, blocks, free)
    table, held = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    fl, fc = _i32(free), _i32([pages])
    rows = [1, B // 2, B - 1]
    for step in range(3):
        lens, new = rng.integers(0, page * blocks - T, B), rng.integers(0, T + 1, B)
        wl = lens.copy()
        good = held.clone()
        if step == 1:
            held[rows] = bad
            wl[rows] = -1                        # how the plain form leaves a row out
        before = held.clone()
        slots, status = torch.full((B, T), 7, dtype=torch.int32, device="cuda"), torch.full((B,), 7, dtype=torch.int32, device="cuda")
        fw.switchsd_kv_map(_i32(lens), _i32(new), table, held, fl, fc, slots, page=page, status=status)
        want_slots, want_status = st.step(wl.tolist(), new.tolist(), T, page)
        wt, wh, wf, wc = st.arrays()
        assert int(fc.cpu()[0]) == wc
        assert np.array_equal(fl.cpu().numpy(), wf)
        assert np.array_equal(table.cpu().numpy(), wt)
        assert np.array_equal(status.cpu().numpy(), want_status)
        assert np.array_equal(slots.cpu().numpy(), want_slots)
        if step == 1:
            assert torch.equal(held[rows], before[rows])
            held[rows] = good[rows]              # mended by the caller: the next step has every page
        assert np.array_equal(held.cpu().numpy(), wh)
    everything = np.concatenate([wf[:wc], wt[wt >= 0]])
    assert np.array_equal(np.sort(everything), np.arange(pages))  # no page lost, none held twice


@pytest.mark.parametrize("B,T", [(1, 2**31 - 1), (33, (2**31 - 1) // 33)])
def test_map_of_the_longest_step(B, T):
    """B * T just below 2^31: the slots' last places."""
    import torch
    fw = _fw()
    page, blocks, n = 256, 4, 700
    table, held = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    fl, fc = _i32(np.arange(B * blocks)), _i32([B * blocks])
    slots, status = torch.full((B, T), 7, dtype=torch.int32, device="cuda"), torch.full((B,), 7, dtype=torch.int32, device="cuda")
    fw.switchsd_kv_map(_i32(np.full(B, 100)), _i32(np.full(B, n)), table, held, fl, fc, slots, page=page, status=status)
    assert not status.any() and (held == 4).all()
    p = torch.arange(100, 100 + n, device="cuda")
    assert torch.equal(slots[:, :n].long(), table.long()[:, p // page] * page + p % page)
    for b in range(B):
        assert (slots[b, n:] == -1).all()
