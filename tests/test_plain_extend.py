"""The plain form of page granting that perf/more_operators.py measures against, on the CPU: the same tables, lengths and slots as the oracle,
with every page free and sequences that get no token among them."""
import numpy as np
import pytest

from _latent import extend


@pytest.fixture
def cases(monkeypatch):
    import perf.more_operators as cases
    monkeypatch.setattr(cases, "DEV", "cpu")
    return cases


@pytest.mark.parametrize("L,B,H,page,n,new", [(1, 13, 8, 64, (0, 0), (0, 1)), (2, 5, 2, 32, (0, 0), (0, 3)), (3, 4, 2, 32, (0, 50), (0, 3)), (3, 4, 2, 32, (0, 50), (1, 70)), (1, 1, 1, 32, (0, 0), (1, 1)),
                                              (2, 7, 1, 64, (10, 200), (1, 1))])
def test_plain_extend(cases, L, B, H, page, n, new):
    c = dict(kind="extend", L=L, B=B, Hkv=H, page=page, max_pages=-(-(n[1] + new[1]) // page) + 1, n_lo=n[0], n_hi=n[1], new_lo=new[0], new_hi=new[1])
    first_gets_none = 0
    for seed in range(12):
        s = cases.prepare(c, seed)
        first_gets_none += int(s.n_new[0]) == 0
        before = [x.numpy().copy() for x in (s.table, s.len, s.stack)] + [int(s.count)]
        after, slot, start = cases._plain_extend(s, L, B, H, page)
        table, length, slots, starts, count, missed = extend(*before, page, s.n_new.numpy(), s.T)
        assert missed == dict(full=0, clamped=0)
        assert np.array_equal(s.table.numpy(), table) and np.array_equal(after.numpy(), length) and int(s.count) == count
        assert np.array_equal(slot.numpy(), slots) and np.array_equal(start.numpy(), starts)
    assert first_gets_none or new[0]
