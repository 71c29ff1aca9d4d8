"""Slots that share pages: fork, copy-on-write, truncate and compact (host only)."""
import numpy as np
import pytest

P = 128


@pytest.fixture(scope="module")
def B():
    from paper_2402_11809_b200 import build
    build.build()
    from paper_2402_11809_b200 import binding
    return binding


def test_fork_shares_and_write_makes_own(B):
    pg = B.Pager(10, 6, 4)
    a = pg.admit()
    pg.reserve(a, 300)                                       # pages 0, 1, 2
    b = pg.fork(a, 300)
    assert pg.free_pages == 7 and [pg.page_refs(i) for i in range(4)] == [2, 2, 2, 0] and pg.page_refs(10) == -1
    assert (pg.batch_table([a])[0] == pg.batch_table([b])[0]).all() and pg.rows(b) == 3 * P
    pg.reserve(b, 400)                                       # one page of its own behind the shared ones
    mv = pg.make_writable(b, 300, 100)
    assert mv.tolist() == [[2, 4, 300 - 2 * P]]
    assert pg.batch_table([b])[0].tolist() == [0, 1, 4, 3, -1, -1] and pg.batch_table([a])[0, :3].tolist() == [0, 1, 2]
    assert len(pg.make_writable(b, 300, 100)) == 0           # its own by now
    assert len(pg.make_writable(a, 300, 84)) == 0            # nobody else holds page 2 any more
    pg.release(a)
    assert pg.page_refs(0) == 1 and pg.page_refs(2) == 0 and pg.free_pages == 6
    pg.release(b)
    assert pg.free_pages == 10
    pg.close()


def test_page_boundary_needs_no_copy(B):
    pg = B.Pager(8, 4, 2)
    a = pg.admit()
    pg.reserve(a, 2 * P)
    b = pg.fork(a, 2 * P)
    pg.reserve(b, 2 * P + 5)
    assert len(pg.make_writable(b, 2 * P, 5)) == 0           # the row begins a page that nobody shares
    assert len(pg.make_writable(b, P, P)) == 0 and pg.page_refs(1) == 1   # a shared page whose rows are all written anew
    assert len(pg.make_writable(b, 0, 0)) == 0
    pg.close()


def test_refusals_change_nothing(B):
    pg = B.Pager(3, 4, 2)
    a = pg.admit()
    pg.reserve(a, 3 * P)
    for bad in (-1, 3 * P + 1, 4 * P):
        with pytest.raises(B.SpaceError) as e:
            pg.fork(a, bad)
        assert e.value.code == B.E_INVALID_ARG
    b = pg.fork(a, 200)
    with pytest.raises(B.SpaceError) as e:
        pg.fork(a, 0)
    assert e.value.code == B.E_WORKSPACE                      # no slot left
    before = pg.batch_table([a, b]).tolist()
    with pytest.raises(B.SpaceError) as e:
        pg.make_writable(b, 100, 10)
    assert e.value.code == B.E_WORKSPACE                      # no free page
    with pytest.raises(B.SpaceError) as e:
        pg.make_writable(b, 250, 10)                          # rows that are not reserved
    assert e.value.code == B.E_INVALID_ARG
    assert pg.batch_table([a, b]).tolist() == before and pg.page_refs(0) == 2
    for call in (lambda: pg.truncate(b, -1), lambda: pg.truncate(7, 0), lambda: pg.make_writable(b, -1, 5)):
        with pytest.raises(B.SpaceError) as e:
            call()
        assert e.value.code == B.E_INVALID_ARG
    pg.truncate(a, 2 * P)                                     # page 2 is free again
    assert pg.make_writable(b, 100, 10).tolist() == [[0, 2, 100]]
    pg.truncate(a, 1)
    assert pg.rows(a) == P and pg.page_refs(1) == 1           # b still holds it
    pg.close()


def test_no_room_for_the_move(B):
    import ctypes as C
    pg = B.Pager(4, 2, 2)
    a = pg.admit()
    pg.reserve(a, 10)
    b = pg.fork(a, 10)
    n = C.c_int32(9)
    assert B.lib.space_pager_make_writable(pg._h, b, 10, 1, None, 0, C.byref(n)) == B.E_WORKSPACE and n.value == 0
    assert pg.page_refs(0) == 2
    assert B.lib.space_pager_make_writable(pg._h, b, 0, 1, None, 0, C.byref(n)) == B.OK   # nothing is kept: no move
    pg.close()


def test_random_walk_against_a_model(B):
    """Contents as the moves leave them, reference counts and free pages against a model of its own."""
    rng = np.random.default_rng(5)
    n_pages, pps, slots = 23, 5, 6
    pg = B.Pager(n_pages, pps, slots)
    store = np.zeros((n_pages, P), dtype=np.int64)            # one number per row
    model, stamp = {}, 0                                      # slot -> its rows

    def run(moves):
        assert not set(moves[:, 0]) & set(moves[:, 1]) and len(set(moves[:, 1])) == len(moves)
        for s, t, r in moves:
            store[t, :r] = store[s, :r]

    for _ in range(1500):
        op = int(rng.integers(0, 6))
        live = list(model)
        if op == 0 and len(live) < slots:
            model[pg.admit()] = []
        elif op == 1 and live:
            s = live[rng.integers(len(live))]
            add = int(rng.integers(1, 200))
            n = len(model[s])
            if n + add > pps * P:
                continue
            try:
                pg.reserve(s, n + add)
                run(pg.make_writable(s, n, add))
            except B.SpaceError as e:
                assert e.code == B.E_WORKSPACE
                continue
            t = pg.batch_table([s])[0]
            for r in range(n, n + add):
                stamp += 1
                store[t[r // P], r % P] = stamp
                model[s].append(stamp)
        elif op == 2 and live and len(live) < slots:
            s = live[rng.integers(len(live))]
            n = int(rng.integers(0, len(model[s]) + 1))
            model[pg.fork(s, n)] = model[s][:n]
        elif op == 3 and live:
            s = live[rng.integers(len(live))]
            n = int(rng.integers(0, len(model[s]) + 1))
            pg.truncate(s, n)
            model[s] = model[s][:n]
        elif op == 4 and live and rng.random() < 0.4:
            s = live[rng.integers(len(live))]
            pg.release(s)
            del model[s]
        elif op == 5 and rng.random() < 0.3:
            while True:
                mv = pg.compact(int(rng.integers(1, 6)))
                run(mv)
                if not len(mv):
                    break
            used = n_pages - pg.free_pages
            assert all((pg.page_refs(i) > 0) == (i < used) for i in range(n_pages))
        refs = np.zeros(n_pages, dtype=int)
        for s, rows in model.items():
            t = pg.batch_table([s])[0]
            held = pg.rows(s) // P
            assert (t[:held] >= 0).all() and (t[held:] == -1).all() and held * P >= len(rows)
            np.add.at(refs, t[:held], 1)
            assert [int(store[t[r // P], r % P]) for r in range(len(rows))] == rows
        assert refs.tolist() == [pg.page_refs(i) for i in range(n_pages)] and pg.free_pages == int((refs == 0).sum())
    pg.close()
