"""What steps and tables hand to the library, with tensors that say they are on a GPU and a library call that only looks at its arguments."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")


class OnGpu(torch.Tensor):
    is_cuda = True


@pytest.fixture
def calls(monkeypatch):
    """-> (module, the steps of the calls that were made)"""
    from paper_2603_06660_amd import kv
    made = []
    monkeypatch.setattr(kv, "_call", lambda name, device, *a: made.append((name, kv._Step.from_buffer_copy(C.string_at(a[2], C.sizeof(kv._Step))))
                                                                          if name == "pag_kv_extend" else (name, None)))
    return kv, made


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def tables_of(kv, requests, max_pages=3):
    return kv.KvTables.from_tensors(ints(requests), ints(requests, max_pages).as_subclass(OnGpu), ints(9), ints(1), 16)


def step_of(kv, requests, total):
    return kv.KvStep(None, ints(requests + 1), ints(requests), ints(total), ints(total), torch.zeros(total, dtype=torch.int64), granted=ints(requests),
                     lengths=ints(requests), free_count=ints(1), scratch=ints(requests + 1), tokens=total)


def test_a_step_that_does_not_fit_is_refused_every_time_and_stays_as_it_was(calls):
    kv, made = calls
    two, three, step = tables_of(kv, 2), tables_of(kv, 3), step_of(kv, 2, 4)
    for _ in range(3):                       # unbound, then bound to the tables that it fits
        for _ in range(2):
            with pytest.raises(kv.PagError):
                three.extend(ints(3), 4, out=step)
        before = len(made)
        two.extend(ints(2), 4, out=step)
        assert len(made) == before + 1 and made[-1][1].requests == 2 and made[-1][1].table == two.table.data_ptr()
        assert step.table is two.table and made[-1][1].offsets == step.offsets.data_ptr()
    assert len(made) == 3
    with pytest.raises(kv.PagError):
        step._with(3)
    assert step._with(4).requests == 2


def test_lengths_that_tables_took_over_are_not_written_for_others(calls):
    """A committed step's arrays are the tables' own from then on: the next step in it, of any tables, gets new ones."""
    kv, made = calls
    for in_place in (False, True):
        a, b, step = tables_of(kv, 2), tables_of(kv, 2), step_of(kv, 2, 4)
        a.extend(ints(2), 4, out=step, commit=in_place)
        if not in_place:
            a.commit(step)
        held = (a.lengths.data_ptr(), a.free_count.data_ptr())
        assert (step.lengths.data_ptr(), step.free_count.data_ptr()) == held == (a._t.lengths, a._t.free_count)
        for tables in (b, a):
            tables.extend(ints(2), 4, out=step)
            s = made[-1][1]
            assert s.lengths not in held and s.free_count not in held
            assert (s.lengths, s.free_count) == (step.lengths.data_ptr(), step.free_count.data_ptr())
        # nobody has taken these over: they are written again
        again = step.lengths
        a.extend(ints(2), 4, out=step)
        assert step.lengths is again
        # in place for the second tables: theirs, and only theirs
        b.extend(ints(2), 4, out=step, commit=True)
        assert (made[-1][1].lengths, made[-1][1].free_count) == (b._t.lengths, b._t.free_count) and (a._t.lengths, a._t.free_count) == held


def test_two_steps_in_turn_keep_their_arrays(calls):
    kv, made = calls
    a, steps = tables_of(kv, 2), [step_of(kv, 2, 4) for _ in range(2)]
    mine = [s.lengths for s in steps]
    for i in range(6):
        a.extend(ints(2), 4, out=steps[i % 2])
        a.commit(steps[i % 2])
        assert steps[i % 2].lengths is mine[i % 2] and len(steps[i % 2]._holders) == 1


def test_a_refused_call_hands_nothing_over(calls):
    kv, made = calls
    a, step = tables_of(kv, 2), step_of(kv, 2, 4)
    mine = step.lengths
    with pytest.raises(kv.PagError):
        a.extend(ints(3), 4, out=step, commit=True)
    assert step.lengths is mine and not made


def test_tensors_that_require_a_gradient_are_refused(calls):
    kv, _ = calls
    x, slopes = torch.zeros(3, 2, 8, requires_grad=True), torch.zeros(2, requires_grad=True)
    for t in (x, x * 2.0):
        with pytest.raises(kv.PagError, match="gradient"):
            kv._rows(t, (3, 2, 8), x.device, "q")
        kv._rows(t.detach(), (3, 2, 8), x.device, "q")
        with torch.no_grad():
            kv._rows(t, (3, 2, 8), x.device, "q")
    with pytest.raises(kv.PagError, match="gradient"):
        kv._array(slopes, torch.float32, (2,), slopes.device, "slopes")
    assert kv._array(slopes.detach(), torch.float32, (2,), slopes.device, "slopes") == slopes.data_ptr()
