"""The cache's calls have no forward derivative either: tensors that carry a tangent are refused, since what comes out would have lost it."""
import pytest
from test_kv_abi import kv  # noqa: F401

torch = pytest.importorskip("torch")
forward = torch.autograd.forward_ad


def test_tensors_that_carry_a_tangent_are_refused(kv):
    x, slopes = torch.zeros(3, 2, 8), torch.zeros(2)
    rows = lambda t: kv._rows(t, (3, 2, 8), t.device, "q")
    array = lambda t: kv._array(t, torch.float32, (2,), t.device, "slopes")
    with forward.dual_level():
        dual, dual_slopes = forward.make_dual(x, torch.ones_like(x)), forward.make_dual(slopes, torch.ones_like(slopes))
        assert not dual.requires_grad
        for call in (lambda: rows(dual), lambda: rows(2.0 * dual), lambda: array(dual_slopes)):
            with pytest.raises(kv.PagError, match="tangent"):
                call()
            # no_grad leaves tangents on
            with torch.no_grad(), pytest.raises(kv.PagError, match="tangent"):
                call()
            with torch.inference_mode():
                call()
        # tensors beside it, and its value alone, are what they were
        assert rows(x) == (x.data_ptr(), 16, 8) and array(slopes) == slopes.data_ptr()
        assert rows(forward.unpack_dual(dual).primal)[0] == x.data_ptr()
    assert rows(x)[0] == x.data_ptr()


@pytest.mark.gpu
def test_calls_on_tensors_that_carry_a_tangent_are_refused(kv):
    cache, tables = kv.KvCache(4, 2, 64, 16), kv.KvTables(1, 4, 4, 16, device="cuda")
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    step, blocks, rotation = tables.extend(ints([3]), 3), kv.KvBlocks(cache, 16), kv.KvRotation(torch.rand(8, device="cuda"))
    x, q = torch.randn(3, 2, 64, device="cuda").half(), torch.randn(3, 4, 64, device="cuda").half()
    ids, chosen = torch.zeros(3, 2, 2, dtype=torch.int64, device="cuda"), torch.zeros(3, 2, 2, dtype=torch.int32, device="cuda")
    slopes = torch.ones(4, device="cuda")
    calls = [lambda f: cache.append(f(x), x, step.slots), lambda f: cache.append(x, f(x), step.slots), lambda f: cache.attend(f(q), step),
             lambda f: cache.attend(q, step, slopes=f(slopes)), lambda f: cache.attend_selected(f(q), ids, step),
             lambda f: cache.append_rotated(x, x, step.slots, step.positions, rotation, q=f(q)), lambda f: cache.append_rotated(f(x), x, step.slots, step.positions, rotation),
             lambda f: cache.append_rotated(x, x, step.slots, step.positions, kv.KvRotation(f(torch.rand(8, device="cuda")))), lambda f: blocks.select(f(q), step, 2),
             lambda f: blocks.attend(f(q), chosen, step)]
    with forward.dual_level():
        for call in calls:
            with pytest.raises(kv.PagError, match="tangent"):
                call(lambda t: forward.make_dual(t, torch.ones_like(t)))
            call(lambda t: t)
