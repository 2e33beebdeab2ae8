"""The engine's sync from microscaled messages among its other syncs: which model a message is a
difference from, what errors it carries, and that a call that fails has moved nothing.

Tolerances as in test_gpu_mx.py: the new model within half a step of fp32 of the 64-bit mean, variances
within 1e-12; x, mx_base and mx_residual bit for bit where a message was quantized."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from test_gpu_mx import _same, _workload

pytestmark = pytest.mark.gpu

FORMATS = [ref.E2M1, ref.E4M3]


@pytest.fixture(scope="module")
def A():
    assert torch.cuda.is_available()
    import paper_2007_06134_amd as A
    return A


def _const(**kw):
    import workloads as W
    return _workload(**{**dict(period_mode=W.PERIOD_CONST, p_init=4, k_s=0, total_steps=200), **kw})


def _sync_is_of(A, eng, w, base, res, fmt=ref.E2M1, feedback=True):
    """One average_mx, checked against the reference's of the replicas with this base and residual."""
    d = ref.difference(eng.x.cpu().numpy(), base, res)
    _, _, v = ref.quantize(d, fmt)
    new, want = ref.average(v, w.offsets(), base)
    var = eng.average_mx(fmt, error_feedback=feedback)
    assert np.all(np.abs(var - want) <= 1e-12 * want)
    got = eng.mx_base.cpu().numpy()
    assert np.all(np.abs(got - new) <= 2.0 ** -24 * (1 + 1e-6) * np.abs(new) + 2.0 ** -149)
    assert _same(eng.x.cpu().numpy(), np.repeat(got[None], w.K, 0)) and eng.get_state().cnt == 0
    left = (d - v).astype(np.float32)
    if feedback:
        assert _same(eng.mx_residual.cpu().numpy(), left)
    return left


def _to_a_sync(eng, kind):
    """Steps, then a sync of fp32 replicas: the model that all workers hold."""
    if kind == "average":
        eng.local_steps(5)
        eng.average()
    elif kind == "step_average":
        eng.local_steps(2)
        eng.step_average()
    elif kind == "run":
        assert eng.run(8)[2] == 2
    else:
        assert eng.run_traced(8)[2] == 2
    assert eng.get_state().cnt == 0
    x = eng.x.cpu().numpy()
    assert _same(x, np.repeat(x[:1], len(x), 0))
    return x[0]


@pytest.mark.parametrize("kind", ["average", "step_average", "run", "run_traced"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_messages_are_differences_from_the_last_sync_of_any_kind(A, fmt, kind):
    """A sync of fp32 replicas between two of messages: the next message starts from its model and owes
    nothing from before."""
    w = _const(K=5)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(4)
        eng.average_mx(fmt)
        for _ in range(2):
            base = _to_a_sync(eng, kind)
            assert _same(eng.mx_base.cpu().numpy(), base) and not eng.mx_residual.any()
            eng.local_steps(4)
            left = _sync_is_of(A, eng, w, base, np.zeros((w.K, w.P), np.float32), fmt)
            base = eng.mx_base.cpu().numpy()
            eng.local_steps(3)
            _sync_is_of(A, eng, w, base, left, fmt)


@pytest.mark.parametrize("kind", ["average", "step_average", "run", "run_traced"])
def test_the_first_messages_after_other_syncs_need_a_base(A, kind):
    """Without one they would be whole models in a few bits: refused, with nothing moved, until mx_begin."""
    w = _const(K=4)
    with A.Adpsgd.from_workload(w) as eng:
        base = _to_a_sync(eng, kind)
        eng.local_steps(3)
        x, st = eng.x.clone(), eng.get_state()
        with pytest.raises(A.AdpsgdError, match="mx_begin") as e:
            eng.average_mx()
        assert e.value.code == A.ESTATE and torch.equal(eng.x, x)
        assert (eng.get_state().cnt, eng.get_state().t) == (st.cnt, st.t)
        with pytest.raises(ValueError):        # the workers have stepped on: whose parameters?
            eng.mx_begin()
        eng.mx_begin(torch.from_numpy(base))
        _sync_is_of(A, eng, w, base, np.zeros((w.K, w.P), np.float32))
    with A.Adpsgd.from_workload(w) as eng:
        base = _to_a_sync(eng, kind)
        eng.mx_begin()
        assert _same(eng.mx_base.cpu().numpy(), base)
        eng.local_steps(3)
        _sync_is_of(A, eng, w, base, np.zeros((w.K, w.P), np.float32))


def test_a_run_that_ends_between_syncs(A):
    """Its last sync's model is gone: messages are refused until there is a base again.  One without a
    sync in it leaves the base and the residual as they are."""
    w = _const(K=3)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(1)
        eng.average_mx()
        base, res = eng.mx_base.cpu().numpy(), eng.mx_residual.cpu().numpy()
        assert eng.run(3)[2] == 0
        left = _sync_is_of(A, eng, w, base, res)
        base = eng.mx_base.cpu().numpy()
        with pytest.raises(A.AdpsgdError):
            eng.run(-1)                                     # refused: nothing ran
        eng.local_steps(2)
        _sync_is_of(A, eng, w, base, left)
        assert eng.run(6)[2] == 1
        x = eng.x.clone()
        with pytest.raises(A.AdpsgdError, match="mx_begin"):
            eng.average_mx()
        assert torch.equal(eng.x, x)
        eng.average()                                       # a sync that the base follows
        base = eng.x[0].cpu().numpy()
        eng.local_steps(3)
        _sync_is_of(A, eng, w, base, np.zeros((w.K, w.P), np.float32))
        assert eng.run(6)[2] == 1
        eng.reset()                                         # zero replicas, zero base
        eng.local_steps(3)
        _sync_is_of(A, eng, w, np.zeros(w.P, np.float32), np.zeros((w.K, w.P), np.float32))


def test_a_run_that_stops_at_a_sum_that_is_not_finite(A):
    w = _workload(K=3, total_steps=40, k_s=0)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(3)
        eng.average_mx()
        eng.x[0, 5] = float("nan")
        with pytest.raises(A.AdpsgdError) as e:
            eng.run(20)
        assert e.value.code == A.ENONFINITE
        with pytest.raises(A.AdpsgdError, match="mx_begin"):
            eng.average_mx()


def test_errors_are_not_carried_past_a_message_without_feedback(A):
    w = _const(K=4)
    zero = np.zeros((w.K, w.P), np.float32)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(4)
        left = _sync_is_of(A, eng, w, np.zeros(w.P, np.float32), zero)
        assert left.any()
        base = eng.mx_base.cpu().numpy()
        eng.local_steps(4)
        _sync_is_of(A, eng, w, base, None, feedback=False)
        assert not eng.mx_residual.any()
        base = eng.mx_base.cpu().numpy()
        eng.local_steps(4)
        _sync_is_of(A, eng, w, base, zero)


@pytest.mark.parametrize("where", ["cpu", "cuda", "stream"])
def test_resumes_bit_exactly_from_mx_begin(A, where):
    """A checkpoint of x, m, the controller, mx_base and mx_residual into a new engine."""
    w = _workload(K=3)
    with A.Adpsgd.from_workload(w) as eng:
        for _ in range(3):
            eng.local_steps(4)
            eng.average_mx()
        saved = [t.clone() for t in (eng.x, eng.m, eng.mx_base, eng.mx_residual)], eng.get_state()
        eng.local_steps(4)
        want = eng.average_mx(), eng.x.clone(), eng.mx_residual.clone()
    torch.cuda.synchronize()
    with A.Adpsgd.from_workload(w, stream=torch.cuda.Stream() if where == "stream" else None) as eng:
        eng.x.copy_(saved[0][0])
        eng.m.copy_(saved[0][1])
        eng.set_state(saved[1])
        # (on the caller's stream just before, as the copies above, and dropped just behind)
        base, res = [t.cpu() if where == "cpu" else t * 1.0 for t in saved[0][2:]]
        eng.mx_begin(base, res)
        del base, res
        eng.local_steps(4)
        assert np.array_equal(eng.average_mx(), want[0])
        assert torch.equal(eng.x, want[1]) and torch.equal(eng.mx_residual, want[2])


def test_another_runs_state_needs_its_base(A):
    """A checkpoint without mx_base: refused, as the last sync's model is not known."""
    w = _const(K=2)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(5)
        st = eng.get_state()
        st.p = 3
        eng.set_state(st)                          # (its own, changed)
        eng.average_mx()
        saved = eng.x.clone(), eng.m.clone(), eng.get_state()
    with A.Adpsgd.from_workload(w) as eng:
        eng.x.copy_(saved[0])
        eng.m.copy_(saved[1])
        eng.set_state(saved[2])
        with pytest.raises(A.AdpsgdError, match="mx_begin"):
            eng.average_mx()
        eng.mx_begin()                             # (taken right behind a sync)
        eng.local_steps(2)
        _sync_is_of(A, eng, w, saved[0][0].cpu().numpy(), np.zeros((w.K, w.P), np.float32))


def test_mx_begin_refuses(A):
    w = _const(K=2)
    with A.Adpsgd.from_workload(w) as eng:
        P, K = w.P, w.K
        good = torch.zeros(P)
        for args in ((good.double(),), (good[:-1],), (good[None],), (good, torch.zeros(P)), (good, torch.zeros(K, P).double()),
                     (good, torch.zeros(K, P + 1)), (None, torch.zeros(K + 1, P))):
            with pytest.raises(ValueError):
                eng.mx_begin(*args)
            assert eng.mx_base is None and eng.mx_residual is None
        eng.mx_begin(good, torch.zeros(K, P))


@pytest.mark.parametrize("fails", ["adpsgd_mx_quantize", "adpsgd_mx_product_workspace", "adpsgd_mx_average_workspace"])
def test_a_sync_that_fails_has_moved_nothing(A, monkeypatch, fails):
    """Its buffers are there before anything is sent, and the counter restarts behind the last call."""
    w = _const(K=3)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(4)
        eng.average_mx(products=True)
        eng.local_steps(3)
        before = [t.clone() for t in (eng.x, eng.mx_base, eng.mx_residual)]
        real = getattr(A._native.lib, fails)
        with monkeypatch.context() as m:
            if fails.endswith("_workspace"):       # more than any GPU has: torch raises at once
                m.setattr(A._native.lib, fails, lambda *a: 1 << 50)
            else:
                m.setattr(A._native.lib, fails, lambda *a: A.EINVAL)
            with pytest.raises(RuntimeError):
                eng.average_mx(A.MX_E4M3, products=True)
        assert getattr(A._native.lib, fails) is real
        assert eng.get_state().cnt == 3
        for t, b in zip((eng.x, eng.mx_base, eng.mx_residual), before):
            assert torch.equal(t, b)
        base, res = before[1].cpu().numpy(), before[2].cpu().numpy()
        _sync_is_of(A, eng, w, base, res, A.MX_E4M3)


def test_torchs_default_type_does_not_matter(A):
    w = _const(K=2)
    old = torch.get_default_dtype()
    torch.set_default_dtype(torch.float64)
    try:
        with A.Adpsgd.from_workload(w) as eng:
            eng.local_steps(2)
            assert np.all(np.isfinite(eng.average_mx(products=True)[0]))
            assert eng.mx_base.dtype == eng.mx_residual.dtype == torch.float32
    finally:
        torch.set_default_dtype(old)


def test_inference_mode_does_not_matter(A):
    """A sync inside it leaves the engine usable outside, and the other way round."""
    w = _const(K=2)
    zero = np.zeros((w.K, w.P), np.float32)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(2)
        with torch.inference_mode():
            eng.average_mx()
        eng.local_steps(2)
        eng.average()
        base = eng.x[0].cpu().numpy()
        eng.local_steps(2)
        with torch.inference_mode():
            _sync_is_of(A, eng, w, base, zero)
        eng.reset()
        assert not eng.mx_base.any() and not eng.mx_residual.any()
        with torch.inference_mode():
            eng.mx_begin(torch.ones(w.P), torch.ones(w.K, w.P))
        eng.mx_begin()
        eng.local_steps(2)
        _sync_is_of(A, eng, w, np.zeros(w.P, np.float32), zero)


def test_replicas_that_require_gradients(A):
    """The engine's syncs update them as an optimizer does."""
    w = _const(K=2)
    with A.Adpsgd.from_workload(w) as eng:
        eng.x.requires_grad_()
        eng.local_steps(2)
        before = eng.x._version
        eng.average_mx()
        assert eng.x._version > before
        eng.average()
        eng.mx_begin()


def test_engine_sync_of_a_larger_model(A):
    """Several chunks a tensor, tensors that share chunks, rows of many blocks."""
    import workloads as W
    w = _const(K=8, sizes=W.log_uniform_sizes(1002, 62, 64, 2.4e6, 1_300_001, multiple=1, minimum=1))
    assert w.P == 1_300_001
    with A.Adpsgd.from_workload(w) as eng:
        base, res = np.zeros(w.P, np.float32), np.zeros((w.K, w.P), np.float32)
        for fmt in (A.MX_E2M1, A.MX_E4M3):
            eng.local_steps(4)
            res = _sync_is_of(A, eng, w, base, res, fmt)
            base = eng.mx_base.cpu().numpy()
        eng.local_steps(1)
        eng.average()
        base = eng.x[0].cpu().numpy()
        eng.local_steps(2)
        _sync_is_of(A, eng, w, base, np.zeros((w.K, w.P), np.float32))
