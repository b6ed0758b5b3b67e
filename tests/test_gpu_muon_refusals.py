"""A training step with `muon` that is refused leaves the worker as it was."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2009_14783_amd import binding
    binding.lib()            # a missing library is a failure, not a skip
    return binding


@pytest.mark.parametrize("which", ["encoder", "pairs"])
def test_refused_steps_leave_the_worker_as_it_was(hs, which):
    from paper_2009_14783_amd import synth
    from paper_2009_14783_amd.step import PairWorker, Worker
    pairs = which == "pairs"
    model = synth.S2S_MODELS["s2s_tiny"] if pairs else synth.MODELS["tiny"]
    lay = hs.hs_s2s_param_layout(hs.make_s2s_cfg(**model)) if pairs else hs.hs_param_layout(hs.make_cfg(**model))
    worker = (PairWorker if pairs else Worker)(model, "bf16", synth.init_params(lay, 3))
    rng = synth.rng_for(4)
    mb = synth.make_pair_batch(rng, [16, 9], [20, 7], 24, 32, model["vocab"], "uniform") if pairs else \
        synth.make_micro_batch(rng, [16, 32], 32, model["vocab"], "uniform")
    batches = [worker.upload(mb)]
    adam = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-6)
    worker.train_step(batches, adam, muon={})
    torch.cuda.synchronize()
    state = lambda: [t.clone() for t in (worker.w, worker.m, worker.v, worker.w_lowp)]
    before = state()
    without = {k: v for k, v in adam.items() if k != "beta1"}
    for bad, muon, denom, error in ((without, {}, None, KeyError), (dict(adam, beta2=1.0), {}, None, hs.HsError), (dict(adam, eps=-1.0), {}, None, hs.HsError),
                                    (adam, dict(steps=70), None, hs.HsError), (adam, dict(coeff=np.zeros((4, 3))), None, hs.HsError),
                                    (adam, dict(momentum=1.0), None, hs.HsError), (adam, {}, -1.0, hs.HsError)):
        with pytest.raises(error):
            worker.train_step(batches, bad, denom=denom, muon=muon)
        with pytest.raises(error):
            worker.matrices.apply(worker, 4.0 if denom is None else denom, bad, muon, worker.t + 1)
        torch.cuda.synchronize()
        assert worker.t == 1
        assert all(torch.equal(a, b) for a, b in zip(before, state())), (bad, muon)
    worker.train_step(batches, adam, muon={})
    torch.cuda.synchronize()
    assert worker.t == 2 and not torch.equal(before[0], worker.w)
    worker.close()
