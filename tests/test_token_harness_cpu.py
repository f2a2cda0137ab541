"""CPU-side checks of what the harness asks of the tensors it hands to the language-model operators.  Tensors are fake ones of a
second GPU: nothing is allocated, and a call that is refused reaches no library."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def sim():
    """What a simulation of two nodes on GPU 0 knows, without a library context."""
    from paper_2105_09080_amd import harness
    s = object.__new__(harness.Simulation)
    s.n, s.d, s.ld, s.ctx = 2, 64, 64, None
    s.device, s._device_index, s._stream_address = torch.device("cuda:0"), 0, 0
    s._foreign = lambda: False
    return s


@pytest.fixture
def fake():
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        yield lambda *shape, dtype=torch.float32, device="cuda:0": torch.empty(shape, dtype=dtype, device=device)


@pytest.mark.parametrize("other", ["cuda:1", "cpu"])
def test_tensors_of_another_device_are_refused(sim, fake, other):
    tok, x, stats = fake(2, 3, dtype=torch.int32), fake(2, 3, 8), fake(2, 3, 2)
    tok1, x1, stats1 = fake(2, 3, dtype=torch.int32, device=other), fake(2, 3, 8, device=other), fake(2, 3, 2, device=other)
    for call in (lambda: sim.embed(tok1, 0, 4, 8), lambda: sim.embed_grad(tok1, x, 0, 4), lambda: sim.embed_grad(tok, x1, 0, 4),
                 lambda: sim.dropout(x1, 0.5, seed=1), lambda: sim.dropout(x, 0.5, seed=1, residual=x1),
                 lambda: sim.dropout(x, 0.5, seed=1, out=x1), lambda: sim.layer_norm(x1, 0, 8),
                 lambda: sim.layer_norm(x, 0, 8, residual=x1), lambda: sim.layer_norm_grad(x1, x1, stats1, 0, 8),
                 lambda: sim.layer_norm_grad(x, x1, stats, 0, 8), lambda: sim.layer_norm_grad(x, x, stats1, 0, 8),
                 lambda: sim.layer_norm_grad(x, x, stats, 0, 8, more=x1), lambda: sim.token_loss(x1, tok),
                 lambda: sim.token_loss(x, tok1), lambda: sim.token_loss(x, tok, grad=x1)):
        with pytest.raises(ValueError, match="GPU|device|stats"):
            call()


def test_tensors_that_autograd_follows_are_refused(sim, fake):
    """What comes back would be cut off from them without a word."""
    tok, x, stats = fake(2, 3, dtype=torch.int32), fake(2, 3, 8), fake(2, 3, 2)
    leaf = fake(2, 3, 8).requires_grad_()
    for w in (leaf, leaf * 2):
        calls = (lambda: sim.embed_grad(tok, w, 0, 4), lambda: sim.dropout(w, 0.5, seed=1), lambda: sim.dropout(x, 0.5, seed=1, residual=w),
                 lambda: sim.dropout(x, 0.5, seed=1, out=w), lambda: sim.layer_norm(w, 0, 8), lambda: sim.layer_norm(x, 0, 8, residual=w),
                 lambda: sim.layer_norm_grad(w, x, stats, 0, 8), lambda: sim.layer_norm_grad(x, w, stats, 0, 8),
                 lambda: sim.layer_norm_grad(x, x, stats, 0, 8, more=w), lambda: sim.token_loss(w, tok), lambda: sim.token_loss(x, tok, grad=w))
        for call in calls:
            with pytest.raises(ValueError, match="requires grad"):
                call()
        assert sim._rows(w.detach(), x)[:2] == (3, 8)
        with torch.no_grad():
            assert sim._rows(w, x)[:2] == (3, 8)


@pytest.mark.parametrize("ld", [64, 70])
def test_the_state_that_is_handed_out_is_a_view(sim, monkeypatch, ld):
    """Its shape is the caller's to change; the bound buffer keeps its own."""
    from paper_2105_09080_amd import harness
    sim.ld, buf, sim.g = ld, torch.zeros(2, ld), torch.ones(2, ld)
    sim._addr = {buf.data_ptr(): buf}
    monkeypatch.setattr(harness.B, "gpga_current_x", lambda ctx: buf.data_ptr())
    for name, whole in (("X", buf), ("G", sim.g)):
        getattr(sim, name).t_()
        getattr(sim, name).unsqueeze_(0)
        assert getattr(sim, name).shape == (2, 64) and whole.shape == (2, ld) and getattr(sim, name).data_ptr() == whole.data_ptr()
        getattr(sim, name).fill_(3.0)
        assert bool((whole[:, :64] == 3.0).all())
