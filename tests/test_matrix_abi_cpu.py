"""CPU-side checks of the operators whose parameters are matrices: header and binding say the same, a NULL context and numbers that do
not fit are refused, and the harness refuses tensors that it cannot hand on.  No kernel is launched here."""
import ctypes
import os
import re

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("gpga_gated_ff", "gpga_gated_ff_grad", "gpga_orthogonalize")


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gpga.h")).read(), flags=re.S)


def test_activations_are_those_of_the_header():
    from paper_2105_09080_amd import binding as B
    values = dict(re.findall(r"GPGA_(SILU|GELU) = (\d)", header()))
    assert {k.lower(): int(v) for k, v in values.items()} == B.ACTIVATION


@pytest.mark.parametrize("name", NAMES)
def test_arguments_are_those_of_the_header(name):
    from paper_2105_09080_amd import binding as B
    arguments = re.search(name + r"\s*\(([^)]*)\)", header()).group(1).split(",")
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}
    want = [ctypes.c_void_p if "*" in a else kinds[a.split()[0]] for a in arguments]
    assert next(types for n, _, types in B.SIGNATURES if n == name) == want
    assert B.raw_status(name, *[None if t is ctypes.c_void_p else 0 for t in want]) == B.GPGA_EINVAL


@pytest.mark.parametrize("wide", [2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1])
def test_numbers_that_do_not_fit_their_argument_are_refused(wide):
    from paper_2105_09080_amd import binding as B
    calls = ((("T", "D", "F"), lambda T=1, D=1, F=1: B.gpga_gated_ff(None, None, T, D, F, 1, 0, 0, 0, 0, 0, None, None)),
             (("T", "D", "F"), lambda T=1, D=1, F=1: B.gpga_gated_ff_grad(None, None, None, None, T, D, F, 1, 0, 0, 0, 0, 0, None)),
             (("rows", "cols", "count", "steps"), lambda rows=1, cols=1, count=1, steps=1: B.gpga_orthogonalize(
                 None, 0, rows, cols, count, None, 0.0, False, steps, 1.5, -0.5, 0.0, 0.0, 1.0)))
    for names, call in calls:
        for name in names:
            with pytest.raises(B.GpgaError, match="32 bits"):
                call(**{name: wide})
            with pytest.raises(B.GpgaError) as e:
                call(**{name: -1})
            assert "32 bits" not in str(e.value) and e.value.status == B.GPGA_EINVAL


@pytest.fixture
def sim():
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
    x, hidden, v = fake(2, 3, 8), fake(2, 3, 20), fake(2, 24)
    x1, hidden1, v1 = fake(2, 3, 8, device=other), fake(2, 3, 20, device=other), fake(2, 24, device=other)
    for call in (lambda: sim.gated_ff(x1, 0, 1, 2, 10), lambda: sim.gated_ff_grad(x1, x, hidden, 0, 1, 2), lambda: sim.gated_ff_grad(x, x1, hidden, 0, 1, 2),
                 lambda: sim.gated_ff_grad(x, x, hidden1, 0, 1, 2), lambda: sim.orthogonalize(0, 4, 6, velocity=v1, mu=0.5)):
        with pytest.raises(ValueError, match="GPU|device"):
            call()


def test_tensors_that_autograd_follows_and_wrong_shapes_are_refused(sim, fake):
    x, hidden, v = fake(2, 3, 8), fake(2, 3, 20), fake(2, 24)
    leaf, hleaf, vleaf = fake(2, 3, 8).requires_grad_(), fake(2, 3, 20).requires_grad_(), fake(2, 24).requires_grad_()
    for call in (lambda: sim.gated_ff(leaf, 0, 1, 2, 10), lambda: sim.gated_ff_grad(leaf, x, hidden, 0, 1, 2), lambda: sim.gated_ff_grad(x, leaf, hidden, 0, 1, 2),
                 lambda: sim.gated_ff_grad(x, x, hleaf, 0, 1, 2), lambda: sim.orthogonalize(0, 4, 6, velocity=vleaf, mu=0.5)):
        with pytest.raises(ValueError, match="requires grad"):
            call()
    for h in (fake(2, 3, 19), fake(2, 4, 20), fake(2, 3, 40)[..., ::2], fake(2, 3, 20, dtype=torch.bfloat16), fake(2, 60)):
        with pytest.raises(ValueError, match="hidden"):
            sim.gated_ff_grad(x, x, h, 0, 1, 2)
    for w in (fake(2, 23), fake(2, 48)[:, ::2], fake(2, 24, dtype=torch.float64)):
        with pytest.raises(ValueError, match="velocity"):
            sim.orthogonalize(0, 4, 6, velocity=w, mu=0.5)
    with pytest.raises(ValueError, match="act"):
        sim.gated_ff(x, 0, 1, 2, 10, act="relu")
