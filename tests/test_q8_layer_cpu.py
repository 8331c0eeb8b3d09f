"""Q8Mlp on the CPU, its operators replaced by a record of their calls: all of a pass goes
through them, on the stream that the caller gives."""
import pytest
import torch

from paper_2607_21224_amd import layer, q8
from paper_2607_21224_amd.layer import Q8Mlp


class Record:
    """Stands for the module of operators: allocates on the CPU and notes what is called."""
    ACTIVATIONS = q8.ACTIVATIONS

    def __init__(self):
        self.calls = []

    @staticmethod
    def empty_rows(T, D, dtype, device=None):
        return q8.empty_rows(T, D, dtype, "cpu")

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return getattr(q8, name)
        return lambda *a, **kw: self.calls.append((name, a, kw))


def one_pass(monkeypatch, mlp, T, stream):
    record, outside = Record(), []
    monkeypatch.setattr(layer, "q8", record)
    # torch's operations on a stream of their own
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda *a, **kw: outside.append(a))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: outside.append(s) or _Nothing())
    row, grads = (torch.zeros(mlp.numel) for _ in range(2))
    s = mlp.saved(T, device="cpu")
    x = torch.zeros((T, mlp.dim), dtype=mlp.act_dtype)
    mlp.forward(row, x, s, stream=stream)
    mlp.backward(row, x.clone(), s, grads, stream=stream)
    return record.calls, outside, s


class _Nothing:
    def __enter__(self):
        pass

    def __exit__(self, *a):
        pass


@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
@pytest.mark.parametrize("stream", [0, 12345, None])
def test_a_pass_runs_on_the_stream_that_is_given(monkeypatch, kind, stream):
    """The null stream's number, 0, among them: a stream of torch's pool in its place is not
    ordered against it."""
    calls, outside, _ = one_pass(monkeypatch, Q8Mlp(64, 128, kind), 7, stream)
    assert outside == []
    assert calls and all(kw["stream"] is stream for _, _, kw in calls)


def test_the_gated_kind_sums_both_halves_in_one_product(monkeypatch):
    """One rounding of the gradient of the norm's output, and the halves of z where
    the activation looks for them."""
    D, F, T = 64, 128, 7
    mlp = Q8Mlp(D, F, "swiglu")
    calls, _, s = one_pass(monkeypatch, mlp, T, None)
    by_name = {n: [(a, kw) for m, a, kw in calls if m == n] for n in {m for m, _, _ in calls}}
    inputs = by_name["cpdp_q8_grad_input"]
    assert [tuple(a[0].shape) for a, _ in inputs] == [(T, D), (T, 2 * F)]
    assert len(by_name["cpdp_q8_matmul"]) == 2
    # w1 and w1u are one matrix of 2 F rows, g and u are columns of its product
    at, at_u = mlp.tensors["w1"][0], mlp.tensors["w1u"][0]
    assert at_u == at + F * D
    for half in (0, 1):
        z, (w, scale) = s.z[half], s.w1[half]
        assert z.data_ptr() == s.z_all[:, half * F:].data_ptr() and z.shape == (T, F)
        assert w.data_ptr() == s.w_in[0][half * F:].data_ptr() and scale.shape == (F,)
