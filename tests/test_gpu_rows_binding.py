"""What the binding refuses of the arrays it is given, and what it tells torch of the memory it writes."""
import pytest
import torch

from test_gpu_binding import _case, _ring
from test_gpu_distill import inputs

pytestmark = pytest.mark.gpu


def batch(N=6, V=500, K=8):
    s, ids, t, lse = inputs(N, V, K, "fp32", seed=1)
    return s.cuda(), ids.cuda(), t.cuda(), lse.cuda(), torch.ones(N, device="cuda")


WRONG = [torch.uint8, torch.bool, torch.int16, torch.int64, torch.float32]


@pytest.mark.parametrize("dtype", WRONG)
def test_the_row_error_array_is_of_32_bit_integers(gpu_lib, dtype):
    """The kernels write four bytes per row: an array of smaller elements would be written past its end."""
    z, ids, t, lse, w = batch()
    T, u = torch.ones(6, device="cuda"), torch.full((6,), 0.5, device="cuda")
    calls = [(lambda o: gpu_lib.sample(z, T, u, kept=True, out=o)), (lambda o: gpu_lib.top_logits(z, 8, out=o)),
             (lambda o: gpu_lib.distill_loss(z, ids, t, teacher_lse=lse, out=o)),
             (lambda o: gpu_lib.distill_step(z, ids, t, w, teacher_lse=lse, out=o))]
    for call in calls:
        out = call(None)
        for good in (torch.int32, torch.uint32):
            call(dict(out, row_err=torch.empty(6, dtype=good, device="cuda")))
        with pytest.raises(gpu_lib.DsdeError, match="row_err must be torch.int32, got " + str(dtype)):
            call(dict(out, row_err=torch.zeros(6, dtype=dtype, device="cuda")))
        with pytest.raises(gpu_lib.DsdeError, match="row_err has 5 elements, needs 6"):
            call(dict(out, row_err=torch.zeros(5, dtype=torch.int32, device="cuda")))


@pytest.mark.parametrize("dtype", WRONG)
def test_the_sequence_error_array_is_of_32_bit_integers(gpu_lib, dtype):
    step, st, args = _case()
    out = gpu_lib.step(*args, *_ring(st), st.sl_max)
    verdict = gpu_lib.verify(*args)
    bad = torch.zeros(out["seq_err"].numel(), dtype=dtype, device="cuda")
    text = "seq_err must be torch.int32, got " + str(dtype)
    with pytest.raises(gpu_lib.DsdeError, match=text):
        gpu_lib.step(*args, *_ring(st), st.sl_max, out=dict(out, seq_err=bad))
    with pytest.raises(gpu_lib.DsdeError, match=text):
        gpu_lib.verify(*args, out=dict(verdict, seq_err=bad))
    state = gpu_lib.new_calibration_state(len(bad))
    with pytest.raises(gpu_lib.DsdeError, match=text):
        gpu_lib.calibration_update(args[2], args[3], verdict["accepted"], verdict["kld"], bad, state)


@pytest.mark.parametrize("call", ["distill_grad", "distill_step"])
def test_a_gradient_over_saved_logits_is_noticed(gpu_lib, call):
    """distill keeps the logits for its backward; a gradient written over them raises their version, so that the
    backward refuses them."""
    z, ids, t, lse, w = batch()
    x = z.clone().requires_grad_(True)
    loss = gpu_lib.distill(x, ids, t, teacher_lse=lse)
    over = x.detach()  # the same memory and version
    if call == "distill_grad":
        record = gpu_lib.distill_loss(over, ids, t, teacher_lse=lse)["record"]
        gpu_lib.distill_grad(over, ids, t, record, w, grad=over)
    else:
        gpu_lib.distill_step(over, ids, t, w, teacher_lse=lse, grad=over)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


def test_reused_outputs_are_noticed(gpu_lib):
    """The teacher's entries that distill keeps, overwritten by the next call's."""
    z, _, _, _, _ = batch()
    teacher = gpu_lib.top_logits(z, 8)
    x = (z + 1.0).requires_grad_(True)
    loss = gpu_lib.distill(x, teacher["ids"], teacher["values"], teacher["lse"])
    gpu_lib.top_logits(-z, 8, out=teacher)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


def test_every_output_of_the_row_operators_is_a_write(gpu_lib):
    z, ids, t, lse, w = batch()
    T, u = torch.ones(6, device="cuda"), torch.full((6,), 0.5, device="cuda")
    calls = [(lambda o: gpu_lib.sample(z, T, u, kept=True, out=o)), (lambda o: gpu_lib.top_logits(z, 8, out=o)),
             (lambda o: gpu_lib.distill_loss(z, ids, t, teacher_lse=lse, out=o)),
             (lambda o: gpu_lib.distill_step(z, ids, t, w, teacher_lse=lse, out=o))]
    for call in calls:
        out = call(None)
        before = {k: v._version for k, v in out.items()}
        given = {k: v.clone() for k, v in out.items()}
        call(out)
        for k, v in out.items():
            assert v._version > before[k], k
            assert torch.equal(v, given[k]), k
        assert z._version == 0 and ids._version == 0  # inputs are not


def test_inference_tensors_have_no_version(gpu_lib):
    z, ids, t, lse, w = batch()
    want = gpu_lib.distill_step(z, ids, t, w, teacher_lse=lse)
    with torch.inference_mode():
        got = gpu_lib.distill_step(z, ids, t, w, teacher_lse=lse)
    again = gpu_lib.distill_step(z, ids, t, w, teacher_lse=lse, grad=got["grad"], out=dict(got))
    assert torch.equal(again["loss"], want["loss"]) and torch.equal(again["grad"], want["grad"])
