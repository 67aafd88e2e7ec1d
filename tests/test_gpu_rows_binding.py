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
