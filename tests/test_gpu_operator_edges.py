"""GPU parity of the operators at the end of a training step where values stand that must not matter (rows that do not count,
masked classes) and where logits are far from 0."""
import pytest

from test_gpu_operators import ce_check, ce_inputs, ce_reference, ce_run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [1e8, -1e12, 1e30, 3.3e38])
@pytest.mark.parametrize("T,D", [(3, 72), (70, 3), (71, 75), (300, 72)], ids=str)
def test_finite_values_in_rows_that_do_not_count_reach_nothing(T, D, value, dtype):
    """Padding may hold any finite number: the bits of a call whose padding is of the counted rows' size, and the formulas."""
    import torch
    V = 501
    x, w, b, labels = ce_inputs(T, D, V, dtype)
    out = torch.zeros(T, dtype=torch.bool, device="cuda")
    out[::3] = True
    out[T - 1] = True
    labels[out] = -100
    clean, clean_alone = ce_run(x, w, b, labels), ce_run(x, w, b, labels, grads=False)
    x[out] = value
    got, alone = ce_run(x, w, b, labels), ce_run(x, w, b, labels, grads=False)
    ce_check(got, ce_reference(x, w, b, labels), dtype, D, V, T)
    for k in got:
        assert torch.equal(got[k], clean[k]), k
    for k in alone:
        assert torch.equal(alone[k], clean_alone[k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(2, 64), (70, 75), (300, 64)], ids=str)
def test_finite_weights_of_masked_classes_reach_nothing(T, D, dtype):
    """Rows of w of classes whose bias is -inf (padding up to a round number of classes): any finite number gives the same bits."""
    import torch
    V = 700
    x, w, b, labels = ce_inputs(T, D, V, dtype)
    labels = labels % 451
    b[451:] = float("-inf")
    clean, clean_alone = ce_run(x, w, b, labels), ce_run(x, w, b, labels, grads=False)
    w[451:] = 1e30
    got, alone = ce_run(x, w, b, labels), ce_run(x, w, b, labels, grads=False)
    for k in got:
        assert torch.equal(got[k], clean[k]), k
    for k in alone:
        assert torch.equal(alone[k], clean_alone[k]), k
    # what is not finite there stays in the sums, as the formula has it
    w[600, 1] = float("nan")
    assert bool(torch.isnan(ce_run(x, w, b, labels)["row_loss"]).all())
    assert bool(torch.isnan(ce_run(x, w, b, labels, grads=False)["row_loss"]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [50, 99, 150, 1000])
@pytest.mark.parametrize("size", [(1, 64, 700), (20, 64, 40), (20, 512, 700), (65, 64, 700), (300, 64, 40), (300, 64, 700), (300, 72, 20011),
                                  (2000, 264, 20011)], ids=str)
def test_masked_classes_beside_low_logits(size, shift, dtype):
    """Whole parts of the classes masked, all others at logits around -shift: probability 0 and gradients of 0 for the masked
    ones, the formulas for the rest.  Sizes of shared K, single tiles and tiles of pairs."""
    import torch
    T, D, V = size
    keep = 8 if V == 40 else V // 4
    x, w, b, labels = ce_inputs(T, D, V, dtype)
    labels = labels % keep
    b -= shift
    b[keep:] = float("-inf")
    ref, got = ce_reference(x, w, b, labels), ce_run(x, w, b, labels)
    ce_check(got, dict(ref, mag_l=ref["mag_l"][:, :keep]), dtype, D, V, T)
    assert not bool(got["dw"][keep:].any()) and not bool(got["dbias"][keep:].any())
    # nothing left: 0 / 0
    b[:] = float("-inf")
    none = ce_run(x, w, b, labels)
    assert bool(torch.isnan(none["row_loss"]).all()) and bool(torch.isnan(none["dx"]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 64, 700), (20, 33, 700), (70, 64, 501), (300, 64, 5003), (700, 264, 20011)], ids=str)
def test_rows_that_do_not_count_beside_infinite_weights(size, dtype):
    """Their rows of dx and their losses are 0, whatever w holds; the counted rows' are NaN, as the formulas have it."""
    import torch
    T, D, V = size
    x, w, b, labels = ce_inputs(T, D, V, dtype)
    out = torch.zeros(T, dtype=torch.bool, device="cuda")
    out[::3] = True
    labels[out] = V
    w[V // 2, 1], w[V // 3, 2] = float("inf"), float("nan")
    got = ce_run(x, w, b, labels)
    assert not bool(got["dx"][out].any()) and not bool(got["row_loss"][out].any())
    assert bool(torch.isnan(got["row_loss"][~out]).all()) and bool(torch.isnan(got["dx"][~out][:, 2]).all())
    labels[:] = -1      # no row counts
    got = ce_run(x, w, b, labels)
    assert not any(bool(got[k].any()) for k in got)
