"""What the operators at the end of a training step refuse, on the host, before anything is launched (the pointers are never
followed), and what their scratch sizes say."""
import ctypes

import pytest

import paper_2112_05387_b200 as lp


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()


BIG = 1 << 44
P = 1 << 20      # an aligned address that nothing follows


def ce(dtype=lp.LP_BF16, T=4, D=8, V=16, x=P, w=P, bias=P, labels=P, loss=P, row_loss=P, dx=P, dw=P, dbias=P, scratch=P, nbytes=BIG):
    vp = ctypes.c_void_p
    return lp.lp_status_string(lp.library().lp_linear_cross_entropy(dtype, T, D, V, vp(x), vp(w), vp(bias), vp(labels), 1.0, vp(loss),
                                                                    vp(row_loss), vp(dx), vp(dw), vp(dbias), vp(scratch), nbytes, None))


def ortho(dtype=lp.LP_BF16, batch=1, rows=4, cols=8, g=P, out=P, steps=5, eps=1e-7, scratch=P, nbytes=BIG):
    vp = ctypes.c_void_p
    return lp.lp_status_string(lp.library().lp_orthogonalize(dtype, batch, rows, cols, vp(g), vp(out), steps, None, eps, vp(scratch), nbytes, None))


def muon(dtype=lp.LP_BF16, batch=1, rows=4, cols=8, w=P, g=P, m=P, steps=5, eps=1e-7, scratch=P, nbytes=BIG):
    vp = ctypes.c_void_p
    return lp.lp_status_string(lp.library().lp_muon_update(dtype, batch, rows, cols, vp(w), vp(g), vp(m), 0.1, 0.9, 1, 0.0, 1.0, steps, None, eps,
                                                           vp(scratch), nbytes, None))


@pytest.mark.parametrize("name", ["x", "w", "labels", "loss", "scratch"])
def test_linear_cross_entropy_needs_its_operands(name):
    assert ce(**{name: None}) == lp.lp_status_string(-1)


@pytest.mark.parametrize("name", ["x", "w", "bias", "labels", "loss", "row_loss", "dx", "dw", "dbias", "scratch"])
def test_linear_cross_entropy_refuses_addresses_off_their_boundary(name):
    assert ce(**{name: P + 8}) == lp.lp_status_string(-4)


@pytest.mark.parametrize("call", [ce, ortho, muon])
def test_types_that_are_none_of_the_library(call):
    assert call(dtype=7) == lp.lp_status_string(-10)


@pytest.mark.parametrize("name,value", [(n, v) for n, top in (("T", 1 << 28), ("D", 1 << 20), ("V", 1 << 24)) for v in (0, -1, top + 1)])
def test_linear_cross_entropy_refuses_sizes_out_of_range(name, value):
    assert ce(**{name: value}) == lp.lp_status_string(-9)
    sizes = dict(T=4, D=8, V=16)
    sizes[name] = value
    assert lp.lp_linear_cross_entropy_scratch_bytes(lp.LP_F32, sizes["T"], sizes["D"], sizes["V"], True) == 0


@pytest.mark.parametrize("call,names", [(ortho, ["g", "out", "scratch"]), (muon, ["w", "g", "m", "scratch"])])
def test_matrices_are_needed_on_their_boundary(call, names):
    for name in names:
        assert call(**{name: None}) == lp.lp_status_string(-1)
        assert call(**{name: P + 4}) == lp.lp_status_string(-4)


@pytest.mark.parametrize("call", [ortho, muon])
@pytest.mark.parametrize("bad", [dict(batch=0), dict(batch=65536), dict(rows=0), dict(cols=-3), dict(steps=0), dict(steps=33), dict(eps=0.0),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(rows=1 << 18, cols=1 << 18), dict(rows=1, cols=(1 << 24) + 1)], ids=str)
def test_matrices_steps_and_eps_out_of_range(call, bad):
    assert call(**bad) == lp.lp_status_string(-9)


def test_scratch_that_is_too_small():
    n = lp.lp_linear_cross_entropy_scratch_bytes(lp.LP_F32, 100, 40, 3000, True)
    assert n > 0 and ce(lp.LP_F32, 100, 40, 3000, nbytes=n - 1) == lp.lp_status_string(-5)
    n = lp.lp_orthogonalize_scratch_bytes(lp.LP_F32, 2, 300, 200)
    assert n > 0 and ortho(lp.LP_F32, 2, 300, 200, nbytes=n - 1) == lp.lp_status_string(-5)
    assert muon(lp.LP_F32, 2, 300, 200, nbytes=n - 1) == lp.lp_status_string(-5)
    assert lp.lp_orthogonalize_scratch_bytes(lp.LP_BF16, 0, 3, 3) == 0 and lp.lp_orthogonalize_scratch_bytes(9, 1, 3, 3) == 0


def test_scratch_is_bounded_where_the_logits_are_not():
    """65536 rows of 128000 classes: 16 GB of bf16 logits; the gradients take 512 MB of exponentials and the fp32 sums of dw."""
    T, D, V = 65536, 1024, 128000
    n = lp.lp_linear_cross_entropy_scratch_bytes(lp.LP_BF16, T, D, V, True)
    assert n < (512 << 20) + V * D * 4 + T * D * 2 + (T // 64 + 64) * V * 4 + (256 << 20)
    assert lp.lp_linear_cross_entropy_scratch_bytes(lp.LP_BF16, T, D, V, False) < (520 << 20)


def test_scratch_of_few_classes_goes_by_the_classes():
    """Beside the packed features and two planes of exponentials: 8 bytes a row and 32 classes, three floats a row, the largest
    magnitudes and the column sums of 64 rows each, every region on 256 bytes."""
    for dtype, planes in ((lp.LP_F32, 2), (lp.LP_BF16, 1)):
        for T, D, V in ((262144, 64, 10), (100000, 8, 1000)):
            ld_v, ld_d, parts = (V + 31) // 32 * 32, (D + 7) // 8 * 8, 4 * ((V + 127) // 128)
            operands = 2 * planes * (T + V) * ld_d
            alone = operands + T * (8 * parts + 12) + (1 << 16)
            assert 0 < lp.lp_linear_cross_entropy_scratch_bytes(dtype, T, D, V, False) <= alone
            with_grads = alone + 2 * planes * T * ld_v + (T // 64 + 4) * V * 4 + V * D * 4
            assert 0 < lp.lp_linear_cross_entropy_scratch_bytes(dtype, T, D, V, True) <= with_grads


@pytest.mark.parametrize("dtype", [lp.LP_F32, lp.LP_BF16])
def test_scratch_of_the_gradients_is_enough_for_the_loss_alone(dtype):
    for T in (1, 4, 5, 300, 70000, 1 << 20):
        for D in (1, 72, 4096):
            for V in (1, 5, 1000, 130000, 1 << 22):
                alone, both = [lp.lp_linear_cross_entropy_scratch_bytes(dtype, T, D, V, grads) for grads in (False, True)]
                assert 0 < alone <= both, (T, D, V)


def test_step_and_status_need_a_handle_and_a_scratch():
    lib = lp.library()
    assert lib.lp_step_muon_scratch_bytes(None) == 0
    assert lp.lp_status_string(lib.lp_step_muon(None, 0.1, 0.1, 0.9, 1, 0.0, 0.0, None, P, BIG, None)) == lp.lp_status_string(-1)
    assert lp.lp_scratch_status(None) == -1 and lp.lp_scratch_status(P + 8) == -4


def test_binding_refuses_tensors_that_do_not_match():
    import torch
    t = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="torch.bfloat16"):      # another type
        lp.lp_orthogonalize(lp.LP_BF16, 1, 4, 8, t, t, 5, None, 1e-7, P, BIG)
    with pytest.raises(ValueError, match="40 contiguous"):       # another size
        lp.lp_orthogonalize(lp.LP_F32, 1, 5, 8, t, t, 5, None, 1e-7, P, BIG)
    with pytest.raises(ValueError, match="contiguous"):          # another order
        lp.lp_orthogonalize(lp.LP_F32, 1, 8, 4, t.T, t.T, 5, None, 1e-7, P, BIG)
    with pytest.raises(ValueError, match="g is on cpu"):         # another device
        lp.lp_orthogonalize(lp.LP_F32, 1, 4, 8, t, t, 5, None, 1e-7, P, BIG)
    with pytest.raises(ValueError, match="labels"):
        lp.lp_linear_cross_entropy(lp.LP_F32, 4, 8, 16, None, None, None, torch.zeros(4, dtype=torch.int64), 1.0, None, None, None, None,
                                   None, P, BIG)
