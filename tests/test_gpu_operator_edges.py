"""GPU parity of the operators at the end of a training step where values stand that must not matter (rows that do not count,
masked classes), where logits are far from 0, and at the precision that include/lp.h states."""
import pytest

from test_gpu_operators import EPS32, EPSB, ce_check, ce_inputs, ce_reference, ce_run, muon_reference, ortho_reference, ortho_run, \
    ortho_tol, rel, scratch_of, spectrum

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


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("kind", ["even", "low rank", "decay"])
@pytest.mark.parametrize("size", [(1, 24, 90), (1, 48, 2000), (1, 64, 576), (1, 200, 700), (2, 256, 512), (1, 512, 256), (1, 520, 520), (1, 257, 1031)], ids=str)
def test_the_update_in_bf16_is_as_exact_as_the_orthogonalisation(size, kind, nesterov):
    """Weights of 0 and a rate of 1: the step is all there is to see.  With y the step before its rounding to bf16, off by d from
    the formula's r, |rn(y) - r| <= |rn(r) - r| + 2 d (see test_few_singular_values_in_bf16_cost_one_rounding).  Smaller side below
    64: d is LP_F32's bound; else the result is off by 3e-3 of its norm at most.  Then weights that the step is not small beside:
    their rounding and the step's error."""
    import torch
    import paper_2112_05387_b200 as lp
    B, rows, cols = size
    small = min(rows, cols)
    gen = torch.Generator("cuda").manual_seed(12)
    if kind == "even":
        g = torch.randn(*size, generator=gen, device="cuda")
    else:
        g = torch.stack([spectrum(kind, rows, cols, seed=i) for i in range(B)])
    g = g.bfloat16()
    m0 = 0.1 * g.float() * torch.rand(B, 1, 1, generator=gen, device="cuda")
    buf, at, nb = scratch_of(lp.lp_orthogonalize_scratch_bytes(lp.LP_BF16, *size))
    for lr, scale, spread in ((1.0, 1.0, 0.0), (0.5, 1.25, 0.05)):
        w0 = (spread * torch.randn(*size, generator=gen, device="cuda")).bfloat16()
        w, m = w0.clone(), m0.clone()
        lp.lp_muon_update(lp.LP_BF16, *size, w, g, m, lr, 0.9, nesterov, 0.1, scale, 5, None, 1e-7, at, nb)
        assert lp.lp_scratch_status(at) == lp.LP_OK
        want, want_m = muon_reference(w0, g, m0, lr, 0.9, nesterov, 0.1, scale)
        step = float((want - (1 - lr * 0.1) * w0.double()).norm())
        rounding = float((want.bfloat16().double() - want).norm())
        # (spectra of a few strong directions: LP_F32's bound of test_spectra_of_gradients)
        d = (ortho_tol("f32") if kind == "even" else 3 * 3.4445 ** 5 * 2.0 ** -22) if small < 64 else 3e-3
        off = float((w.double() - want).norm())
        if spread == 0.0 and small >= 64:
            assert off <= 3e-3 * step
        else:
            assert off <= rounding + 2 * d * step
        assert rel(m, want_m) < 4 * EPS32
    del buf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(64, 512, 1000), (300, 64, 2000)], ids=str)
def test_gradients_side_by_side_see_their_own_call(size, dtype):
    """Both gradients' products of a small loss run beside one another.  Two sets of inputs in turn through one scratch, called
    and replayed, with other work on a second stream: every result has the bits of its set taken alone."""
    import torch
    import paper_2112_05387_b200 as lp
    T, D, V = size
    code = lp.LP_F32 if dtype == "f32" else lp.LP_BF16
    sets = [ce_inputs(T, D, V, dtype, seed=s, ignored=0.1) for s in (0, 1)]
    alone = [ce_run(*s) for s in sets]
    buf, at, n = scratch_of(lp.lp_linear_cross_entropy_scratch_bytes(code, T, D, V, True))
    outs = [[{k: torch.zeros_like(v) for k, v in alone[0].items()} for _ in range(20)] for _ in range(2)]
    st, beside = torch.cuda.Stream(), torch.cuda.Stream()
    a = torch.randn(1024, 1024, device="cuda")

    def calls():
        for i in range(20):
            for s in (0, 1):
                o = outs[s][i]
                lp.lp_linear_cross_entropy(code, T, D, V, *sets[s], 1.0, o["loss"], o["row_loss"], o["dx"], o["dw"], o["dbias"], at, n, st.cuda_stream)

    def check():
        torch.cuda.synchronize()
        assert lp.lp_scratch_status(at, st.cuda_stream) == lp.LP_OK
        for s in (0, 1):
            for o in outs[s]:
                for k in o:
                    assert torch.equal(o[k], alone[s][k]), k
                    o[k].zero_()
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        calls()
    for _ in range(4):
        with torch.cuda.stream(beside):
            for _ in range(20):
                a = a @ a * 1e-3
        calls()
        check()
        with torch.cuda.stream(beside):
            for _ in range(20):
                a = a @ a * 1e-3
        with torch.cuda.stream(st):
            graph.replay()
        check()
    del buf


STATED = [(1, 64, 576), (1, 100, 100), (1, 200, 700), (1, 700, 300), (1, 400, 8192), (2, 256, 512), (1, 512, 2304), (1, 1000, 1000)]


@pytest.mark.parametrize("kind", ["even", "low rank", "spike", "decay", "few", "equal", "identity"])
@pytest.mark.parametrize("size", STATED, ids=str)
def test_the_orthogonalisation_is_as_exact_as_stated(size, kind):
    """The figures of include/lp.h.  LP_BF16: 3e-3 of the norm for the spectra of gradients (without the low parts of the first
    iterates 4.9e-3 and more for those of a few strong directions), 4e-3 for eight directions alone, 5e-3 where all singular values
    are alike, 1.1e-2 for multiples of the identity, where a rounding of A or B to 11 bits is the same for all of them.  LP_F32:
    5e-5."""
    import torch
    B, rows, cols = size
    small = min(rows, cols)
    gen = torch.Generator("cuda").manual_seed(13)
    if kind == "even":
        g = torch.randn(*size, generator=gen, device="cuda")
    elif kind == "equal":
        u, v = [torch.linalg.qr(torch.randn(n, small, generator=gen, device="cuda"))[0] for n in (rows, cols)]
        g = (u @ v.mT).expand(B, rows, cols)
    elif kind == "identity":
        g = torch.eye(rows, cols, device="cuda").expand(B, rows, cols)
    elif kind == "few":
        g = torch.randn(B, rows, 8, generator=gen, device="cuda") @ torch.randn(B, 8, cols, generator=gen, device="cuda")
    else:
        g = torch.stack([spectrum(kind, rows, cols, seed=i) for i in range(B)])
    g = g.contiguous()
    assert rel(ortho_run(g), ortho_reference(g)) < 5e-5
    h = g.bfloat16()
    assert rel(ortho_run(h), ortho_reference(h)) < {"few": 4e-3, "equal": 5e-3, "identity": 1.1e-2}.get(kind, 3e-3)


@pytest.mark.parametrize("n", [345, 392, 427, 500])
def test_identities_that_are_rounded_worst(n):
    """The scalar iteration x <- (a + b x^2 + c x^4) x from 1 / sqrt(n), x^2 and the factor rounded to 11 bits, is off by 1.02e-2 at
    most for n from 64 to 131072, at n = 392 (6.7e-3 from 1000 on)."""
    import torch
    g = torch.eye(n, device="cuda")[None].bfloat16()
    assert rel(ortho_run(g), ortho_reference(g)) < 1.1e-2


@pytest.mark.parametrize("name", ["small_preact_bf16", "wrn28_10", "tiny"])
def test_the_step_is_as_exact_as_stated(name):
    """include/lp.h: O of lp_step_muon is as exact as lp_orthogonalize's, 4e-3 of its norm in LP_BF16 and 5e-5 in LP_F32.  No decay, a rate of 1: the weights
    (fp32) move by the step alone, and are rounded by half a step of fp32 once."""
    import numpy as np
    import torch
    import paper_2112_05387_b200 as lp
    from conftest import small_cfg
    from harness import GpuRun
    from workloads import scaled
    cfg = {"tiny": lambda: scaled("tiny"), "small_preact_bf16": lambda: small_cfg("preact", dtype="bf16", stage_channels=(16, 32)),
           "wrn28_10": lambda: scaled("wrn28_10", N=2)}[name]()
    run = GpuRun(cfg)
    K, f32 = run.net.K, cfg["dtype"] == "f32"
    buf, at, nb = scratch_of(lp.lp_step_muon_scratch_bytes(run.h))
    gen = torch.Generator("cuda").manual_seed(14)
    dt = torch.float32 if f32 else torch.bfloat16
    x = [torch.randn(*run.net.boundary[k], generator=gen, device="cuda").to(dt) for k in range(K)]
    labels = torch.randint(0, cfg["num_classes"], (cfg["N"],), generator=gen, device="cuda", dtype=torch.int32)
    loss = torch.zeros(K, 2, device="cuda")
    lp.lp_modules_fwd_bwd_all(run.h, x, labels, None, 0.7, loss, None)
    before = [lp.lp_get_params(run.h, k).astype(np.float64) for k in range(K)]
    grads = [lp.lp_get_grads(run.h, k).astype(np.float64) for k in range(K)]
    lp.lp_step_muon(run.h, 1.0, 0.0, 0.0, False, 0.0, 0.0, None, at, nb)
    assert lp.lp_last_device_status(run.h) == 0
    worst = 0.0
    for k in range(K):
        after, off = lp.lp_get_params(run.h, k).astype(np.float64), 0
        for pname, kind, shape in run.net.param_layout(k):
            n = int(np.prod(shape))
            if kind == "conv_w":
                g = torch.from_numpy(grads[k][off:off + n].reshape(1, shape[0], n // shape[0]).copy()).cuda()
                o = ortho_reference(g)[0].cpu().numpy().reshape(-1) * max(1.0, shape[0] * shape[0] / n) ** 0.5
                p0 = before[k][off:off + n]
                error = np.linalg.norm(after[off:off + n] - (p0 - o))
                rounding = EPS32 * (np.linalg.norm(p0) + np.linalg.norm(o))
                worst = max(worst, (error - rounding) / np.linalg.norm(o))
            off += n
    assert worst < (5e-5 if f32 else 4e-3)
    del buf


@pytest.mark.parametrize("size", [(1, 699, 16307), (2, 41, 4994), (3, 27, 12087), (3, 1203, 6259), (1, 307, 30), (1, 3553, 274), (4, 731, 300), (16, 1497, 300), (261, 32, 2),
                                  (1001, 640, 20011), (6140, 468, 3), (6599, 198, 4)], ids=str)
def test_gradients_in_fp32_are_as_exact_as_stated(size):
    """Two K blocks an accumulation are 24 steps of the tensor core, each of which cuts the sum off by 2^-25 of it on average: 7.2e-7
    where a term of the first step is all of it (a row's label in dx, a row in dw).  Operands of 22 bits: 2^-22.  Together less
    than 1e-6."""
    T, D, V = size
    x, w, b, labels = ce_inputs(T, D, V, "f32", seed=15)
    got, ref = ce_run(x, w, b, labels), ce_reference(x, w, b, labels)
    for k in ("dx", "dw"):
        assert rel(got[k], ref[k]) < 1e-6, k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(2, 64, 300), (20, 64, 700), (65, 200, 5003), (300, 64, 700), (700, 264, 20011)], ids=str)
@pytest.mark.parametrize("lift", [0.0, 2000.0])
def test_confident_rows_keep_their_small_losses(size, lift, dtype):
    """Rows whose label's logit is the largest by 2 to 20 or so, all logits `lift` higher.  Logits off by e move such a row's loss by
    2 e (1 - p) <= 2 e row_loss, and what is left is the statistics' own error, whatever the logits: the sum of exponentials from
    1 on is off by 2^-24 at most for each term that is added to the largest, 32 in a part of 128 columns (four chains), 2 where
    the chains meet, up to 20 parts a lane and 5 exchanges between lanes, and its logarithm by a few more: 64.  dl: the label's the
    same; the others' a product of probabilities off by 2 e each (LP_BF16: fp16 exponentials and one
    rounding to bf16)."""
    import torch
    T, D, V = size
    f32 = dtype == "f32"
    x, w, b, labels = ce_inputs(T, D, V, dtype, seed=17)
    gen = torch.Generator("cuda").manual_seed(18)
    y = labels.long()
    gap = 2 + 18 * torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
    for _ in range(6):      # along the label's weights until its logit is the largest by `gap`
        l = x.double() @ w.double().T + b.double()
        at = l.gather(1, y[:, None])[:, 0]
        top = l.scatter(1, y[:, None], float("-inf")).amax(1)
        x = (x.double() + ((top + gap - at) / (w.double()[y] ** 2).sum(1))[:, None] * w.double()[y]).to(x.dtype)
    b = (b.double() + lift).to(b.dtype)
    ref, got, alone = ce_reference(x, w, b, labels), ce_run(x, w, b, labels), ce_run(x, w, b, labels, grads=False)
    assert float(ref["row_loss"].median()) < 1e-2
    acc = lambda K: ((48 + K / 256) if f32 else K / 16 + 4) * 2 * EPS32  # noqa: E731  (as in ce_check)
    rep = 3 * 2.0 ** -22 if f32 else 0.0
    e_l = (rep + acc(D)) * ref["mag_l"].amax(1) + 8 * EPS32 * ref["l"].abs().amax(1)
    tol = 2 * e_l * ref["row_loss"] + 64 * EPS32
    for r in (got, alone):
        assert bool(((r["row_loss"].double() - ref["row_loss"]).abs() <= tol).all())
    p1 = ref["d"].abs()
    e_d = 2 * e_l[:, None] * p1 + (4 * 2.0 ** -22 * p1 + 2.0 ** -38 if f32 else (EPSB + 2.0 ** -10) * p1 + 2.0 ** -24)
    e_d = e_d.scatter_add(1, y[:, None], torch.full((T, 1), 64 * EPS32, dtype=torch.float64, device="cuda"))
    aw = ref["w"].abs()
    tol = abs(ref["g"]) * (e_d @ aw + (rep + acc(V)) * (p1 @ aw)) + 2 * (EPS32 if f32 else EPSB) * ref["dx"].abs() + 1e-30
    assert bool(((got["dx"].double() - ref["dx"]).abs() <= tol).all())
