"""GPU parity of the operators at the end of a training step (linear layer + softmax cross entropy over many classes,
orthogonalisation, the update with it) against plain statements in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

COEFFS = (3.4445, -4.7750, 2.0315)
EPS16, EPSB, EPS32 = 2.0 ** -11, 2.0 ** -8, 2.0 ** -24   # half a step of fp16, bf16, fp32, relative to the value


def scratch_of(nbytes):
    import torch
    buf = torch.full((nbytes + 256,), 0xFF, dtype=torch.uint8, device="cuda")   # (0xFFFF is a NaN in every type)
    return buf, (buf.data_ptr() + 255) // 256 * 256, nbytes


# ---------------------------------------------------------------------------------------------
# linear layer + softmax cross entropy
# ---------------------------------------------------------------------------------------------
def ce_inputs(T, D, V, dtype, bias=True, seed=0, ignored=0.0):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.randn(T, D, generator=g, device="cuda").to(dt)
    w = (torch.randn(V, D, generator=g, device="cuda") * 1.5 / D ** 0.5).to(dt)
    b = (torch.randn(V, generator=g, device="cuda") * 0.5).to(dt) if bias else None
    labels = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    if ignored:
        labels[torch.rand(T, generator=g, device="cuda") < ignored] = -100
    return x, w, b, labels


def ce_run(x, w, b, labels, grads=True, scale=1.0, stream=None, want=("dx", "dw", "dbias")):
    import torch
    import paper_2112_05387_b200 as lp
    T, D, V = x.shape[0], x.shape[1], w.shape[0]
    dt = lp.LP_F32 if x.dtype == torch.float32 else lp.LP_BF16
    buf, at, n = scratch_of(lp.lp_linear_cross_entropy_scratch_bytes(dt, T, D, V, grads))
    new = lambda like: torch.full_like(like, 7.0)  # noqa: E731
    got = dict(loss=torch.full((2,), 7.0, device="cuda"), row_loss=torch.full((T,), 7.0, device="cuda"))
    if grads:
        got.update({k: new(v) for k, v in (("dx", x), ("dw", w), ("dbias", b)) if v is not None and k in want})
    lp.lp_linear_cross_entropy(dt, T, D, V, x, w, b, labels, scale, got["loss"], got["row_loss"], got.get("dx"),
                               got.get("dw"), got.get("dbias"), at, n, stream)
    assert lp.lp_scratch_status(at, stream) == lp.LP_OK
    del buf
    return got


def ce_reference(x, w, b, labels, scale=1.0):
    """The formulas in 64 bits, and the sums of magnitudes that the error bounds below go by."""
    import torch
    x, w = x.double(), w.double()
    y = labels.long()
    keep = (y >= 0) & (y < w.shape[0])
    x = torch.where(keep[:, None], x, torch.zeros_like(x))
    l = x @ w.T
    if b is not None:
        l = l + b.double()
    lse = torch.logsumexp(l, 1)
    n = int(keep.sum())
    at = torch.where(keep, y, torch.zeros_like(y))[:, None]
    target = l.gather(1, at)[:, 0]
    row_loss = torch.where(keep, lse - target, torch.zeros_like(lse))
    p = torch.exp(l - lse[:, None])
    d = p.scatter_add(1, at, -torch.ones_like(target)[:, None]) * keep[:, None]
    g = scale / n if n else 0.0
    mag_l = x.abs() @ w.abs().T + (b.double().abs() if b is not None else 0.0)
    return dict(loss=row_loss.sum() / n if n else row_loss.sum(), n=n, row_loss=row_loss, dx=g * (d @ w), dw=g * (d.T @ x),
                dbias=g * d.sum(0), g=g, d=d, p=p * keep[:, None], keep=keep, mag_l=mag_l, x=x, w=w, l=l, lse=lse)


def ce_check(got, ref, dtype, D, V, T):
    """Bounds element by element.
    Logits: operands of LP_F32 are kept to 2^-22 each (two 11-bit parts) and lo * lo is left out: 3 * 2^-22 of the sum of
    magnitudes; bf16 operands are exact.  Accumulation in fp32: at most 2^-23 of the magnitudes for each of the K steps of a
    round (48) and each round, or, without rounds, for each of D / 16 steps (a step inside the tensor core may truncate).
    lse, exp, loss: a few fp32 operations on values of the size of lse.
    dl: 2^-8 (LP_BF16; from fp16 exponentials, 2^-11, absolute 2^-25) or 3 * 2^-22 (LP_F32) of the probability, plus what the
    logits' error makes of it (twice the largest of the row, relative).  Products: as above, over V or T.  Result: one rounding."""
    f32 = dtype == "f32"
    acc = lambda K: ((48 + K / 256) if f32 else K / 16 + 4) * 2 * EPS32  # noqa: E731
    rep = 3 * 2.0 ** -22 if f32 else 0.0
    e_l = (rep + acc(D)) * ref["mag_l"].amax(1) + 8 * EPS32 * (1 + ref["lse"].abs())
    e_l = e_l * ref["keep"]
    err = (got["row_loss"].double() - ref["row_loss"]).abs()
    assert bool((err <= 2 * e_l + 8 * EPS32 * (1 + ref["lse"].abs())).all()), float((err / (2 * e_l + 1e-30)).max())
    assert abs(float(got["loss"][0]) - float(ref["loss"])) <= 2 * float(e_l.max()) + 1e-6 * (1 + abs(float(ref["loss"])))
    assert int(got["loss"][1]) == ref["n"]
    g = abs(ref["g"])
    if f32:
        e_d = (3 * 2.0 ** -22 + 2 * e_l[:, None]) * ref["p"] + 4 * 2.0 ** -22 * ref["d"].abs() + 2.0 ** -38
    else:
        e_d = (EPSB + 2 * EPS16 + 2 * e_l[:, None]) * ref["p"] + (EPSB + 2 * e_l[:, None]) * ref["d"].abs() + 2.0 ** -24
    e_d = e_d * ref["keep"][:, None]
    out = EPS32 if f32 else EPSB
    aw, ax, ad = ref["w"].abs(), ref["x"].abs(), ref["d"].abs()
    worst = {}
    if "dx" in got:
        tol = g * (e_d @ aw + (rep + acc(V)) * (ad @ aw)) + 2 * out * ref["dx"].abs() + 1e-30
        worst["dx"] = float(((got["dx"].double() - ref["dx"]).abs() / tol).max())
    if "dw" in got:
        pieces = 4 * EPS32
        tol = g * (e_d.T @ ax + (rep + acc(T) + pieces) * (ad.T @ ax)) + 2 * out * ref["dw"].abs() + 1e-30
        worst["dw"] = float(((got["dw"].double() - ref["dw"]).abs() / tol).max())
    if "dbias" in got:
        tol = g * (e_d.sum(0) + T * 2 * EPS32 * ad.sum(0)) + 2 * out * ref["dbias"].abs() + 1e-30
        worst["dbias"] = float(((got["dbias"].double() - ref["dbias"]).abs() / tol).max())
    assert all(v <= 1.0 for v in worst.values()), worst
    # and in the norm, where roundings average out: half of the bound of one rounding, or fp32's own level
    for k in worst:
        ref_n = float(ref[k].norm())
        if ref_n > 0:
            rel = float((got[k].double() - ref[k]).norm()) / ref_n
            assert rel < (2e-5 if f32 else 2 * EPSB), (k, rel)


# one row, one feature, two classes; the edges of 32-column groups, 64-wide K blocks, 128 and 256 tiles from both sides; odd
# feature counts (rows off the 16 bytes that a copy needs); more tiles than SMs
CE_SIZES = [(1, 1, 2), (1, 8, 1), (3, 5, 7), (2, 16, 33), (31, 64, 127), (33, 65, 129), (64, 512, 1000), (127, 63, 255),
            (129, 72, 257), (257, 200, 513), (300, 1000, 2049), (1, 640, 20011), (700, 33, 1111), (513, 264, 5003),
            (2, 40, 3001), (3, 130, 777), (4, 2048, 1001), (5, 128, 4000), (2, 30000, 50), (65, 96, 300), (2, 77, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", CE_SIZES, ids=str)
def test_linear_cross_entropy_matches_the_formulas(size, dtype):
    T, D, V = size
    x, w, b, labels = ce_inputs(T, D, V, dtype, bias=V % 2 == 1, ignored=0.2 if T > 2 else 0.0)
    ref = ce_reference(x, w, b, labels, scale=0.5)
    got = ce_run(x, w, b, labels, scale=0.5)
    ce_check(got, ref, dtype, D, V, T)
    alone = ce_run(x, w, b, labels, grads=False)
    ce_check(alone, ref, dtype, D, V, T)


# ---------------------------------------------------------------------------------------------
# orthogonalisation
# ---------------------------------------------------------------------------------------------
def ortho_reference(g, steps=5, coeffs=COEFFS, eps=1e-7):
    import torch
    a, b, c = coeffs
    x = g.double()
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    x = x / torch.clamp(x.flatten(1).norm(dim=1), min=eps)[:, None, None]
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * s @ s) @ x
    return x.mT if tall else x


def ortho_run(g, steps=5, coeffs=None, eps=1e-7, out=None, stream=None):
    import torch
    import paper_2112_05387_b200 as lp
    B, m, n = g.shape
    dt = lp.LP_F32 if g.dtype == torch.float32 else lp.LP_BF16
    buf, at, nb = scratch_of(lp.lp_orthogonalize_scratch_bytes(dt, B, m, n))
    out = torch.full_like(g, 7.0) if out is None else out
    lp.lp_orthogonalize(dt, B, m, n, g, out, steps, coeffs, eps, at, nb, stream)
    assert lp.lp_scratch_status(at, stream) == lp.LP_OK
    del buf
    return out


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


def ortho_tol(dtype, steps=5):
    """Relative to the norm.  An absolute error of X grows by at most a in a step.  LP_BF16: one bf16 rounding of the result,
    fp16 roundings of the last two iterates (the earlier ones keep 22 bits), each of half a step at most, and of B in every step
    (its own rounding touches B X once, relative to |B| |X|).  LP_F32: 22 bits of X, A and B in each step on matrices of even
    spectrum, whose norm grows as an error does."""
    a = COEFFS[0]
    if dtype == "f32":
        return steps * 3 * a * 2.0 ** -21
    return EPSB + EPS16 * (1 + a + a * a)


ORTHO_SIZES = [(1, 1, 1), (3, 1, 5), (3, 7, 1), (2, 16, 27), (5, 16, 144), (18, 64, 576), (2, 33, 31), (1, 127, 129), (1, 128, 128),
               (2, 129, 257), (1, 257, 129), (3, 320, 64), (1, 640, 5760), (1, 2048, 512), (70, 24, 40), (1, 1000, 1003),
               (2, 128, 1152), (1, 5000, 7), (1, 2, 6000000), (1, 1500000, 3), (200, 64, 64), (1, 100, 40000), (3, 1152, 127), (1, 17, 33), (2, 3, 3000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", ORTHO_SIZES, ids=str)
def test_orthogonalize_matches_the_formulas(size, dtype):
    import torch
    g = torch.randn(*size, generator=torch.Generator("cuda").manual_seed(1), device="cuda") * 1e-3
    g = g.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    out = ortho_run(g)
    ref = ortho_reference(g)
    for b in range(size[0]):
        assert rel(out[b], ref[b]) < ortho_tol(dtype), b


# ---------------------------------------------------------------------------------------------
# linear layer + softmax cross entropy: where it can go wrong
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 48])
def test_rows_in_pieces_equal_the_formulas(D, dtype):
    """More exponentials than a piece may keep, and more than the sums of dw would take: three pieces (fp32), two (bf16).  Rows
    of dw of 16 bytes, and of whole sectors."""
    T, V = 3000, 100000
    x, w, b, labels = ce_inputs(T, D, V, dtype, ignored=0.1)
    ref = ce_reference(x, w, b, labels)
    got = ce_run(x, w, b, labels)
    ce_check(got, ref, dtype, D, V, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 3, 70, 300])
def test_rows_that_do_not_count_reach_nothing(dtype, T):
    """Labels below 0 or past the last class; such a row of x holds NaN and infinities."""
    import torch
    D, V = 72, 501
    x, w, b, labels = ce_inputs(T, D, V, dtype)
    out = torch.zeros(T, dtype=torch.bool, device="cuda")
    out[::3] = True
    labels[out] = torch.tensor([-100, -1, V, 2 ** 31 - 1, -2 ** 31], device="cuda", dtype=torch.int32).repeat(T)[:int(out.sum())]
    clean = ce_run(x, w, b, labels)
    ref = ce_reference(x, w, b, labels)
    if T > 1:
        ce_check(clean, ref, dtype, D, V, T)
    x[out] = float("nan")
    x[out, 0] = float("inf")
    got = ce_run(x, w, b, labels)
    for k in got:
        assert torch.equal(got[k], clean[k]), k
    assert bool((got["row_loss"][out] == 0).all()) and bool((got["dx"][out] == 0).all())
    alone = ce_run(x, w, b, labels, grads=False)
    assert bool((alone["row_loss"][out] == 0).all()) and float(alone["loss"][1]) == T - int(out.sum())
    if T == 1:   # no row counts: the loss and the gradients are zeros
        assert float(got["loss"][0]) == 0 and float(alone["loss"][0]) == 0
        assert all(not bool(got[k].any()) for k in ("dx", "dw", "dbias"))


@pytest.mark.parametrize("T", [20, 300])
def test_long_sums_are_added_up_in_fp32(T):
    """20000 features: 1250 steps of the tensor cores, each of which cuts the sum off (2^-24 of it at most, half of that on
    average and always towards zero).  Rounds of 256 steps are added up apart: 2^-25 * 256 = 7.6e-6 of a logit at most, and half
    of that where the sum grows evenly; the loss is a difference of logits of its own size."""
    D, V = 20000, 300
    x, w, b, labels = ce_inputs(T, D, V, "bf16")
    ref = ce_reference(x, w, b, labels)
    got = ce_run(x, w, b, labels)
    ce_check(got, ref, "bf16", D, V, T)
    err = (got["row_loss"].double() - ref["row_loss"]).abs()
    assert bool((err <= 2.0 ** -25 * 256 * 2 * ref["l"].abs().amax(1) + 8 * EPS32 * (1 + ref["lse"].abs())).all())


@pytest.mark.parametrize("T", [2, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_classes_and_extreme_logits(dtype, T):
    import torch
    D, V = 64, 700
    x, w, b, labels = ce_inputs(T, D, V, dtype)
    labels = labels % 100
    # most classes masked, whole tiles among them: probability 0, no gradient
    b[100:] = float("-inf")
    ref, got = ce_reference(x, w, b, labels), ce_run(x, w, b, labels)
    ref = dict(ref, mag_l=ref["mag_l"][:, :100])
    ce_check(got, ref, dtype, D, V, T)
    assert not bool(got["dw"][100:].any()) and not bool(got["dbias"][100:].any())
    # the type's lowest value: the same
    low = b.clone()
    low[100:] = torch.finfo(b.dtype).min
    again = ce_run(x, w, low, labels)
    for k in got:
        assert torch.equal(got[k], again[k]), k
    # the label's class masked in one row: an infinite loss there and in the mean, the other rows as they were
    labels[0] = 500
    got = ce_run(x, w, b, labels)
    assert float(got["row_loss"][0]) == float("inf") and float(got["loss"][0]) == float("inf")
    assert bool(torch.isfinite(got["row_loss"][1:]).all()) and bool(torch.isfinite(got["dx"]).all())
    alone = ce_run(x, w, b, labels, grads=False)
    assert float(alone["row_loss"][0]) == float("inf") and bool(torch.isfinite(alone["row_loss"][1:]).all())
    # nothing left of any row: NaN, as 0 / 0 is
    b[:] = float("-inf")
    assert bool(torch.isnan(ce_run(x, w, b, labels)["row_loss"]).all())
    assert bool(torch.isnan(ce_run(x, w, b, labels, grads=False)["row_loss"]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_and_large_features(dtype):
    """An infinity in a counted row: that row's loss is NaN (inf - inf), no other row's is.  Logits of some thousands."""
    import torch
    T, D, V = 40, 64, 700
    for grads in (True, False):
        for rows in (T, 2):
            x, w, b, labels = (t[:rows] if i in (0, 3) else t for i, t in enumerate(ce_inputs(T, D, V, dtype)))
            x, labels = x.clone(), labels.clone()
            x[1, 3] = float("inf")
            got = ce_run(x, w, b, labels, grads=grads)
            assert bool(torch.isnan(got["row_loss"][1])) and bool(torch.isnan(got["loss"][0]))
            assert bool(torch.isfinite(got["row_loss"][torch.arange(rows) != 1]).all())
    x, w, b, labels = ce_inputs(T, D, V, dtype)
    x = x * 1000
    ref, got = ce_reference(x, w, b, labels), ce_run(x, w, b, labels)
    ce_check(got, ref, dtype, D, V, T)


def test_classes_past_two_to_the_31_elements():
    """The last rows of a w of more than 2^31 elements, through the loss and all gradients."""
    import torch
    T, D, V = 300, 4096, 540000
    g = torch.Generator("cuda").manual_seed(0)
    x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    w = torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    keep = torch.tensor([0, 1, 262143, 524287, 524288, 524289, V - 2, V - 1], device="cuda")
    w[keep] = (torch.randn(8, D, generator=g, device="cuda") / D ** 0.5).bfloat16()
    labels = keep[torch.randint(0, 8, (T,), generator=g, device="cuda")].int()
    got = ce_run(x, w, None, labels)
    # all other classes have logit 0: V - 8 of them, of one probability
    l = x.double() @ w[keep].double().T
    lse = torch.logsumexp(torch.cat([l, torch.full((T, 1), float(np.log(V - 8)), dtype=torch.float64, device="cuda")], 1), 1)
    p = torch.exp(l - lse[:, None])
    d = p - (labels[:, None] == keep[None, :]).double()
    target = (l * (labels[:, None] == keep[None, :])).sum(1)
    assert float((got["row_loss"].double() - (lse - target)).abs().max()) < 2e-5 * 13
    assert rel(got["dw"][keep], (d.T @ x.double()) / T) < 2 * EPSB
    other = torch.exp(-lse)[None, :] @ x.double() / T
    assert rel(got["dw"][V - 5:V - 2], other.expand(3, D)) < 2 * EPSB + 1e-2      # (a small sum: fp16 steps of its terms, 2^-25 each)
    assert rel(got["dx"], (d @ w[keep].double()) / T) < 2 * EPSB


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_gradients_equal_those_taken_together(dtype):
    import torch
    x, w, b, labels = ce_inputs(130, 96, 1500, dtype, ignored=0.2)
    whole = ce_run(x, w, b, labels)
    for k in ("dx", "dw", "dbias"):
        got = ce_run(x, w, b, labels, want=(k,))
        assert sorted(got) == sorted(["loss", "row_loss", k])
        for name in got:
            assert torch.equal(got[name], whole[name]), name


def test_gradients_are_the_differences_of_the_loss():
    """fp32: central differences of the loss along random directions.  Truncation h^2 / 6 times a third derivative of order 1 and
    the loss's own error (2e-7 of it) over h."""
    import torch
    T, D, V = 50, 40, 300
    x, w, b, labels = ce_inputs(T, D, V, "f32", ignored=0.2)
    got = ce_run(x, w, b, labels, scale=1.0)
    gen = torch.Generator("cuda").manual_seed(3)
    h = 1e-2
    for name, t in (("dx", x), ("dw", w), ("dbias", b)):
        u = torch.randn(t.shape, generator=gen, device="cuda")
        u /= u.norm()
        args = {"dx": x, "dw": w, "dbias": b}

        def loss(sign):
            a = dict(args)
            a[name] = t + sign * h * u
            return float(ce_run(a["dx"], a["dw"], a["dbias"], labels, grads=False)["loss"][0])
        d = (loss(1) - loss(-1)) / (2 * h)
        assert abs(d - float((got[name] * u).sum())) < h * h + 6 * 2e-7 / h, name


# ---------------------------------------------------------------------------------------------
# orthogonalisation: where it can go wrong
# ---------------------------------------------------------------------------------------------
def spectrum(kind, m, n, seed=0):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    if kind == "low rank":
        return torch.randn(m, 8, generator=g, device="cuda") @ torch.randn(8, n, generator=g, device="cuda") + \
            0.1 * torch.randn(m, n, generator=g, device="cuda")
    if kind == "spike":
        return torch.randn(m, 1, generator=g, device="cuda") @ torch.randn(1, n, generator=g, device="cuda") + \
            0.01 * torch.randn(m, n, generator=g, device="cuda")
    k = min(m, n)
    u, _ = torch.linalg.qr(torch.randn(m, k, generator=g, device="cuda"))
    v, _ = torch.linalg.qr(torch.randn(n, k, generator=g, device="cuda"))
    return u @ torch.diag(torch.logspace(0, -3, k, device="cuda")) @ v.mT


@pytest.mark.parametrize("kind", ["low rank", "spike", "decay"])
@pytest.mark.parametrize("size", [(48, 300), (300, 48), (200, 700), (520, 520)], ids=str)
def test_spectra_of_gradients(kind, size):
    """Weak directions are brought up by a^5 = 485, and an error with them.  LP_F32: two steps' errors of 2^-21 of the strong
    directions in full, 3 a^5 2^-21 / 2 at most where all energy was in one of them.  LP_BF16: bf16 and fp16 roundings as for an
    even spectrum, and the first iterates' 22 bits."""
    import torch
    g = spectrum(kind, *size)[None]
    out, ref = ortho_run(g), ortho_reference(g)
    assert rel(out, ref) < 3 * COEFFS[0] ** 5 * 2.0 ** -22
    h = g.bfloat16()
    assert rel(ortho_run(h), ortho_reference(h)) < ortho_tol("bf16")
    # what the operator is for: singular values near 1 (in [0.5, 1.3] for those above 1 / 100 of the norm)
    s, s0 = torch.linalg.svdvals(out[0].double()), torch.linalg.svdvals(g[0].double())
    strong = s0 / s0.norm() > 1e-2
    assert float(s.max()) < 1.3 and int((s > 0.5).sum()) >= int(strong.sum())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(20, 50), (90, 300), (300, 170)], ids=str)
def test_matrices_of_a_batch_do_not_touch_one_another(dtype, size):
    """A matrix of zeros stays one, one with a NaN or an infinity becomes NaN, and the others have the same bits as without."""
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.randn(5, *size, generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(dt)
    good = ortho_run(g)
    g[1] = 0
    g[2, 3, 4] = float("nan")
    g[3, 1, 1] = float("-inf")
    out = ortho_run(g)
    assert torch.equal(out[0], good[0]) and torch.equal(out[4], good[4])
    assert not bool(out[1].any())
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(out[3]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 24, 40), (1, 200, 330), (2, 330, 200)], ids=str)
def test_scale_steps_coefficients_and_place(dtype, size):
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.randn(*size, generator=torch.Generator("cuda").manual_seed(4), device="cuda").to(dt)
    base = ortho_run(g)
    for k in (-100, -12, 40, 100):          # (powers of two: the same matrix to the bit, whatever the exponent)
        assert torch.equal(ortho_run((g.double() * 2.0 ** k).to(dt), eps=1e-30), base), k
    # a norm below eps is not brought up to 1
    tiny = (g.double() * 1e-4 / g.double().flatten(1).norm(dim=1).max()).to(dt)
    assert rel(ortho_run(tiny, eps=1e-3), ortho_reference(tiny, eps=1e-3)) < ortho_tol(dtype)
    for steps, coeffs in ((1, None), (2, None), (7, (1.875, -1.25, 0.375)), (3, (1.5, -0.5, 0.0))):
        out = ortho_run(g, steps=steps, coeffs=coeffs)
        assert rel(out, ortho_reference(g, steps, coeffs or COEFFS)) < ortho_tol(dtype, max(steps, 5)), (steps, coeffs)
    place = g.clone()
    ortho_run(place, out=place)
    assert torch.equal(place, base)


def test_a_batch_past_two_to_the_31_elements():
    import torch
    B, n = 34, 8192
    g = torch.zeros(B, n, n, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator("cuda").manual_seed(5)
    for b in (0, 31, 32, B - 1):
        g[b] = torch.randn(n, n, generator=gen, device="cuda").bfloat16()
    out = ortho_run(g, steps=2, out=g.clone())
    assert not bool(out[30].any())
    for b in (0, 31, 32, B - 1):
        assert rel(out[b], ortho_reference(g[b:b + 1], 2)[0]) < ortho_tol("bf16"), b


# ---------------------------------------------------------------------------------------------
# the update
# ---------------------------------------------------------------------------------------------
def muon_reference(w, g, m, lr, mu, nesterov, wd, scale):
    w, g, m = w.double(), g.double(), m.double()
    m = mu * m + g
    u = g + mu * m if nesterov else m
    return (1 - lr * wd) * w - lr * scale * ortho_reference(u), m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("size", [(1, 16, 144), (3, 33, 65), (1, 130, 1000), (2, 513, 129), (1, 257, 1031)], ids=str)
def test_update_matches_the_formulas(size, nesterov, dtype):
    """Three updates in a row.  A step moves the weights by lr * scale * |O|; O is off by ortho_tol of its norm (LP_BF16: without
    low parts, of all five iterates: 2^-11 (a + a^2 + ... + a^4) more); the weights are rounded once a step."""
    import torch
    import paper_2112_05387_b200 as lp
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    code = lp.LP_F32 if dtype == "f32" else lp.LP_BF16
    lr, mu, wd, scale = 0.05, 0.9, 0.1, 1.25
    gen = torch.Generator("cuda").manual_seed(6)
    w = torch.randn(*size, generator=gen, device="cuda").to(dt)
    m = torch.randn(*size, generator=gen, device="cuda") * 1e-3
    buf, at, nb = scratch_of(lp.lp_orthogonalize_scratch_bytes(code, *size))
    for _ in range(3):
        g = (torch.randn(*size, generator=gen, device="cuda") * 1e-3).to(dt)
        want_w, want_m = muon_reference(w, g, m, lr, mu, nesterov, wd, scale)
        lp.lp_muon_update(code, *size, w, g, m, lr, mu, nesterov, wd, scale, 5, None, 1e-7, at, nb)
        assert lp.lp_scratch_status(at) == lp.LP_OK
        assert rel(m, want_m) < 4 * EPS32
        o = ortho_tol(dtype) + (0 if dtype == "f32" else EPS16 * sum(COEFFS[0] ** k for k in range(1, 5)))
        off = float((w.double() - want_w).norm())
        rounding = (EPS32 * 4 if dtype == "f32" else EPSB) * float(want_w.norm())
        assert off < rounding + lr * scale * o * float(ortho_reference(want_m).norm())
    del buf


def step_state(lp, run):
    K = run.net.K
    return [lp.lp_get_params(run.h, k).astype(np.float64) for k in range(K)], [lp.lp_get_grads(run.h, k).astype(np.float64) for k in range(K)]


@pytest.mark.parametrize("name", ["tiny", "small_preact_bf16", "resnet56", "wrn28_10"])
def test_step_with_orthogonalised_updates_of_a_network(name):
    """lp_step_muon on the gradients of a network's passes: convolution weights by the formulas, the rest by SGD, multipliers as
    in lp_step; the next pass sees the new weights (a handle that is given them computes the same).  Four updates: the later
    ones are graph launches."""
    import torch
    import paper_2112_05387_b200 as lp
    from conftest import small_cfg
    from harness import GpuRun
    from workloads import scaled
    cfg = {"tiny": lambda: scaled("tiny"), "small_preact_bf16": lambda: small_cfg("preact", dtype="bf16", stage_channels=(16, 32)),
           "resnet56": lambda: scaled("resnet56", N=4), "wrn28_10": lambda: scaled("wrn28_10", N=2)}[name]()
    run = GpuRun(cfg)
    K, f32 = run.net.K, cfg["dtype"] == "f32"
    nb = lp.lp_step_muon_scratch_bytes(run.h)
    assert nb > 0
    buf, at, nb = scratch_of(nb)
    lr_conv, lr, mu, wd, c = 0.02, 0.01, 0.9, 5e-4, 0.3
    dt = torch.float32 if f32 else torch.bfloat16
    mom = None
    gen = torch.Generator("cuda").manual_seed(7)
    shapes = [tuple(run.net.boundary[k]) for k in range(K)] + [None]
    x = [torch.randn(*run.net.boundary[k], generator=gen, device="cuda").to(dt) for k in range(K)]
    labels = torch.randint(0, cfg["num_classes"], (cfg["N"],), generator=gen, device="cuda", dtype=torch.int32)
    kap = [torch.randn(*shapes[k + 1], generator=gen, device="cuda").mul_(0.1).to(dt) for k in range(K - 1)]
    loss = torch.zeros(K, 2, device="cuda")
    with pytest.raises(lp.LpError):
        lp.lp_step_muon(run.h, lr_conv, lr, mu, True, wd, c, None, at, nb)      # no gradients yet
    for it in range(4):
        lp.lp_modules_fwd_bwd_all(run.h, x, labels, kap, 0.7, loss, None)
        assert lp.lp_last_device_status(run.h) == 0
        before, grads = step_state(lp, run)
        kap0 = [t.double() for t in kap]
        r = [torch.empty_like(t) for t in kap]
        for k in range(K - 1):
            lp.lp_get_residual(run.h, k, r[k], None)
        lp.lp_step_muon(run.h, lr_conv, lr, mu, it % 2 == 0, wd, c, kap, at, nb)
        assert lp.lp_last_device_status(run.h) == 0
        after, _ = step_state(lp, run)
        mom = mom or [np.zeros_like(p) for p in before]
        for k in range(K):
            off = 0
            for pname, kind, shape in run.net.param_layout(k):
                n = int(np.prod(shape))
                p0, g, m, p1 = before[k][off:off + n], grads[k][off:off + n], mom[k][off:off + n], after[k][off:off + n]
                if kind == "conv_w":
                    rows = shape[0]
                    mat = lambda a: torch.from_numpy(a.reshape(1, rows, n // rows).copy()).cuda()  # noqa: E731
                    want, wm = muon_reference(mat(p0), mat(g), mat(m), lr_conv, mu, it % 2 == 0, wd, max(1.0, rows * rows / n) ** 0.5)
                    m[:] = wm.cpu().numpy().reshape(-1)
                    step = np.linalg.norm(want.cpu().numpy().reshape(-1) - p0)
                    # fp32 networks: gradients of 64 x 9 elements and more of uneven spectrum, see test_spectra_of_gradients
                    tol = (3 * COEFFS[0] ** 5 * 2.0 ** -22 if f32 else 3e-2) * step + 8 * EPS32 * np.linalg.norm(p0)
                    assert np.linalg.norm(p1 - want.cpu().numpy().reshape(-1)) < tol, (it, k, pname)
                else:
                    m[:] = mu * m + g + wd * p0
                    assert np.linalg.norm(p1 - (p0 - lr * m)) < 1e-6 * (np.linalg.norm(p0) + lr * np.linalg.norm(m)), (it, k, pname)
                off += n
        for k in range(K - 1):
            want = kap0[k] + c * r[k].double()
            assert rel(kap[k], want) < (1e-6 if f32 else 2 * EPSB)
        if it in (0, 3):   # the operand copies are those of the new weights
            other = GpuRun(cfg)
            for k in range(K):
                lp.lp_set_params(other.h, k, after[k].astype(np.float32))
            la, lb = torch.zeros(K, 2, device="cuda"), torch.zeros(K, 2, device="cuda")
            lp.lp_modules_fwd_bwd_all(run.h, x, labels, kap, 0.7, la, None)
            lp.lp_modules_fwd_bwd_all(other.h, x, labels, kap, 0.7, lb, None)
            assert lp.lp_last_device_status(run.h) == 0 and lp.lp_last_device_status(other.h) == 0
            assert float((la - lb).abs().max()) <= 1e-4 * float(lb.abs().max())
    launched, _, direct = lp.lp_call_graphs(run.h)
    assert launched >= 2


# ---------------------------------------------------------------------------------------------
# streams, recordings, the same bits
# ---------------------------------------------------------------------------------------------
def test_the_same_bits_again_on_another_stream_and_in_recordings():
    """Two recordings with a scratch each, replayed on streams of their own at the same time, eager calls between them."""
    import torch
    import paper_2112_05387_b200 as lp
    x, w, b, labels = ce_inputs(300, 128, 5000, "bf16", ignored=0.2)
    eager = ce_run(x, w, b, labels)
    g = torch.randn(2, 200, 300, device="cuda").bfloat16()
    small = torch.randn(3, 40, 90, device="cuda")
    want, want_small = ortho_run(g), ortho_run(small)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ce_run(x, w, b, labels, stream=side.cuda_stream)
    assert all(torch.equal(got[k], eager[k]) for k in eager)
    held, replays = [], []
    for _ in range(2):
        outs = {k: torch.zeros_like(v) for k, v in eager.items()}
        o, os = torch.zeros_like(g), torch.zeros_like(small)
        nbs = [lp.lp_linear_cross_entropy_scratch_bytes(lp.LP_BF16, 300, 128, 5000, True), lp.lp_orthogonalize_scratch_bytes(lp.LP_BF16, 2, 200, 300),
               lp.lp_orthogonalize_scratch_bytes(lp.LP_F32, 3, 40, 90)]
        bufs = [scratch_of(n) for n in nbs]
        graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=st):
            s = st.cuda_stream
            lp.lp_linear_cross_entropy(lp.LP_BF16, 300, 128, 5000, x, w, b, labels, 1.0, outs["loss"], outs["row_loss"], outs["dx"], outs["dw"],
                                       outs["dbias"], bufs[0][1], bufs[0][2], s)
            lp.lp_orthogonalize(lp.LP_BF16, 2, 200, 300, g, o, 5, None, 1e-7, bufs[1][1], bufs[1][2], s)
            lp.lp_orthogonalize(lp.LP_F32, 3, 40, 90, small, os, 5, None, 1e-7, bufs[2][1], bufs[2][2], s)
        held.append((bufs, graph))
        replays.append((graph, torch.cuda.Stream(), outs, o, os))
    for _ in range(3):
        for graph, st, outs, o, os in replays:
            for t in list(outs.values()) + [o, os]:
                t.fill_(7)
        torch.cuda.synchronize()
        for graph, st, *_ in replays:
            with torch.cuda.stream(st):
                graph.replay()
        again = ce_run(x, w, b, labels)
        torch.cuda.synchronize()
        assert all(torch.equal(again[k], eager[k]) for k in eager)
        for _, _, outs, o, os in replays:
            assert all(torch.equal(outs[k], eager[k]) for k in eager)
            assert torch.equal(o, want) and torch.equal(os, want_small)
    del held


def test_nothing_is_written_outside_the_results():
    """Guards around every output and the scratch; odd sizes."""
    import torch
    import paper_2112_05387_b200 as lp
    for dtype, dt in ((lp.LP_F32, torch.float32), (lp.LP_BF16, torch.bfloat16)):
        T, D, V = 133, 75, 1003

        def guarded(n, t=dt):
            whole = torch.full((n + 128,), 3.0, dtype=t, device="cuda")
            return whole, whole[64:64 + n]
        x, w, b, labels = ce_inputs(T, D, V, "f32" if dtype == lp.LP_F32 else "bf16")
        outs = [guarded(2, torch.float32), guarded(T, torch.float32), guarded(T * D), guarded(V * D), guarded(V)]
        nb = lp.lp_linear_cross_entropy_scratch_bytes(dtype, T, D, V, True)
        s = torch.full((nb + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
        at = (s.data_ptr() + 255) // 256 * 256
        lp.lp_linear_cross_entropy(dtype, T, D, V, x, w, b, labels, 1.0, *[o[1] for o in outs], at, nb)
        for rows, cols in ((33, 77), (141, 203), (203, 141)):
            g = torch.randn(2, rows, cols, device="cuda").to(dt)
            o = guarded(g.numel())
            nbo = lp.lp_orthogonalize_scratch_bytes(dtype, 2, rows, cols)
            so = torch.full((nbo + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
            ao = (so.data_ptr() + 255) // 256 * 256
            lp.lp_orthogonalize(dtype, 2, rows, cols, g, o[1], 5, None, 1e-7, ao, nbo)
            outs.append(o)
            end = ao - so.data_ptr() + nbo
            assert bool((so[end:] == 0x5A).all()) and bool((so[:ao - so.data_ptr()] == 0x5A).all())
        end = at - s.data_ptr() + nb
        assert bool((s[end:] == 0x5A).all())
        for whole, part in outs:
            assert bool((whole[:64] == 3).all()) and bool((whole[-64:] == 3).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tensors_on_16_byte_boundaries(dtype):
    """Every tensor 16 bytes past a 256-byte boundary (whole sectors are 32): the same bits as on the boundary."""
    import torch
    off = 4 if dtype == "f32" else 8

    def moved(t, n):
        whole = torch.zeros(t.numel() + 64, dtype=t.dtype, device="cuda")
        part = whole[n:n + t.numel()].view(t.shape)
        part.copy_(t)
        return part
    x, w, b, labels = ce_inputs(200, 96, 1504, dtype, ignored=0.1)
    want = ce_run(x, w, b, labels)
    import paper_2112_05387_b200 as lp
    code = lp.LP_F32 if dtype == "f32" else lp.LP_BF16
    buf, at, n = scratch_of(lp.lp_linear_cross_entropy_scratch_bytes(code, 200, 96, 1504, True))
    got = {k: moved(torch.zeros_like(v), 4 if v.dtype == torch.float32 else 8) for k, v in want.items()}
    lp.lp_linear_cross_entropy(code, 200, 96, 1504, moved(x, off), moved(w, off), moved(b, off), moved(labels, 4), 1.0, got["loss"], got["row_loss"],
                               got["dx"], got["dw"], got["dbias"], at, n)
    assert lp.lp_scratch_status(at) == lp.LP_OK
    assert all(torch.equal(got[k], want[k]) for k in want)
    for size in ((2, 40, 96), (2, 160, 288), (1, 288, 160)):
        g = torch.randn(*size, device="cuda").to(x.dtype)
        assert torch.equal(ortho_run(moved(g, off), out=moved(torch.zeros_like(g), off)), ortho_run(g)), size
    del buf


def test_the_step_recorded_and_replayed_equals_the_calls():
    """Passes and lp_step_muon in a recording of the handle, launched twice, against a handle that makes the calls."""
    import torch
    import paper_2112_05387_b200 as lp
    from conftest import small_cfg
    from harness import GpuRun
    cfg = small_cfg("postbn", dtype="f32", stage_channels=(16, 32))
    runs = [GpuRun(cfg) for _ in range(2)]
    gen = torch.Generator("cuda").manual_seed(9)
    K = runs[0].net.K
    x = [torch.randn(*runs[0].net.boundary[k], generator=gen, device="cuda") for k in range(K)]
    labels = torch.randint(0, cfg["num_classes"], (cfg["N"],), generator=gen, device="cuda", dtype=torch.int32)
    st = torch.cuda.Stream()
    s = st.cuda_stream
    state = []
    for r, run in enumerate(runs):
        buf, at, nb = scratch_of(lp.lp_step_muon_scratch_bytes(run.h))
        loss = torch.zeros(K, 2, device="cuda")
        torch.cuda.synchronize()

        def step():
            lp.lp_modules_fwd_bwd_all(run.h, x, labels, None, 0.7, loss, None, s)
            lp.lp_step_muon(run.h, 0.02, 0.01, 0.9, True, 1e-3, 0.0, None, at, nb, s)
        step()
        if r == 0:
            lp.lp_graph_begin(run.h, s)
            step()
            gid = lp.lp_graph_end(run.h, s)
            for _ in range(2):
                lp.lp_graph_launch(run.h, gid, s)
        else:
            for _ in range(2):
                step()
        assert lp.lp_last_device_status(run.h, s) == 0
        state.append([lp.lp_get_params(run.h, k) for k in range(K)])
        del buf
    for a, b in zip(*state):
        assert np.linalg.norm(a - b) < 1e-5 * np.linalg.norm(b)     # (gradients of convolutions are added up by atomics)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_gradients_of_rows_in_pieces(dtype):
    """Odd rows of dw and dx over several pieces, each gradient asked for by itself: the formulas, and the same bits."""
    import torch
    T, D, V = 3000, 33, 100001
    x, w, b, labels = ce_inputs(T, D, V, dtype, ignored=0.1, seed=5)
    got = ce_run(x, w, b, labels, scale=3.0)
    ce_check(got, ce_reference(x, w, b, labels, scale=3.0), dtype, D, V, T)
    for want in ("dx", "dw", "dbias"):
        one = ce_run(x, w, b, labels, scale=3.0, want=(want,))
        assert set(one) == {"loss", "row_loss", want} and all(torch.equal(one[k], got[k]) for k in one), want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(2, 40, 90), (1, 200, 330), (1, 600, 900)], ids=str)
def test_the_update_recorded_and_replayed_equals_the_calls(size, dtype):
    """One launch, shared K, and tiles of CTA pairs; a replay sees the weights and the momentum that the one before left."""
    import torch
    import paper_2112_05387_b200 as lp
    code, dt = (lp.LP_F32, torch.float32) if dtype == "f32" else (lp.LP_BF16, torch.bfloat16)
    gen = torch.Generator("cuda").manual_seed(11)
    g, w0 = [torch.randn(*size, generator=gen, device="cuda").to(dt) for _ in range(2)]
    m0 = torch.randn(*size, generator=gen, device="cuda")
    n = lp.lp_orthogonalize_scratch_bytes(code, *size)
    buf, at, n = scratch_of(n)
    state = []
    for recorded in (False, True):
        w, m, st = w0.clone(), m0.clone(), torch.cuda.Stream()
        torch.cuda.synchronize()

        def update():
            lp.lp_muon_update(code, *size, w, g, m, 0.02, 0.9, True, 0.1, 1.5, 5, None, 1e-7, at, n, st.cuda_stream)
        if recorded:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                update()
            with torch.cuda.stream(st):
                for _ in range(3):
                    graph.replay()
        else:
            for _ in range(3):
                update()
        assert lp.lp_scratch_status(at, st.cuda_stream) == lp.LP_OK
        state.append((w, m))
    assert torch.equal(state[0][0], state[1][0]) and torch.equal(state[0][1], state[1][1]) and not torch.equal(state[0][0], w0)
    del buf


@pytest.mark.parametrize("size", [(3, 1, 5), (7, 2, 3), (40, 3, 40), (9, 4, 100), (1, 16, 144), (2, 32, 4000), (1, 1000, 63), (40, 48, 2000)], ids=str)
def test_few_singular_values_in_bf16_cost_one_rounding(size):
    """With y before the rounding off by d from the formula's r: |rn(y) - r| <= |rn(y) - y| + d <= |rn(r) - y| + d <= |rn(r) - r| + 2 d,
    where d is the bound of LP_F32."""
    import torch
    g = torch.randn(*size, generator=torch.Generator("cuda").manual_seed(3), device="cuda").bfloat16()
    out, ref = ortho_run(g).double(), ortho_reference(g)
    assert float((out - ref).norm()) <= float((ref.bfloat16().double() - ref).norm()) + 2 * ortho_tol("f32") * float(ref.norm())


def test_a_head_and_its_layer_trained_together():
    """The operators as a program uses them: features from a hidden layer, the loss of a head over many classes, its gradients,
    orthogonalised updates of both weights.  Every step's gradients are those of the formulas in 64 bits for its weights."""
    import torch
    import paper_2112_05387_b200 as lp
    T, D0, D, V = 96, 48, 64, 1200
    gen = torch.Generator("cuda").manual_seed(8)
    x0 = torch.randn(T, D0, generator=gen, device="cuda")
    labels = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    w0 = torch.randn(D, D0, generator=gen, device="cuda") * 0.2
    w1 = torch.randn(V, D, generator=gen, device="cuda") * 0.1
    bias = torch.zeros(V, device="cuda")
    m0, m1 = torch.zeros_like(w0), torch.zeros_like(w1)
    sb = [scratch_of(lp.lp_orthogonalize_scratch_bytes(lp.LP_F32, 1, *w.shape)) for w in (w0, w1)]
    for _ in range(3):
        a = torch.relu(x0 @ w0.T)
        got = ce_run(a, w1, bias, labels)
        p0, p1, pb = (t.double().requires_grad_() for t in (w0, w1, bias))
        loss = torch.nn.functional.cross_entropy(torch.relu(x0.double() @ p0.T) @ p1.T + pb, labels.long())
        loss.backward()
        g0 = ((got["dx"] * (a > 0)).T @ x0).contiguous()
        assert abs(float(got["loss"][0]) - float(loss.detach())) < 2e-5
        assert rel(got["dw"], p1.grad) < 2e-5 and rel(got["dbias"], pb.grad) < 2e-5 and rel(g0, p0.grad) < 2e-5
        for w, g, m, s in ((w0, g0, m0, sb[0]), (w1, got["dw"], m1, sb[1])):
            want, _ = muon_reference(w[None], g[None], m[None], 0.02, 0.95, True, 0.0, 1.0)
            lp.lp_muon_update(lp.LP_F32, 1, *w.shape, w, g, m, 0.02, 0.95, True, 0.0, 1.0, 5, None, 1e-7, s[1], s[2])
            assert rel(w[None], want) < 1e-4
        bias -= 0.1 * got["dbias"]
