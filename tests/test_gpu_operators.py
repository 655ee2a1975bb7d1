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
               (2, 128, 1152), (1, 5000, 7), (200, 64, 64), (1, 100, 40000), (3, 1152, 127), (1, 17, 33), (2, 3, 3000)]


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
