"""Time one operator of the end of a training step through the C ABI and print its time and rate.

  python -m paper_2112_05387_b200.operator_bench --op ce --rows 4096 --width 2048 --classes 32000 [--dtype bf16] [--loss-only] [--bias]
  python -m paper_2112_05387_b200.operator_bench --op ortho --batch 7 --rows 640 --cols 5760 [--dtype f32] [--steps 5]
  python -m paper_2112_05387_b200.operator_bench --op muon --rows 4096 --cols 4096
  python -m paper_2112_05387_b200.operator_bench --op step --workload wrn28_10      (lp_step_muon beside lp_step)

Also the small command that profiler captures are taken on.  Inputs are seeded N(0,1) tensors; results are not checked here
(tests do that).  Times are CUDA events around calls back to back, after three calls.
"""
import argparse
import json


def timed(f, reps):
    import torch
    for _ in range(3):
        f()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record()
    for _ in range(reps):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / reps


def scratch_for(nbytes):
    import torch
    buf = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
    return buf, (buf.data_ptr() + 255) // 256 * 256


def main():
    import torch
    import paper_2112_05387_b200 as lp
    ap = argparse.ArgumentParser()
    ap.add_argument("--op", default="ce", choices=["ce", "ortho", "muon", "step"])
    ap.add_argument("--dtype", default="bf16", choices=["bf16", "f32"])
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--classes", type=int, default=32000)
    ap.add_argument("--loss-only", action="store_true")
    ap.add_argument("--bias", action="store_true")
    ap.add_argument("--batch", type=int, default=1)
    ap.add_argument("--cols", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--workload", default="wrn28_10")
    ap.add_argument("--reps", type=int, default=20)
    a = ap.parse_args()
    dt, code = (torch.bfloat16, lp.LP_BF16) if a.dtype == "bf16" else (torch.float32, lp.LP_F32)
    g = torch.Generator("cuda").manual_seed(0)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    line = {"op": a.op, "dtype": a.dtype}
    if a.op == "ce":
        T, D, V = a.rows, a.width, a.classes
        x, w = rand(T, D).to(dt), (rand(V, D) / D ** 0.5).to(dt)
        bias = rand(V).to(dt) if a.bias else None
        labels = torch.randint(0, V, (T,), device="cuda", generator=g, dtype=torch.int32)
        loss = torch.empty(2, device="cuda")
        grads = [None if t is None or a.loss_only else torch.empty_like(t) for t in (x, w, bias)]
        need = lp.lp_linear_cross_entropy_scratch_bytes(code, T, D, V, not a.loss_only)
        buf, at = scratch_for(need)
        ms = timed(lambda: lp.lp_linear_cross_entropy(code, T, D, V, x, w, bias, labels, 1.0, loss, None, *grads, at, need), a.reps)
        line.update(shape=[T, D, V], loss_only=a.loss_only, tflops=(2.0 if a.loss_only else 6.0) * T * D * V / ms / 1e9, scratch_bytes=need)
    elif a.op in ("ortho", "muon"):
        B, m, n = a.batch, a.rows, a.cols
        grad = rand(B, m, n).to(dt)
        need = lp.lp_orthogonalize_scratch_bytes(code, B, m, n)
        buf, at = scratch_for(need)
        if a.op == "ortho":
            out = torch.empty_like(grad)
            ms = timed(lambda: lp.lp_orthogonalize(code, B, m, n, grad, out, a.steps, None, 1e-7, at, need), a.reps)
        else:
            w, mom = rand(B, m, n).to(dt), torch.zeros(B, m, n, device="cuda")
            ms = timed(lambda: lp.lp_muon_update(code, B, m, n, w, grad, mom, 1e-3, 0.95, True, 0.0, 1.0, a.steps, None, 1e-7, at, need), a.reps)
        s, l = min(m, n), max(m, n)
        line.update(shape=[B, m, n], tflops=B * a.steps * (s * (s + 1.0) * (l + s) + 2.0 * s * s * l) / ms / 1e9, scratch_bytes=need)
    else:
        from workloads import get_config
        cfg = get_config(a.workload)
        h = lp.lp_create(lp.desc_from_config(cfg))
        code = cfg["dtype"]
        act = torch.float32 if code == "f32" else torch.bfloat16
        x = [rand(*lp.lp_boundary_shape(h, k)).to(act) for k in range(h.K)]
        labels = torch.randint(0, cfg["num_classes"], (cfg["N"],), device="cuda", generator=g, dtype=torch.int32)
        loss = torch.zeros(h.K, 2, device="cuda")
        need = lp.lp_step_muon_scratch_bytes(h)
        buf, at = scratch_for(need)

        def passes():
            lp.lp_modules_fwd_bwd_all(h, x, labels, None, cfg["rho"], loss, None)
        # (a step applies fresh gradients only: the passes alone are taken off)
        base = timed(passes, a.reps)
        sgd = timed(lambda: (passes(), lp.lp_step(h, 0.0, 0.9)), a.reps) - base
        ms = timed(lambda: (passes(), lp.lp_step_muon(h, 0.0, 0.0, 0.9, True, 0.0, 0.0, None, at, need)), a.reps) - base
        line.update(workload=a.workload, dtype=code, passes_ms=base, lp_step_ms=sgd, scratch_bytes=need)
    line["ms"] = ms
    print(json.dumps(line))


if __name__ == "__main__":
    main()
