"""Norms, gradient norm and AdamW from several host threads at once, each on its own stream and buffers, with sizes that differ in
the shared memory a launch asks for: what a kernel is allowed does not depend on the call that another thread makes."""

import os
import subprocess
import sys
import threading

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (rows, width, pitch behind the width, fp32 gradients with dh): the same kernel in each direction for all of a line, with 37 to 100 KB
# of shared memory a block
ALIKE = [
    [(200, 4096, 0, True), (200, 4096, 0, False), (200, 2304, 0, True), (200, 2304, 0, False)],
    [(200, 4001, 3, True), (200, 4001, 3, False), (200, 2501, 3, True), (200, 2501, 3, False)],
]


def inputs(torch, B, seed, T, d, pad, wide):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    bf = lambda *s: r(*s).bfloat16()  # noqa: E731
    s = dict(x=bf(T, d + pad)[:, :d], w=bf(d), b=bf(d), dy=r(T, d) if wide else bf(T, d), dh=bf(T, d) if wide else None)
    s.update(y=torch.zeros(T, d, device="cuda", dtype=torch.bfloat16), dx=torch.zeros(T, d, device="cuda", dtype=torch.bfloat16))
    s.update(mean=torch.zeros(T, device="cuda"), rstd=torch.zeros(T, device="cuda"), dw=torch.zeros(d, device="cuda"), db=torch.zeros(d, device="cuda"))
    s["ws"] = torch.zeros(B.spo_workspace_bytes(B.WS_LAYERNORM_BWD, T=T, d=d), dtype=torch.uint8, device="cuda")
    s.update(p=r(d), m=torch.zeros(d, device="cuda"), v=torch.zeros(d, device="cuda"), norm=torch.zeros(4, device="cuda"))
    s["ws2"] = torch.zeros(B.spo_workspace_bytes(B.WS_GRAD_NORM), dtype=torch.uint8, device="cuda")
    s["grads"], s["step"] = B.grad_list([s["dw"], s["db"]]), B.adamw_list([s["p"]], [s["dw"]], [s["m"]], [s["v"]])
    return s


def calls(B, s):
    B.spo_layernorm_fwd(s["x"], None, s["w"], s["b"], None, s["y"], None, s["mean"], s["rstd"], None)
    B.spo_layernorm_bwd(s["dy"], s["x"], s["w"], None, s["mean"], s["rstd"], s["dh"], s["dx"], s["dw"], s["db"], 0, s["ws"], None)
    B.spo_grad_norm(s["grads"], s["norm"], s["ws2"], None, max_norm=1.0)
    B.spo_adamw_update(s["step"], s["norm"][1:2], None, None, B.default_adamw_params(), None)


def bare(B, torch, s, times):
    """The norm's two calls again and again without the binding's checks, so that threads meet between a call's first step and its launch
    (a limit lowered there refused some launches in a thousand)."""
    L, p = B.lib(), lambda t: None if t is None else t.data_ptr()  # noqa: E731
    (T, d), ld, st = s["x"].shape, s["x"].stride(0), torch.cuda.current_stream().cuda_stream
    code = B.DTYPE_BF16
    fwd = (p(s["x"]), ld, None, code, p(s["w"]), p(s["b"]), code, None, T, d, 1e-6, B.NORM_LAYER, p(s["y"]), code, None, p(s["mean"]),
           p(s["rstd"]), None, st)
    bwd = (p(s["dy"]), code if s["dh"] is None else B.DTYPE_F32, p(s["x"]), ld, code, p(s["w"]), code, None, p(s["mean"]), p(s["rstd"]), p(s["dh"]),
           T, d, B.NORM_LAYER, p(s["dx"]), p(s["dw"]), p(s["db"]), B.DTYPE_F32, 0, p(s["ws"]), s["ws"].numel(), None, st)
    refused = 0
    for _ in range(times // 2):
        refused += L.spo_layernorm_fwd(*fwd) != 0
        refused += L.spo_layernorm_bwd(*bwd) != 0
    assert refused == 0, "%d of %d calls refused" % (refused, times)


RESULTS = ("y", "mean", "rstd", "dx", "dw", "db", "norm", "p", "m", "v")


def main():
    import torch
    from paper_2509_13232_b200 import binding as B
    B.lib()
    for line in ALIKE:
        got, errors, start = {}, [], threading.Barrier(len(line))

        def work(i):
            try:
                with torch.cuda.stream(torch.cuda.Stream()):
                    s = inputs(torch, B, i, *line[i])
                    start.wait(60)
                    for _ in range(100):
                        calls(B, s)
                    bare(B, torch, s, 20000)
                    torch.cuda.current_stream().synchronize()
                    got[i] = {k: s[k].cpu() for k in RESULTS}
            except Exception as e:                                   # noqa: BLE001 - reported below
                errors.append(e)

        threads = [threading.Thread(target=work, args=(i,)) for i in range(len(line))]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not errors, errors
        for i, shape in enumerate(line):
            s = inputs(torch, B, i, *shape)
            for _ in range(100):
                calls(B, s)
            torch.cuda.synchronize()
            assert all(torch.equal(got[i][k], s[k].cpu()) for k in RESULTS), shape
    print("alike")


def test_four_threads_with_sizes_of_their_own():
    out = subprocess.run([sys.executable, "-m", "tests.test_gpu_step_threads"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "alike" in out.stdout, out.stdout + out.stderr


def test_a_captured_call_beside_smaller_ones():
    """A captured call replayed after calls of the same kernel that ask for less."""
    import torch
    from paper_2509_13232_b200 import binding as B
    for line in ALIKE:
        s = [inputs(torch, B, i, *shape) for i, shape in enumerate(line)]
        once = lambda q: (B.spo_layernorm_fwd(q["x"], None, q["w"], q["b"], None, q["y"], None, q["mean"], q["rstd"], None),  # noqa: E731
                          B.spo_layernorm_bwd(q["dy"], q["x"], q["w"], None, q["mean"], q["rstd"], q["dh"], q["dx"], q["dw"], q["db"], 0, q["ws"], None))
        once(s[0])
        torch.cuda.synchronize()
        want = [s[0][k].clone() for k in ("y", "dx", "dw", "db")]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            once(s[0])
        for q in s[1:]:
            once(q)
        for k in ("y", "dx", "dw", "db"):
            s[0][k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, s[0][k]) for a, k in zip(want, ("y", "dx", "dw", "db")))


if __name__ == "__main__":
    main()
