"""Calls from several host threads at once, the first ones of a process among them, each on its own stream and buffers: what the
library looks up on first use (driver entry point, device properties, kernel attributes) is the same for all."""

import os
import subprocess
import sys
import threading

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def calls(B, torch, seed):
    """One call of each operator on inputs of this seed; the results after a synchronize of the current stream."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for T in (5, 300):
        d, V, K = 128, 2000, 4
        H, W = torch.randn(T, d, generator=g, device="cuda").bfloat16(), (0.1 * torch.randn(V, d, generator=g, device="cuda")).bfloat16()
        y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        logp, lse, ent, tlp = (torch.zeros(*s, device="cuda") for s in ((T,), (T,), (T,), (T, K)))
        ids = torch.zeros(T, K, dtype=torch.int32, device="cuda")
        ws = torch.zeros(B.spo_workspace_bytes(B.WS_LOGPROBS, T=T, d=d, V=V, B=K), dtype=torch.uint8, device="cuda")
        B.spo_logprobs(H, W, y, None, logp, lse, ent, ids, tlp, ws, None)
        dH, dW = torch.zeros_like(H), torch.zeros_like(W)
        ws2 = torch.zeros(B.spo_workspace_bytes(B.WS_LOGPROBS_BWD, T=T, d=d, V=V), dtype=torch.uint8, device="cuda")
        B.spo_logprobs_bwd(H, W, y, None, lse, ent, lse, None, logp, dH, dW, 0, ws2, None)
        out += [logp, lse, ent, ids, tlp, dH, dW]
    G = torch.randn(2, 100, 300, generator=g, device="cuda")
    X = torch.zeros_like(G)
    ws3 = torch.zeros(B.spo_workspace_bytes(B.WS_MUON, T=100, d=300, B=2), dtype=torch.uint8, device="cuda")
    B.spo_orthogonalize(G, X, ws3, B.default_muon_params(), None)
    torch.cuda.current_stream().synchronize()
    return [x.cpu() for x in out + [X]]


def main():
    import torch
    from paper_2509_13232_b200 import binding as B
    torch.zeros(1, device="cuda")
    start = threading.Barrier(4)
    got, errors = {}, []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(60)
                for _ in range(3):
                    got[i] = calls(B, torch, i)
        except Exception as e:                                   # noqa: BLE001 - reported below
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for i in range(4):
        for a, b in zip(got[i], calls(B, torch, i)):
            assert torch.equal(a, b)
    print("alike")


def test_first_calls_of_four_threads():
    out = subprocess.run([sys.executable, "-m", "tests.test_gpu_operator_threads"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "alike" in out.stdout, out.stdout + out.stderr


if __name__ == "__main__":
    main()
