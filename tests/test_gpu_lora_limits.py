"""The adapters' calls at their limits: factors of nearly 2^31 elements, no rows in
narrow layers, several ranges of rows captured into graphs."""
import pytest
import torch

import paper_2105_14713_amd as onexn
from test_gpu_fc_lora import BF16, F32, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    onexn.load_library()


@pytest.mark.parametrize("r,width", [(127, 2 ** 24), (15, 2 ** 27)])
def test_largest_factors(r, width):
    """127 * 2^24 and 15 * 2^27 elements a factor: what is nonzero lies at their ends."""
    print("lora largest factors", r, width, flush=True)
    T, L = 3, 1
    last = width - 1
    A = torch.zeros(L, r, width, dtype=BF16, device="cuda")
    A[0, 0, 0], A[0, r - 1, last], A[0, r - 1, last - 8] = 2.0, 3.0, -1.0
    x = torch.zeros(T, width, dtype=BF16, device="cuda")
    x[0, last], x[1, last - 8], x[2, 0] = 1.0, 4.0, 5.0
    narrow = torch.zeros(L, r, 16, dtype=BF16, device="cuda")
    narrow[0, 0, 1], narrow[0, r - 1, 2] = 1.0, 2.0
    ids = torch.zeros(T, dtype=torch.int32, device="cuda")
    u = torch.empty(T, r, device="cuda")
    y = onexn.fc_lora_fwd(x, A, narrow, ids, u=u)
    want_u = torch.zeros(T, r)
    want_u[0, r - 1], want_u[1, r - 1], want_u[2, 0] = 3.0, -4.0, 10.0
    assert torch.equal(u.cpu(), want_u)
    want_y = torch.zeros(T, 16)
    want_y[0, 2], want_y[1, 2], want_y[2, 1] = 6.0, -8.0, 10.0
    assert torch.equal(y.float().cpu(), want_y)
    dy = torch.zeros(T, 16, dtype=BF16, device="cuda")
    dy[0, 2], dy[1, 1], dy[2, 2] = 1.0, 1.0, -2.0            # g: 2 at rank r - 1; 1 at rank 0; -4 at rank r - 1
    dx, dA, _ = onexn.fc_lora_bwd(x, A, narrow, ids, None, dy, need=(True, True, False))
    assert float(dx[0, last]) == 6.0 and float(dx[0, last - 8]) == -2.0 and float(dx[1, 0]) == 2.0
    assert float(dx[2, last]) == -12.0 and int(dx.count_nonzero()) == 5
    del dx
    assert float(dA[0, r - 1, last]) == 2.0 and float(dA[0, 0, last - 8]) == 4.0 and float(dA[0, r - 1, 0]) == -20.0
    assert sum(int(dA[0, j].count_nonzero()) for j in range(r)) == 3
    del A, x, dA
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(3, 200), (200, 3), (2, 2)])
def test_no_rows_in_narrow_layers(m, n, dt):
    A, B = torch.ones(2, 4, m, dtype=dt, device="cuda"), torch.ones(2, 4, n, dtype=dt, device="cuda")
    x, dy = torch.empty(0, m, dtype=dt, device="cuda"), torch.empty(0, n, dtype=dt, device="cuda")
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    assert onexn.fc_lora_fwd(x, A, B, ids).shape == (0, n)
    dA, dB = torch.full((2, 4, m), 7.0, device="cuda"), torch.full((2, 4, n), 7.0, device="cuda")
    onexn.fc_lora_bwd(x, A, B, ids, torch.empty(0, 4, device="cuda"), dy, dA=dA, dB=dB)
    assert not dA.any() and not dB.any()


@pytest.mark.parametrize("T,m,n,r,L,dt", [(3000, 256, 200, 12, 1, BF16), (5000, 300, 3, 40, 2, F32), (3000, 2, 5, 8, 2, BF16)])
def test_ranges_captured_and_replayed(T, m, n, r, L, dt):
    """Two graphs in turn, eager calls and other inputs between: every replay as the eager call."""
    print("lora captured", T, m, n, r, L, dt, flush=True)

    def step(d, out):
        u = d["x"].new_empty((T, r), dtype=F32)
        out["y"].copy_(onexn.fc_lora_fwd(d["x"], d["A"], d["B"], d["ids"], d["base"], d["scale"], u=u))
        dx, dA, dB = onexn.fc_lora_bwd(d["x"], d["A"], d["B"], d["ids"], u, d["dy"], d["dbase"], d["scale"])
        out["dx"].copy_(dx), out["dA"].copy_(dA), out["dB"].copy_(dB)

    def buffers():
        return {"y": torch.empty(T, n, dtype=dt, device="cuda"), "dx": torch.empty(T, m, dtype=dt, device="cuda"),
                "dA": torch.empty(L, r, m, device="cuda"), "dB": torch.empty(L, r, n, device="cuda")}
    cases = [{k: v.cuda() for k, v in make(T, m, n, r, L, "mixed", dt, dt, False, s).items()} for s in range(4)]
    graphs = []
    for s in range(2):
        d, out = {k: v.clone() for k, v in cases[s].items()}, buffers()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(d, out)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(d, out)
        graphs.append((g, d, out))
    for turn in range(6):
        for k, (g, d, out) in enumerate(graphs):
            new = cases[(turn + k) % 4]
            for name, v in new.items():
                d[name].copy_(v)
            for v in out.values():
                v.fill_(float("nan"))
            g.replay()
            want = buffers()
            step(new, want)
            torch.cuda.synchronize()
            for name in want:
                assert torch.equal(out[name], want[name]), (turn, k, name)
