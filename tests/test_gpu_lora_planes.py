"""The adapters' products where every one of u's and g's 24 bits counts, bit for
bit against 64 bits, and that fewer planes of them would not pass."""
import pytest
import torch

import paper_2105_14713_amd as onexn
import plane_cases
from adapter_reference import forward

F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(BF16, BF16)]
TYPE_IDS = ["bf16"]

CASES = [  # T, m, n, r, L, how: each rank class in each way that rows are put into tiles
    (1, 40, 50, 2, 1, "mixed"), (33, 200, 168, 2, 3, "mixed"), (40, 200, 168, 16, 3, "mixed"),
    (64, 130, 300, 20, 9, "mixed"), (50, 200, 168, 40, 4, "mixed"), (50, 200, 168, 101, 2, "mixed"),
    (300, 96, 200, 12, 5, "mixed"), (300, 96, 200, 30, 5, "runs"), (300, 96, 200, 64, 3, "mixed"),
    (300, 96, 200, 128, 2, "mixed"), (300, 40, 48, 4, 1100, "mixed"),
    (50, 600, 168, 16, 1, "mixed"), (50, 168, 600, 24, 1, "mixed"), (50, 600, 600, 64, 1, "mixed"),
    (50, 600, 168, 128, 1, "mixed"),
    (50, 200, 168, 9, 1, "mixed"), (50, 200, 168, 32, 1, "mixed"), (50, 168, 200, 63, 1, "mixed"),
    (50, 200, 168, 96, 1, "mixed"),
    (4200, 96, 104, 16, 5, "mixed"), (4200, 96, 104, 32, 5, "runs"), (4200, 600, 104, 50, 3, "runs"),
    (4200, 96, 104, 70, 2, "runs"), (8200, 64, 72, 40, 1, "mixed"), (8200, 64, 72, 64, 3, "runs"),
    (30, 7, 6, 3, 2, "mixed"),
]
IDS = ["x".join(map(str, c)) for c in CASES]


def with_planes(c, keep):
    """The product with u held as `keep` gives it."""
    u, _ = forward(c["x"], c["A"], c["B"], c["ids"], None, c["scale"])
    u = keep(u.float())
    y = c["base"].double().clone()
    for l in range(c["A"].shape[0]):
        at = c["ids"] == l
        y[at] += u[at].double() @ c["B"][l].double()
    return y


SHORT = [(keep, name) for keep, name in ((lambda v: plane_cases.cut(v, 1), "one"),
                                         (lambda v: plane_cases.cut(v, 2), "two"),
                                         (plane_cases.cut_two_rounded, "two_rounded"))]


def differs_in_every_row(c, odt):
    """Whether fewer planes change every row that has an adapter, and three none."""
    _, ref = forward(c["x"], c["A"], c["B"], c["ids"], c["base"], c["scale"])
    some = (c["ids"] >= 0) & (c["ids"] < c["A"].shape[0])
    for keep, name in SHORT:
        other = (with_planes(c, keep).to(odt) != ref.to(odt)).any(1)
        assert torch.equal(other, some), name
    assert torch.equal(with_planes(c, lambda v: plane_cases.cut(v, 3)), ref)
    return some.any()


@pytest.mark.parametrize("types", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_fewer_planes_would_not_pass(case, types):
    assert differs_in_every_row(plane_cases.product(*case, *types, sum(case[:5])), types[1])


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_every_bit_of_u(case, types):
    print("lora planes", case, types, flush=True)
    c = plane_cases.product(*case, *types, sum(case[:5]))
    ref_u, ref_y = forward(c["x"], c["A"], c["B"], c["ids"], c["base"], c["scale"])
    d = {k: v.cuda() for k, v in c.items()}
    u = torch.empty(ref_u.shape, device="cuda")
    y = onexn.fc_lora_fwd(d["x"], d["A"], d["B"], d["ids"], d["base"], d["scale"], u=u)
    assert torch.equal(u.cpu().double(), ref_u)
    assert torch.equal(y.cpu(), ref_y.to(types[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_every_bit_of_g(case, types):
    """The same product as an input gradient: dy, B and A in the places of x, A and B."""
    print("lora planes, input gradient", case, types, flush=True)
    c = plane_cases.product(*case, *types, sum(case[:5]))
    _, ref = forward(c["x"], c["A"], c["B"], c["ids"], c["base"], c["scale"])
    d = {k: v.cuda() for k, v in c.items()}
    dx, _, _ = onexn.fc_lora_bwd(None, d["B"], d["A"], d["ids"], None, d["x"], d["base"], d["scale"],
                                 need=(True, False, False))
    assert torch.equal(dx.cpu(), ref.to(types[1]))
