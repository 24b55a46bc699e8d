"""The adapters' products where every one of u's and g's 24 bits counts, bit for
bit against 64 bits, and that fewer planes of them would not pass."""
import pytest
import torch

import paper_2105_14713_amd as onexn
import plane_cases
from adapter_reference import forward

F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]
TYPE_IDS = ["bf16", "bf16_yf32", "f32"]

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
    (4200, 200, 168, 9, 1, "mixed"), (4200, 72, 80, 63, 1, "mixed"), (4200, 80, 72, 50, 2, "runs"),
    (4200, 72, 80, 100, 1, "mixed"), (30, 7, 6, 3, 2, "mixed"),
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


GRADIENTS = [  # T, m, n, r, L, how: each rank class of the gradients' kernel, one range of rows and several
    (1, 40, 50, 2, 1, "runs"), (60, 200, 168, 9, 3, "mixed"), (60, 129, 131, 30, 3, "mixed"),
    (300, 96, 200, 64, 4, "mixed"), (300, 130, 90, 101, 2, "runs"), (1024, 72, 136, 16, 2, "mixed"),
    (1100, 72, 136, 16, 2, "mixed"), (3000, 256, 264, 32, 3, "runs"), (3000, 136, 72, 48, 1, "mixed"),
    (5000, 72, 80, 128, 2, "mixed"), (300, 40, 48, 4, 60, "mixed"), (30, 7, 6, 3, 2, "mixed"),
]
GRADIENT_IDS = ["x".join(map(str, c)) for c in GRADIENTS]


@pytest.mark.parametrize("case", GRADIENTS, ids=GRADIENT_IDS)
def test_gradients_of_fewer_planes_would_not_pass(case):
    c = plane_cases.gradients(*case, BF16, sum(case[:5]))
    ref = plane_cases.factor_gradients(c)
    used = torch.tensor([bool((c["ids"] == l).any()) for l in range(case[4])])
    for keep, name in SHORT:
        # (g of a second rank of a pair has 16 bits: the first ranks differ, in every column of x;
        # u has 24, in every column of a triple that a row selects.)
        dA, dB = plane_cases.factor_gradients(c, keep)
        assert ((dA != ref[0])[:, ::2].all(2).all(1) == used).all(), name
        assert ((dB != ref[1]) == (ref[1] != 0)).all() and (dB != ref[1]).flatten(1).any(1).equal(used), name
    for a, b in zip(plane_cases.factor_gradients(c, lambda v: plane_cases.cut(v, 3)), ref):
        assert torch.equal(a, b) and torch.equal(b.float().double(), b)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", GRADIENTS, ids=GRADIENT_IDS)
def test_every_bit_of_the_gradients(case, dt):
    print("lora planes, gradients", case, dt, flush=True)
    c = plane_cases.gradients(*case, dt, sum(case[:5]))
    ref = plane_cases.factor_gradients(c)
    d = {k: v.cuda() for k, v in c.items()}
    _, dA, dB = onexn.fc_lora_bwd(d["x"], d["A"], d["B"], d["ids"], d["u"], d["dy"], None, d["scale"],
                                  need=(False, True, True))
    assert torch.equal(dA.cpu().double(), ref[0])
    assert torch.equal(dB.cpu().double(), ref[1])
