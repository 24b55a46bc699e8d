"""Clipping where the factor c = max_norm / N leaves fp32's normal range, and how
often a result is rounded, against 64 bits."""
import math

import pytest
import torch

import paper_2105_14713_amd as onexn

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
E32 = torch.finfo(F32).eps / 2
# N is a 64-bit sum of 64-bit squares: a thread adds at most 2^12 of them one after
# the other for lists of up to 2^31 elements, a workgroup's threads and all partial
# sums (some 2^11) follow in trees and short chains: below 2^14 roundings of
# 2^-53.  c and c * g add two more.
E64 = 2.0 ** -39


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    onexn.load_library()


def exact_norm(grads):
    return math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))


def check(got, grads, c):
    """Half a step of the result's type; a bf16 result is rounded to fp32 first.
    Below the smallest normal number half a step is half the smallest value."""
    for o, g in zip(got, grads):
        ref = g.double() * c
        eps = E64 + torch.finfo(g.dtype).eps / 2 + (1.01 * E32 if g.dtype == BF16 else 0.0)
        info = torch.finfo(g.dtype)
        assert ((o.double() - ref).abs() <= eps * ref.abs() + 0.51 * info.smallest_normal * info.eps).all()


def gradients(sizes, dtypes, top, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    # Uniform magnitudes below top, either sign: finite in both types.
    return [(top * (2 * torch.rand(s, generator=gen, device="cuda", dtype=torch.float64) - 1)).to(dtypes[k % len(dtypes)])
            for k, s in enumerate(sizes)]


@pytest.mark.parametrize("dtypes", [(F32,), (BF16,), (F32, BF16)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("most", [1.0, 1e-3, 1e-5, 1e-20, 1e20, 1e-300])
@pytest.mark.parametrize("sizes", [[1000, 3], [1_000_003, 77]], ids=["one_launch", "two_launches"])
def test_huge_finite_gradients(sizes, most, dtypes):
    print("clip huge", sizes, most, dtypes, flush=True)
    grads = gradients(sizes, dtypes, 3.3e38, len(sizes) + sizes[0])
    assert all(torch.isfinite(g).all() for g in grads)
    N = exact_norm(grads)
    assert N > torch.finfo(F32).max                  # beyond fp32: the norm says so, the clipping holds
    out = [torch.full_like(g, float("nan")) for g in grads]
    norm = onexn.clip_grads(grads, most, out=out)
    assert float(norm) == math.inf
    check(out, grads, most / N)
    here = [g.clone() for g in grads]
    onexn.clip_grads(here, most)
    assert all(torch.equal(a, b) for a, b in zip(here, out))


@pytest.mark.parametrize("most", [1e-30, 1e-43, 5e-45])
def test_small_largest_norms_of_ordinary_gradients(most):
    """A factor below fp32's range, and results that are subnormal or vanish."""
    grads = gradients([4000, 200_001], [F32, BF16], 1.0, 5)
    out = [torch.empty_like(g) for g in grads]
    onexn.clip_grads(grads, most, out=out)
    check(out, grads, most / exact_norm(grads))


@pytest.mark.parametrize("dtypes", [(F32,), (BF16,)], ids=["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[9000], [300_000, 5]], ids=["one_launch", "two_launches"])
def test_results_are_rounded_to_their_type_only(sizes, dtypes):
    """Ordinary gradients: c is not rounded to fp32 before it is multiplied."""
    grads = gradients(sizes, dtypes, 2.0, 9)
    for most in (1.0, 0.37, 1 / 3):
        out = [torch.empty_like(g) for g in grads]
        onexn.clip_grads(grads, most, out=out)
        check(out, grads, most / exact_norm(grads))
