"""Sizes beyond 32 bits are refused by the binding: ctypes would cut 2^32 + 3 rows to 3."""
import pytest
import torch

import paper_2105_14713_amd as onexn


@pytest.mark.parametrize("name", ["rows", "m", "n", "r", "L"])
def test_workspace_size(name):
    kw = dict(rows=100, m=8, n=8, r=4, L=2)
    assert onexn.fc_lora_bwd_workspace_bytes(**kw) >= 100 * 4 * 4
    for big in (2 ** 31, 2 ** 32 + 3):
        with pytest.raises(ValueError, match=name):
            onexn.fc_lora_bwd_workspace_bytes(**dict(kw, **{name: big}))


@pytest.mark.gpu
def test_calls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    T = 2 ** 32 + 3
    ids = torch.empty(T, dtype=torch.int32, device="cuda")
    x = torch.empty(T, 1, dtype=torch.bfloat16, device="cuda")
    A, B = torch.ones(1, 1, 1, dtype=torch.bfloat16, device="cuda"), torch.ones(1, 1, 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="rows"):
        onexn.fc_lora_fwd(x, A, B, ids, out=x)
    with pytest.raises(ValueError, match="rows"):
        onexn.fc_lora_bwd(None, A, B, ids, None, x, out=x, need=(True, False, False))
    del ids, x
    torch.cuda.empty_cache()
