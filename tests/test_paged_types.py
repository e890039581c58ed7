"""The binding of the operators on a paged KV cache refuses tensors whose values are of another type, also one of the same size."""
import os

import pytest
import torch

from paper_2505_20438_amd import ham
from tests.test_paged_cpu import tensors

SAME_SIZE = {torch.bfloat16: (torch.float16, torch.int16), torch.float32: (torch.int32,), torch.int32: (torch.float32,)}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ham.LIB_PATH):
        pytest.skip("libham.so not built")


@pytest.mark.parametrize("name", ["append", "attention", "prompt", "advance", "compact"])
def test_values_of_another_type_are_refused(name):
    s, calls = tensors()
    kw = calls[name]
    for key, t in kw.items():
        if not torch.is_tensor(t) or key == "workspace" or (key == "pool" and name in ("advance", "compact")):   # bytes that are moved
            continue
        for kind in SAME_SIZE[t.dtype]:
            with pytest.raises(ham.HamError, match=f"{key} holds values of {kind}") as e:
                getattr(ham, "ham_op_paged_" + name)(s, **dict(kw, **{key: t.view(kind)}))
            assert e.value.code == ham.HAM_EINVAL


def test_rows_of_the_other_storage_type_are_refused():
    s, calls = tensors()
    for key in ("q", "out"):
        with pytest.raises(ham.HamError, match=f"{key} holds"):
            ham.ham_op_paged_prompt(s, **dict(calls["prompt"], **{key: torch.zeros(6, 256)}))   # fp32 act rows: as many bytes
