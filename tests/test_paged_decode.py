"""What the loop over a pool of pages refuses, before anything is read or changed (no GPU needed)."""
import pytest
import torch


def test_acceptance_refuses_other_types_and_shapes():
    """Logits of a narrower type would be read past their end, more nodes than a step's written past the buffers'."""
    from paper_2405_18628_gb300 import paged_decode as S
    B, T, V = 2, 4, 30
    req = S.PagedRequests(1, B, 1, 1, T, 64, V, 9, 16, 4, 20, device="cpu")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    fine = dict(logits=torch.zeros(B, T, V), cand_tokens=i32(B, T), parent=i32(B, T))
    for name, bad, error in (("logits", torch.zeros(B, T, V, dtype=torch.bfloat16), TypeError), ("logits", torch.zeros(B, T, V, dtype=torch.float16), TypeError),
                             ("logits", torch.zeros(B, T + 1, V), ValueError), ("logits", torch.zeros(B + 1, T, V), ValueError),
                             ("logits", torch.zeros(B, T, V - 1), ValueError), ("cand_tokens", i32(B, T).long(), TypeError), ("cand_tokens", i32(B, T + 1), ValueError),
                             ("parent", i32(B, T).long(), TypeError), ("parent", i32(B, T - 1), ValueError)):
        with pytest.raises(error, match=f"^{name} "):
            req.accept(**dict(fine, **{name: bad}))
    with pytest.raises(ValueError, match="contiguous CUDA"):
        req.accept(**fine)
