"""Arguments of reading keys or values alone, without a GPU."""
import pytest
import torch

from paper_2510_19482_amd import binding as B
from test_attn_devices import cache, ints, rows, two_devices   # noqa: F401
from test_mx4_devices import Tensor, machine   # noqa: F401


@pytest.mark.parametrize("only", ["k", "v"])
def test_the_other_side_is_not_asked_for(two_devices, only, monkeypatch):   # noqa: F811
    made, given = [], []
    monkeypatch.setattr(B, "_empty", lambda shape, dtype, device, stream: made.append(shape) or rows(0, 5, 2))
    setattr(B.lib, "hlq_kv_read", lambda *args: given.append((args[6], args[9])) or 0)
    k, v = B.hlq_kv_read(cache(0), ints(0, 5, dtype=torch.int64), only=only)
    assert made == [(5, 2, 64)] and (k is None, v is None) == (only == "v", only == "k")
    assert [a is None for a in given[0]] == [only == "v", only == "k"]


def test_what_does_not_go_together_is_refused():
    kv, slots, x = B.alloc_kv_cache(3, 16, 2, 32, torch.bfloat16, device="cpu"), torch.zeros(5, dtype=torch.int64), torch.zeros((5, 2, 32))
    for args in (dict(k=x, only="v"), dict(v=x, only="k"), dict(only="q"), dict(only=True), dict(k=x, v=x, only="k")):
        with pytest.raises(ValueError, match="only"):
            B.hlq_kv_read(kv, slots, **args)
    for args in (dict(k=x[:, :1], only="k"), dict(v=x[:4], only="v")):
        with pytest.raises(ValueError, match="rows"):
            B.hlq_kv_read(kv, slots, **args)
    for args in (dict(k=x, only="k"), dict(v=x, only="v")):
        with pytest.raises(ValueError, match="one GPU"):
            B.hlq_kv_read(kv, slots, **args)
