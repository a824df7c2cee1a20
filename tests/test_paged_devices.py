"""Where a PagedKV makes what it is not given.  No GPU is needed: meta tensors stand in for those of another device."""
import pytest


@pytest.fixture(scope="module")
def binding():
    import os

    from paper_2501_04987_amd import binding as b
    from paper_2501_04987_amd import build

    if not os.path.exists(b.LIB_PATH):
        build.build()
    b.load()
    return b


def given(device):
    import torch

    pool = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device=device)
    return dict(k=pool, v=torch.zeros_like(pool), table=torch.full((3, 2), -1, dtype=torch.int32, device=device),
                lens=torch.zeros(3, dtype=torch.int32, device=device))


@pytest.mark.parametrize("names", [("k",), ("k", "v"), ("k", "v", "table", "lens")])
def test_what_is_made_lies_where_the_pool_lies(binding, names):
    at, other = given("cpu"), "meta"
    kv = binding.PagedKV(4, 16, 2, 64, batch=3, table_width=2, device=other, **{n: at[n] for n in names})
    assert kv.device.type == "cpu"
    for name in ("k", "v", "table", "lens", "weights", "positions"):
        assert getattr(kv, name).device.type == "cpu", name
    assert bool((kv.positions == -1).all()) and not bool(kv.weights.any()) and kv.cache.weights == kv.weights.data_ptr()


def test_where_no_pool_is_given_the_device_counts(binding):
    kv = binding.PagedKV(4, 16, 2, 64, batch=3, table_width=2, device="cpu")
    assert {getattr(kv, n).device.type for n in ("k", "v", "table", "lens", "weights", "positions")} == {"cpu"}


def test_numbers_that_32_bits_do_not_hold_are_refused(binding):
    """ctypes would cut them: a budget of 2^32 + 16 would be one of 16."""
    import torch

    kv = binding.PagedKV(4, 16, 2, 64, table_width=2, device="cpu")
    q, starts = torch.zeros(1, 2, 64, dtype=torch.bfloat16), torch.tensor([0, 1], dtype=torch.int32)
    for far in (2 ** 32 + 16, 2 ** 31, -2 ** 31 - 1):
        for call in (lambda: kv.evict(far, 0, 0), lambda: kv.evict(16, far, 0), lambda: kv.evict(16, 0, far), lambda: kv.attend(q, starts, far),
                     lambda: kv.new_attend_scratch(1, far), lambda: kv.new_attend_scratch(far, 1),
                     lambda: binding.PagedKV(4, 16, 2, 64, table_width=2, batch=far, device="meta")):
            with pytest.raises(ValueError, match="32 bits"):
                call()
