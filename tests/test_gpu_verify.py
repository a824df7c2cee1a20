"""GPU: treekv_tree_verify against its rule in 64 bits."""
import math
import random

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def inputs(B, n, V, *, dtype="float32", drawn=True, seed=0, near=0.5, chain=False):
    import torch

    g, rng = torch.Generator().manual_seed(seed), random.Random(seed)
    t = getattr(torch, dtype)
    x = 2.0 * torch.randn(B, n + 1, V, generator=g)
    target = torch.softmax(x, dim=2).to(t)
    draft = torch.softmax(x + near * torch.randn(x.shape, generator=g), dim=2).to(t) if drawn else None
    parents = torch.tensor([[i - 1 if chain else max(-1, i - 1 - rng.randrange(4)) for i in range(n)] for _ in range(B)], dtype=torch.int32)
    tokens = torch.empty(B, n, dtype=torch.int32)
    for b in range(B):
        taken = {}
        for i in range(n):
            p = int(parents[b, i]) + 1
            if drawn:
                tokens[b, i] = int(torch.multinomial(draft[b, p].float(), 1, generator=g))
            else:                                            # the most likely ones, one after the other
                k = taken[p] = taken.get(p, -1) + 1
                tokens[b, i] = int(target[b, p].float().topk(min(V, k + 1)).indices[-1])
    return target, draft, tokens, parents, torch.rand(B, n + 1, generator=g)


def run(binding, target, draft, tokens, parents, uniforms, **kw):
    import torch

    B, n = tokens.shape
    new = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")  # noqa: E731
    path, length, follows = new(B, n), new(B), new(B)
    binding.tree_verify(target.cuda(), tokens.cuda(), parents.cuda(), uniforms.cuda(), path, length, follows,
                        draft=None if draft is None else draft.cuda(), **kw)
    return path.cpu(), length.cpu(), follows.cpu()


def check(binding, *case):
    import torch

    from tests.serve_reference import verify

    got, want = run(binding, *case), verify(*[case[i] for i in (0, 1, 2, 3, 4)])
    for name, x, y in zip(("path", "path_len", "next_token"), got, want):
        assert torch.equal(x, y), (name, x, y)
    return got


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("B,n,V", [(1, 1, 1), (2, 1, 2), (5, 3, 7), (40, 9, 33), (3, 26, 4096), (2, 64, 5003), (16, 5, 32001), (1, 256, 129), (2, 7, 160001), (3, 40, 65537)])
def test_trees(binding, B, n, V, dtype, drawn):
    check(binding, *inputs(B, n, V, dtype=dtype, drawn=drawn, seed=n + V))


@pytest.mark.parametrize("near", [0.05, 2.0, 6.0])
def test_chains_near_and_far_from_the_target(binding, near):
    path, length, _ = check(binding, *inputs(60, 8, 500, near=near, chain=True, seed=2))
    assert (int(length.sum()) > 400) if near < 1 else (int(length.min()) == 0)


@pytest.mark.parametrize("V", [300, 70000])
def test_many_siblings_refused(binding, V):
    """A flat tree whose drafter is far off: refusal after refusal of the same row."""
    import torch

    target, draft, tokens, parents, u = inputs(12, 40, V, near=8.0, seed=3)
    parents.fill_(-1)
    for b in range(12):
        tokens[b] = torch.multinomial(draft[b, 0].float(), 40, replacement=True, generator=torch.Generator().manual_seed(b)).int()
    u.clamp_(min=0.9)
    _, length, _ = check(binding, target, draft, tokens, parents, u)
    assert int((length == 0).sum()) > 0
    g = torch.Generator().manual_seed(9)
    check(binding, target, None, torch.stack([torch.randperm(V, generator=g)[:40].int() for _ in range(12)]), parents, u)


@pytest.mark.parametrize("V", [1000, 66000])
@pytest.mark.parametrize("u", [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan])
def test_uniforms_at_the_ends(binding, u, V):
    for drawn in (True, False):
        target, draft, tokens, parents, uniforms = inputs(4, 6, V, drawn=drawn, seed=4)
        uniforms[:, -1] = u
        check(binding, target, draft, tokens, parents, uniforms)
        uniforms.fill_(u)
        check(binding, target, draft, tokens, parents, uniforms)


@pytest.mark.parametrize("V", [64, 65536])
def test_equal_distributions_and_rows_of_nothing(binding, V):
    import torch

    target, draft, tokens, parents, u = inputs(8, 4, V, seed=5)
    u[:, :-1] = 1.0                                           # u Q(x) < P(x) fails for P = Q: nothing is left, P stays
    check(binding, target, target.clone(), tokens, parents, u)
    target[2, 0], target[3], draft[5, 0] = 0.0, math.nan, 0.0
    target[6, 0] = -1.0
    path, length, follows = check(binding, target, draft, tokens, parents, u)
    assert follows[2] == -1 and follows[3] == -1 and follows[6] == -1
    one = torch.zeros(8, 5, V)
    one[:, :, V - 1] = 1.0                                    # everything at the last token
    _, _, follows = check(binding, one, None, tokens, parents, u)
    assert bool((follows == V - 1).all())


def test_tokens_and_parents_that_are_none(binding):
    target, draft, tokens, parents, u = inputs(6, 12, 200, near=0.05, seed=6)
    tokens[0, 0], tokens[1, 2], tokens[2] = 200, -1, 2147483647
    parents[3], parents[4, 3], parents[5, 1] = -2, 3, 11      # absent; its own parent; a parent behind it
    path, length, _ = check(binding, target, draft, tokens, parents, u)
    assert length[2] == 0 and length[3] == 0


@pytest.mark.parametrize("V", [1031, 66047])
def test_the_drawn_token_over_all_of_the_row(binding, V):
    """With nothing accepted the uniform number alone says which token follows: each token's share of [0, 1)."""
    import torch

    p = torch.softmax(torch.randn(1, 2, V, generator=torch.Generator().manual_seed(7)), dim=2)
    at = torch.tensor([0, 1, 255, 256, 511, 512, 777, V - 2, V - 1])
    p[0, 0, at] += 8 * float(p.max())                         # (wide enough for fp32 uniforms to fall into)
    cdf = p[0, 0].double().cumsum(0)
    middle = ((cdf[at] - p[0, 0, at].double() / 2) / cdf[-1]).float()
    u = torch.stack([torch.zeros(9), middle], dim=1)
    parents = torch.full((9, 1), -2, dtype=torch.int32)
    _, _, follows = check(binding, p.expand(9, 2, V).contiguous(), None, torch.zeros(9, 1, dtype=torch.int32), parents, u)
    assert follows.tolist() == at.tolist()


def test_arguments(binding):
    import torch

    target, draft, tokens, parents, u = [x.cuda() for x in inputs(2, 3, 50)]
    out = [torch.empty(2, 3, dtype=torch.int32, device="cuda")] + [torch.empty(2, dtype=torch.int32, device="cuda") for _ in "ab"]
    good = dict(target=target, tokens=tokens, parents=parents, uniforms=u, path=out[0], path_len=out[1], next_token=out[2], draft=draft)
    binding.tree_verify(**good)
    for name, bad in (("target", target.half()), ("target", target.transpose(1, 2)), ("draft", draft.bfloat16()), ("tokens", tokens.long()),
                      ("parents", parents[:, :2]), ("uniforms", u.double()), ("path", out[0].cpu()), ("path_len", out[0]), ("uniforms", u[:, :3])):
        with pytest.raises(ValueError):
            binding.tree_verify(**{**good, name: bad})
    with pytest.raises(binding.TreeKVError):
        binding.tree_verify(**{**good, "path": tokens})
