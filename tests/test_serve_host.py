"""Argument checks of the paged cache and of the verification of drafts that need no GPU: every call here returns before
anything is enqueued.  And the same host code under AddressSanitizer and UBSan."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2501_04987_amd import binding as b
    from paper_2501_04987_amd import build

    if not os.path.exists(b.LIB_PATH):
        build.build()
    b.load()
    return b


MB = 1 << 20


def cache(b, **kw):
    base = dict(k=0x10 * MB, v=0x20 * MB, table=0x30 * MB, lens=0x31 * MB, weights=0x32 * MB, positions=0x33 * MB, pages=8, page_size=16,
                table_width=4, batch=2, q_heads=4, kv_heads=2, head_dim=64, dtype=b.TREEKV_BF16, softmax_scale=0.0)
    return C.addressof(hold(b.treekv_paged_cache(**{**base, **kw})))


held = []


def hold(x):
    held.append(x)
    return x


BAD_CACHES = [(dict(k=None), -1), (dict(v=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(k=0x10 * MB + 8), -1),
              (dict(v=0x20 * MB + 4), -1), (dict(weights=None), -1), (dict(weights=0x32 * MB + 4), -1), (dict(positions=None), -1), (dict(dtype=2), -1), (dict(pages=0), -1),
              (dict(page_size=0), -1), (dict(page_size=-16), -1), (dict(table_width=0), -1), (dict(batch=0), -1), (dict(kv_heads=0), -1),
              (dict(q_heads=0), -1), (dict(q_heads=5), -1), (dict(softmax_scale=float("nan")), -1), (dict(softmax_scale=float("inf")), -1),
              (dict(head_dim=96), -4), (dict(page_size=8), -4), (dict(page_size=48), -4), (dict(page_size=512), -4),
              (dict(table_width=1 << 27), -4), (dict(batch=1 << 20), -4), (dict(q_heads=1 << 17), -4)]


def test_caches(binding):
    lib = binding.load()
    a, out, other = 0x40 * MB, 0x50 * MB, 0x60 * MB
    for kw, want in BAD_CACHES:
        c = cache(binding, **kw)
        assert lib.treekv_paged_append(c, a, a, 128, 128, other, 3, other, None, None) == want, kw
        assert lib.treekv_paged_attend(c, a, 256, other, 3, 3, out, None, 0, other, 1 << 30, None, None) == want, kw
        assert lib.treekv_paged_evict(c, 20, 2, 10, None, other, 1 << 30, None, None) == want, kw
        assert lib.treekv_paged_attend_scratch_bytes(c, 3, 3, 1) == 0 and lib.treekv_paged_evict_scratch_bytes(c) == 0, kw
    assert lib.treekv_paged_append(None, a, a, 128, 128, other, 3, other, None, None) == -1
    assert lib.treekv_paged_attend(None, a, 256, other, 3, 3, out, None, 0, other, 1 << 30, None, None) == -1
    assert lib.treekv_paged_evict(None, 20, 2, 10, None, other, 1 << 30, None, None) == -1
    assert lib.treekv_paged_attend_scratch_bytes(None, 3, 3, 0) == 0 and lib.treekv_paged_evict_scratch_bytes(None) == 0


def test_a_scale_that_fp32_does_not_hold_in_base_2(binding):
    """Logits are scaled by softmax_scale * log2(e) in fp32: where that is infinite a logit of 0 would be a NaN."""
    lib = binding.load()
    a, out, other = 0x40 * MB, 0x50 * MB, 0x60 * MB
    for scale in (2.4e38, -2.4e38, 3.4e38):
        c = cache(binding, softmax_scale=scale)
        assert lib.treekv_paged_attend(c, a, 256, other, 3, 3, out, None, 0, other, 1 << 30, None, None) == -1, scale
        assert lib.treekv_paged_attend_scratch_bytes(c, 3, 3, 1) == 0
    assert lib.treekv_paged_attend_scratch_bytes(cache(binding, softmax_scale=2.3e38), 3, 3, 1) > 0


def refuses(call, good, bad, want=-1):
    """`good` with each of the (place, value) of `bad` is refused."""
    for i, x in bad:
        assert call(*[x if j == i else y for j, y in enumerate(good)]) == want, (i, x)


def test_append(binding):
    lib, c = binding.load(), cache(binding)
    a, b, starts, pos, st = 0x40 * MB, 0x41 * MB, 0x50 * MB, 0x51 * MB, 0x52 * MB
    good = [c, a, b, 128, 128, starts, 3, pos, st, None]
    refuses(lib.treekv_paged_append, good, [(1, None), (2, None), (1, a + 8), (2, b + 2), (3, 127), (4, 0), (4, -128), (3, 132), (4, 1 << 60), (5, None),
                                            (6, 0), (6, -1), (7, None)])
    # what it writes may not lie in what it reads, or in another output
    refuses(lib.treekv_paged_append, good, [(1, 0x10 * MB), (2, 0x20 * MB + 16), (5, 0x32 * MB), (7, 0x33 * MB), (8, 0x10 * MB), (8, pos), (8, 0x31 * MB)])
    for kw in (dict(v=0x10 * MB + 16), dict(positions=0x32 * MB), dict(weights=0x10 * MB), dict(table=0x10 * MB), dict(lens=0x33 * MB)):
        refuses(lib.treekv_paged_append, good, [(0, cache(binding, **kw))])
    refuses(lib.treekv_paged_append, good, [(0, cache(binding, weights=None, positions=None))])      # no positions are kept


def test_attend(binding):
    lib, c = binding.load(), cache(binding)
    q, out, lse, starts, scratch, st = 0x40 * MB, 0x50 * MB, 0x60 * MB, 0x61 * MB, 0x70 * MB, 0x62 * MB
    need = lib.treekv_paged_attend_scratch_bytes(c, 5, 4, 1)
    assert need >= 5 * 4 * 4
    assert all(lib.treekv_paged_attend_scratch_bytes(c, *x) == 0 for x in ((0, 1, 0), (3, 4, 0), (3, 0, 0), (-1, -1, 0), (2 ** 31 - 1, 2 ** 31 - 1, 0)))
    good = [c, q, 256, starts, 5, 4, out, lse, 1, scratch, need, st, None]
    refuses(lib.treekv_paged_attend, good, [(1, None), (1, q + 8), (2, 255), (2, -256), (2, 260), (2, 1 << 60), (3, None), (4, 0), (4, 3), (5, 0), (5, 6),
                                            (6, None), (6, out + 4), (9, None), (9, scratch + 8), (10, need - 1), (10, 0)])
    # outputs may not lie in each other, in the cache or in what is read
    refuses(lib.treekv_paged_attend, good, [(6, q), (6, q + 256), (7, out), (7, 0x10 * MB), (9, out), (9, 0x20 * MB), (11, lse), (11, 0x31 * MB), (6, 0x30 * MB),
                                            (6, starts - 256)])
    refuses(lib.treekv_paged_attend, good, [(0, cache(binding, weights=None, positions=None)), (0, cache(binding, weights=0x10 * MB)),
                                            (0, cache(binding, weights=0x40 * MB))])
    big = cache(binding, q_heads=65536, kv_heads=1)
    assert lib.treekv_paged_attend(big, q, 65536 * 64, starts, 1 << 20, 1 << 20, 0x100000 * MB, None, 0, scratch, 1 << 40, None, None) == -4


def test_scratch_sizes(binding):
    """Partial results of all shares, in 64 bits; none where there is a workgroup for every compute unit without them."""
    lib = binding.load()
    one = cache(binding, batch=1, table_width=4096, q_heads=32, kv_heads=8, head_dim=128, pages=1 << 20)
    assert lib.treekv_paged_attend_scratch_bytes(one, 1, 1, 0) >= 8 * 256 * 16 * 132 * 4 // 8
    assert lib.treekv_paged_attend_scratch_bytes(one, 1, 1, 1) >= lib.treekv_paged_attend_scratch_bytes(one, 1, 1, 0) + 32 * 4
    f32 = cache(binding, batch=1, table_width=4096, q_heads=32, kv_heads=32, head_dim=128, pages=1 << 20, dtype=binding.TREEKV_F32)
    assert lib.treekv_paged_attend_scratch_bytes(f32, 4096, 4096, 0) == 0
    assert lib.treekv_paged_evict_scratch_bytes(one) >= 8 * 4096 * 16 // 2 * 8
    deep = cache(binding, batch=64, table_width=1 << 20, q_heads=8, kv_heads=8, head_dim=128, pages=1 << 20)
    assert lib.treekv_paged_attend_scratch_bytes(deep, 1, 1, 0) > 0 and lib.treekv_paged_attend_scratch_bytes(deep, 1, 1, 1) == 0      # 2^33 weights
    wide = cache(binding, batch=4096, table_width=1 << 20, q_heads=256, kv_heads=256)
    assert lib.treekv_paged_evict_scratch_bytes(wide) >= 1 << 45


def test_evict(binding):
    lib, c = binding.load(), cache(binding)
    scratch, st = 0x70 * MB, 0x62 * MB
    need = lib.treekv_paged_evict_scratch_bytes(c)
    good = [c, 20, 4, 10, 0x63 * MB, scratch, need, st, None]
    refuses(lib.treekv_paged_evict, good, [(1, 0), (1, -5), (2, -1), (3, -1), (2, 11), (3, 17), (3, 2147483647), (5, None), (5, scratch + 4), (6, need - 1),
                                           (5, 0x10 * MB), (7, scratch), (7, 0x31 * MB), (4, 0x31 * MB + 4), (4, st), (4, scratch), (4, 0x30 * MB), (0, cache(binding, weights=None, positions=None)),
                                           (0, cache(binding, v=0x10 * MB)), (0, cache(binding, lens=0x32 * MB))])


def test_verify(binding):
    lib = binding.load()
    base = dict(target=0x100 * MB, draft=0x200 * MB, tokens=0x10 * MB, parents=0x11 * MB, uniforms=0x12 * MB, path=0x13 * MB, path_len=0x14 * MB,
                next_token=0x15 * MB, scratch=0x16 * MB, scratch_bytes=1 << 20, batch=2, n=9, vocab=1000, dtype=binding.TREEKV_F32)

    def call(**kw):
        args = binding.treekv_verify_args(**{**base, **kw})
        return lib.treekv_tree_verify(C.byref(args), None)

    for kw in (dict(target=None), dict(tokens=None), dict(parents=None), dict(uniforms=None), dict(path=None), dict(path_len=None),
               dict(next_token=None), dict(target=0x100 * MB + 4), dict(draft=0x200 * MB + 8), dict(scratch=0x16 * MB + 8), dict(batch=0), dict(batch=-1),
               dict(n=0), dict(n=257), dict(vocab=0), dict(vocab=-8), dict(dtype=2), dict(path=0x10 * MB), dict(path_len=0x13 * MB + 4),
               dict(next_token=0x14 * MB), dict(path=0x100 * MB + 4096), dict(path_len=0x12 * MB)):
        assert call(**kw) == -1, kw
    assert call(vocab=(1 << 24) + 1) == -4 and call(batch=(1 << 20) + 1, target=1 << 50, draft=None) == -4 and lib.treekv_tree_verify(None, None) == -1
    size = lib.treekv_tree_verify_scratch_bytes
    assert all(size(*x) == 0 for x in ((0, 1, 1), (1, 0, 1), (1, 257, 1), (1, 1, 0), (1, 1, (1 << 24) + 1), (-1, -1, -1)))
    need = size(2, 9, 1000)
    if need:
        assert call(scratch_bytes=need - 1) == -1 and call(scratch=None) == -1 and call(scratch=0x13 * MB) == -1


def test_tensors_on_the_host_are_refused(binding):
    """There is no CPU path: the wrappers raise before anything is enqueued."""
    import torch

    kv = binding.PagedKV(4, 16, 2, 64, table_width=2, device="cpu")
    q, starts = torch.zeros(1, 2, 64, dtype=torch.bfloat16), torch.tensor([0, 1], dtype=torch.int32)
    for call in (lambda: kv.attend(q, starts, 1), lambda: kv.append(q, q, starts, starts[1:]), lambda: kv.evict(4, 0, 0)):
        with pytest.raises((RuntimeError, ValueError, AssertionError)):
            call()
    p, i = torch.ones(1, 2, 8), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises((RuntimeError, ValueError, AssertionError)):
        binding.tree_verify(p, i, i, torch.zeros(1, 2), i.clone(), i[0].clone(), i[0].clone())


def test_the_reference_keeps_the_targets_distribution():
    """What the rule is for: over the drawn drafts and uniform numbers, the first token that comes out has the target's
    distribution.  Exact: the sum over the drafts, with the chance of each acceptance, and over the token that follows."""
    import torch

    from tests.serve_reference import verify

    V, g = 4, torch.Generator().manual_seed(1)
    target, draft = [torch.softmax(torch.randn(1, 3, V, generator=g, dtype=torch.float64), dim=2) for _ in "td"]
    parents = torch.tensor([[-1, -1]], dtype=torch.int32)
    P, Q = target[0, 0], draft[0, 0]
    got = torch.zeros(V, dtype=torch.float64)
    # the numbers at which the outcome changes are found by halving: the rule is asked, not repeated
    def border(ask):
        lo, hi = 0.0, 1.0
        for _ in range(50):
            mid = (lo + hi) / 2
            lo, hi = (mid, hi) if ask(mid) else (lo, mid)
        return lo
    for x in range(V):
        for y in range(V):
            tokens, chance = torch.tensor([[x, y]], dtype=torch.int32), float(Q[x] * Q[y])
            run = lambda a, b, c: verify(target, draft, tokens, parents, torch.tensor([[a, b, c]], dtype=torch.float64))  # noqa: B023,E731
            first = border(lambda u: int(run(u, 1.0, 0.5)[0][0, 0]) == 0)
            got[x] += chance * first
            second = border(lambda u: int(run(1.0, u, 0.5)[0][0, 0]) == 1) if first < 1.0 - 1e-9 else 0.0
            got[y] += chance * (1 - first) * second
            rest = chance * (1 - first) * (1 - second)
            if rest > 1e-12:
                ends = [border(lambda u, z=z: int(run(1.0, 1.0, u)[2][0]) <= z) for z in range(V)]
                for z in range(V):
                    got[z] += rest * (ends[z] - (ends[z - 1] if z else 0.0))
    assert bool((got - P).abs().max() < 1e-9)


def test_host_side_under_asan_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    csrc, san = os.path.join(ROOT, "paper_2501_04987_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize")
    exe = str(tmp_path / "serve_san")
    cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
           "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(csrc, "treekv_serve.hip"), "-x", "hip", os.path.join(san, "serve_driver.cpp"), "-o", exe]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env)
    assert res.returncode == 0 and "serve paths clean" in res.stdout, res.stdout
