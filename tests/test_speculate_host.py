"""Argument checks of the speculative-decoding entry points that need no GPU: every call here returns before anything is
enqueued.  And the same host code under AddressSanitizer and UBSan."""
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


def context(binding, bound=False, **kw):
    base = dict(budget=64, q_heads=4, kv_heads=2, head_dim=128, batch=3, dtype=binding.TREEKV_BF16, n_sink=2, n_recent=20)
    cfg = binding.treekv_config(**{**base, **kw})
    h = C.c_void_p()
    assert binding.load().treekv_init_ex(C.byref(h), C.byref(cfg)) == 0
    if bound:                                              # an address is enough: nothing here gets as far as using it
        assert binding.load().treekv_bind_workspace(h, 0x100000 * bound, 1 << 40) == 0
    return h


def test_tree_calls(binding):
    lib, ok, off = binding.load(), 0x1000, 0x1008
    EINVAL, ENOWS = binding.TREEKV_EINVAL, binding.TREEKV_ENOWS
    h = context(binding, max_chunk=100)
    assert lib.treekv_tree_scratch_bytes(None, 4) == 0
    need = lib.treekv_tree_scratch_bytes(h, 4)
    assert all(lib.treekv_tree_scratch_bytes(h, n) == 0 for n in (-1, 0, 101, 257, 1 << 30))
    attend = [h, ok, ok, ok, ok, 4, ok, ok, ok, max(need, 1), None]
    assert lib.treekv_tree_attend(*attend) == ENOWS        # nothing else is wrong with it
    for i, bad in [(0, None), (1, None), (2, None), (3, None), (4, None), (6, None), (1, off), (2, off), (3, off), (6, off), (8, off),
                   (5, 0), (5, -1), (5, 101), (5, 257)]:
        assert lib.treekv_tree_attend(*[bad if j == i else x for j, x in enumerate(attend)]) == EINVAL, (i, bad)
    if need:
        assert lib.treekv_tree_attend(*attend[:9], need - 1, None) == EINVAL and lib.treekv_tree_attend(*attend[:8], None, need, None) == EINVAL
    commit = [h, ok, ok, ok, ok, ok, 4, ok, ok, 3, ok, ok, ok, ok, None]
    assert lib.treekv_tree_commit(*commit) == ENOWS
    for i, bad in [(0, None), (1, None), (2, None), (3, None), (4, None), (5, None), (7, None), (8, None), (10, None), (1, off), (2, off),
                   (3, off), (6, 0), (6, 101), (9, 0), (9, 5), (9, -1)]:
        assert lib.treekv_tree_commit(*[bad if j == i else x for j, x in enumerate(commit)]) == EINVAL, (i, bad)
    lib.treekv_destroy(h)


def test_scratch_holds_every_slice(binding):
    """What is asked for covers units x row tiles x slices of partial results, in 64 bits, and is 0 where there is one slice."""
    lib = binding.load()
    h = context(binding, budget=2048, q_heads=32, kv_heads=32, batch=16)
    assert lib.treekv_tree_scratch_bytes(h, 16) == 0
    lib.treekv_destroy(h)
    h = context(binding, budget=4096, q_heads=64, kv_heads=8, batch=1)
    sizes = [lib.treekv_tree_scratch_bytes(h, n) for n in (1, 16, 64, 256)]
    assert sizes[0] >= 8 * 2 * 8 * 132 * 4 and all(x % 256 == 0 for x in sizes)
    lib.treekv_destroy(h)


def test_fork(binding):
    lib = binding.load()
    a, b, unbound = context(binding, 1), context(binding, 2, batch=5, max_chunk=64, max_prompt=128, kv_splits=2), context(binding)
    ints = lambda *x: (C.c_int32 * max(len(x), 1))(*x)  # noqa: E731

    def fork(to, frm, src, dst, count=None):
        return lib.treekv_fork(to, frm, ints(*src), ints(*dst), len(src) if count is None else count, None)

    EINVAL = binding.TREEKV_EINVAL
    assert fork(a, unbound, [0], [0]) == binding.TREEKV_ENOWS and fork(unbound, a, [0], [0]) == binding.TREEKV_ENOWS
    assert fork(None, a, [0], [0]) == EINVAL and fork(a, None, [0], [0]) == EINVAL
    assert lib.treekv_fork(a, b, None, ints(0), 1, None) == EINVAL and lib.treekv_fork(a, b, ints(0), None, 1, None) == EINVAL
    assert fork(a, b, [0], [0], 0) == EINVAL and fork(a, b, [0] * 4, [0, 1, 2, 3]) == EINVAL and fork(a, b, [0], [0], -1) == EINVAL
    for src, dst in (([5], [0]), ([-2], [0]), ([0], [3]), ([0], [-1]), ([0, 1], [2, 2]), ([2 ** 31 - 1], [0])):
        assert fork(a, b, src, dst) == EINVAL, (src, dst)
    assert fork(a, a, [0, 1], [1, 2]) == EINVAL            # 1 is read for 2 and written
    for kw in (dict(budget=65), dict(q_heads=2), dict(kv_heads=4), dict(head_dim=64), dict(dtype=1), dict(n_sink=1), dict(n_recent=19),
               dict(softmax_scale=1.0), dict(flags=1), dict(flags=8), dict(rope_base=5.0)):
        other = context(binding, 2, **kw)
        assert fork(a, other, [0], [0]) == EINVAL, kw
        lib.treekv_destroy(other)
    same = context(binding, 1, batch=2)                    # two batches over one workspace: not one state
    assert fork(a, same, [0], [1]) == EINVAL
    for x in (a, b, unbound, same):
        lib.treekv_destroy(x)


def test_qkv_prepare(binding):
    lib, EINVAL, EUN = binding.load(), binding.TREEKV_EINVAL, binding.TREEKV_EUNSUPPORTED
    good = dict(q=0x10000, k=0x20000, v=0x30000, q_out=0x40000, k_out=0x50000, v_out=0x60000, q_stride=512, k_stride=512, v_stride=512,
                tokens=4, q_heads=4, kv_heads=2, head_dim=128, dtype=0, rotary_dim=64, flags=0, eps=1e-6, positions=0x70000,
                inv_freq=0x71000, q_weight=0x72000, k_weight=0x73000)
    call = lambda **kw: lib.treekv_qkv_prepare(C.byref(binding.treekv_qkv_args(**{**good, **kw})), None)  # noqa: E731
    assert lib.treekv_qkv_prepare(None, None) == EINVAL
    for kw in (dict(tokens=0), dict(tokens=-1), dict(dtype=2), dict(q=None), dict(q_out=None), dict(k=None), dict(v_out=None), dict(q_heads=0),
               dict(kv_heads=0), dict(flags=2), dict(flags=4), dict(positions=None), dict(inv_freq=None), dict(rotary_dim=-16),
               dict(rotary_dim=144), dict(rotary_dim=0), dict(eps=-1.0), dict(eps=float("nan")), dict(q=0x10008), dict(k_out=0x50004),
               dict(q_weight=0x72002), dict(k_weight=0x73008), dict(q_stride=504), dict(q_stride=516), dict(k_stride=-512), dict(v_stride=1 << 62),
               dict(q=None, q_out=None), dict(q=None, q_out=None, k=None, k_out=None, v=None, v_out=None),
               dict(k_out=0x40000 + 4 * 512 * 2 - 16), dict(q_out=0x20000), dict(q_out=0x10010), dict(q_out=0x10000, q_stride=768),
               dict(v_out=0x10000 + 3 * 1024), dict(q_out=0x70000), dict(k_out=0x71000), dict(v_out=0x72000), dict(q_out=0x73010)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(head_dim=96), dict(head_dim=256, rotary_dim=256, q_stride=1024), dict(rotary_dim=20), dict(rotary_dim=8)):
        assert call(**kw) == EUN, kw


def test_binding_refuses_wrong_tensors(binding):
    import torch

    x = torch.zeros(3, 2, 64)
    for args, kw in (((), dict(q=None)), ((x, x[:, :, :32]), {}), ((x, x.bfloat16()), {}), ((x, x[:2]), {}), ((x, x, x[:, :1]), {}),
                     ((x.transpose(0, 1),), {}), ((torch.zeros(3, 2, 128)[..., ::2],), {}), ((x,), dict(positions=torch.zeros(3).int())),
                     ((x,), dict(positions=torch.zeros(3), inv_freq=binding.rope_frequencies(64, device="cpu"))),
                     ((x,), dict(positions=torch.zeros(3).int(), inv_freq=torch.zeros(32))), ((x,), dict(q_weight=torch.zeros(32))),
                     ((x,), dict(out=(torch.zeros(3, 2, 32), None, None)))):
        with pytest.raises(ValueError):
            binding.qkv_prepare(*args, **kw)


def test_host_side_under_asan_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    exe, san = str(tmp_path / "speculate_san"), os.path.join(ROOT, "tests", "sanitize")
    csrc = os.path.join(ROOT, "paper_2501_04987_amd", "csrc")
    cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "treekv_host.hip"), os.path.join(csrc, "treekv_speculate.hip"),
           "-x", "hip", os.path.join(san, "host_stubs.cpp"), os.path.join(san, "speculate_driver.cpp"), "-o", exe]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env)
    assert res.returncode == 0 and "speculate paths clean" in res.stdout, res.stdout
