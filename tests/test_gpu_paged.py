"""GPU: the paged cache (append, attend, evict) against its definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def paged(**kw):
    from tests.serve_reference import Paged

    return Paged(**kw)


def held(got, want, room):
    off = (got.double().cpu() - want).abs()
    off[got.cpu() == want] = 0.0                         # infinities of one sign
    assert bool((off <= room).all()), float((off / room.clamp(min=1e-300)).max())


def check_attend(kv, ref, *, weigh=False, sequences=None, **kw):
    import torch

    want = ref.attend(sequences=sequences)
    out = torch.full((ref.total, ref.hkv * ref.G, ref.d), 7.0, dtype=ref.t, device="cuda")
    lse = torch.full(out.shape[:2], 7.0, device="cuda")
    before = kv.weights.clone() if weigh else None
    kv.attend(kw.pop("q", ref.q.cuda()), ref.starts.cuda(), kw.pop("longest", max(max(ref.news), 1)), out, lse, weigh=weigh, **kw)
    rows = torch.ones(ref.total, dtype=torch.bool)
    for b in range(ref.B) if sequences is not None else ():
        if b not in sequences:
            rows[int(ref.starts[b]):int(ref.starts[b]) + ref.news[b]] = False
    held(out.cpu()[rows], want["out"][rows], want["room"][rows])
    held(lse.cpu()[rows], want["lse"][rows], want["lse_room"][rows])
    assert bool((out.cpu()[~rows] == 7.0).all()) and bool((lse.cpu()[~rows] == 7.0).all())
    if weigh:
        total = before.double().cpu() + want["gain"]
        held(kv.weights, total, want["gain_room"] + 2.0 ** -23 * total.abs())
    return out, lse


SHAPES = [
    dict(lens=[1], news=[1], page_size=16, kv_heads=1, group=1, d=64),
    dict(lens=[33], news=[1], page_size=16, kv_heads=2, group=4, d=128),
    dict(lens=[700, 5, 0, 129], news=[1, 1, 0, 1], page_size=32, kv_heads=2, group=7, d=128),
    dict(lens=[64, 17, 200], news=[64, 3, 0], page_size=16, kv_heads=2, group=3, d=64),
    dict(lens=[300, 211, 90], news=[70, 211, 1], page_size=64, kv_heads=1, group=8, d=128),
    dict(lens=[150], news=[150], page_size=256, kv_heads=2, group=1, d=128),
    dict(lens=[600, 31], news=[130, 31], page_size=16, kv_heads=1, group=2, d=64),
    dict(lens=[16, 32, 48, 1, 2, 3, 15, 17] * 9, news=[1, 2, 0, 1, 1, 3, 2, 1] * 9, page_size=16, kv_heads=1, group=2, d=64),
    dict(lens=[1300], news=[40], page_size=128, kv_heads=1, group=16, d=128, scale=0.3),
    dict(lens=[700, 90], news=[1, 1], page_size=16, kv_heads=2, group=3, d=64, scale=-0.2),
    dict(lens=[200, 333], news=[200, 50], page_size=32, kv_heads=2, group=4, d=64, scale=-0.2),
    dict(lens=[2900], news=[70], page_size=32, kv_heads=1, group=2, d=128),
    dict(lens=[90, 70], news=[20, 33], page_size=16, kv_heads=1, group=33, d=64),
    dict(lens=[60, 50], news=[3, 4], page_size=16, kv_heads=1, group=70, d=64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attend(binding, shape, dtype):
    ref = paged(**SHAPES[shape], dtype=dtype, seed=shape)
    kv = ref.on_gpu(binding)
    check_attend(kv, ref, weigh=True)
    check_attend(kv, ref, weigh=False)


# Each way to cut the columns: a row of over a hundred shares; shares made larger so that each is of one sequence; sequences that
# are more than the shares; sequences that share one; row tiles with larger shares.
CUTS = [
    dict(lens=[20000], news=[1], page_size=64, kv_heads=1, group=4, d=128),
    dict(lens=[17000, 300], news=[5, 1], page_size=64, kv_heads=1, group=3, d=64),
    dict(lens=[700, 130, 1000, 31, 512], news=[1, 2, 1, 1, 1], page_size=16, kv_heads=32, group=1, d=64),
    dict(lens=[300, 31, 250, 0, 170, 200, 64], news=[1, 1, 1, 0, 1, 1, 1], page_size=32, kv_heads=64, group=2, d=64),
    dict(lens=[150] * 70, news=[1] * 70, page_size=32, kv_heads=2, group=2, d=128),
    dict(lens=[1501, 950], news=[1, 2], page_size=32, kv_heads=128, group=1, d=64),
    dict(lens=[2600], news=[130], page_size=32, kv_heads=32, group=1, d=64),
    dict(lens=[900, 40, 333, 17], news=[5, 1, 8, 0], page_size=16, kv_heads=2, group=4, d=128),
    dict(lens=[2300, 3], news=[3, 1], page_size=16, kv_heads=1, group=7, d=64),
]


# Chunks among sequences of a token or two.
MIXES = [
    dict(lens=[700, 300, 40, 1, 513, 90, 77, 133], news=[200, 1, 2, 0, 1, 9, 1, 8], page_size=16, kv_heads=2, group=2, d=128),
    dict(lens=[5, 1, 1500, 260, 31, 2, 900, 64, 17], news=[1, 1, 1, 100, 2, 2, 1, 1, 0], page_size=32, kv_heads=1, group=16, d=64),
    dict(lens=[90, 70, 80, 0, 0, 0, 0, 0, 0], news=[70, 17, 9, 0, 0, 0, 0, 0, 0], page_size=64, kv_heads=3, group=1, d=64),
    dict(lens=[400] * 70, news=[1] * 35 + [130] + [1] * 34, page_size=32, kv_heads=1, group=4, d=64),
    dict(lens=[160, 300, 33, 20, 9], news=[80, 1, 1, 3, 2], page_size=16, kv_heads=1, group=17, d=64),
]


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("mix", range(len(MIXES)))
def test_chunks_among_single_tokens(binding, mix, weigh):
    ref = paged(**MIXES[mix], seed=mix)
    check_attend(ref.on_gpu(binding), ref, weigh=weigh)


@pytest.mark.parametrize("lens,news,hkv,group,d", [([900, 400], [600, 400], 1, 2, 128), ([700, 40, 300], [699, 1, 300], 2, 3, 64),
                                                   ([1300], [1300], 1, 1, 64), ([260, 0, 300], [257, 0, 0], 1, 64, 64)])
def test_weights_of_many_rows_over_few_columns(binding, lens, news, hkv, group, d):
    """The rows of a column are summed in parts; what is in a page given up, and behind the last token, stays."""
    import torch

    ref = paged(lens=lens, news=news, page_size=32, kv_heads=hkv, group=group, d=d, seed=23)
    ref.table[0, 2] = -1
    kv = ref.on_gpu(binding)
    before = kv.weights.clone()
    check_attend(kv, ref, weigh=True)
    for b, n in enumerate(lens):
        assert torch.equal(kv.weights[b, :, n if news[b] else 0:], before[b, :, n if news[b] else 0:])
    assert torch.equal(kv.weights[0, :, 64:96], before[0, :, 64:96])
    again = ref.on_gpu(binding)
    again.attend(ref.q.cuda(), ref.starts.cuda(), max(news), weigh=True)
    assert torch.equal(again.weights, kv.weights)


@pytest.mark.parametrize("weigh,dtype", [(False, "bf16"), (True, "bf16"), (True, "f32")])
@pytest.mark.parametrize("cut", range(len(CUTS)))
def test_columns_cut_into_shares(binding, cut, weigh, dtype):
    ref = paged(**CUTS[cut], seed=cut, dtype=dtype)
    check_attend(ref.on_gpu(binding), ref, weigh=weigh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_queries_far_apart(binding, dtype):
    """Tokens 16 MB apart: their places in a tile pass 32 bits."""
    import torch

    ref = paged(lens=[90], news=[70], page_size=16, kv_heads=1, group=2, d=64, dtype=dtype, seed=3)
    wide = torch.empty(70, 1 << 24, dtype=ref.t, device="cuda")
    wide[:, :128] = ref.q.view(70, 128).cuda()
    check_attend(ref.on_gpu(binding), ref, q=wide[:, :128].unflatten(1, (2, 64)), weigh=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_strided_queries_and_an_untracked_cache(binding, dtype):
    import torch

    ref = paged(lens=[90, 40], news=[20, 3], page_size=16, kv_heads=2, group=2, d=64, dtype=dtype, tracked=False)
    kv = ref.on_gpu(binding)
    packed = torch.zeros(ref.total, 8, 64, dtype=ref.t, device="cuda")
    packed[:, 2:6] = ref.q.cuda()
    check_attend(kv, ref, q=packed[:, 2:6])
    with pytest.raises(binding.TreeKVError):
        kv.attend(ref.q.cuda(), ref.starts.cuda(), 20, weigh=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1], [14, 9, 16], [30, 45, 80]])
def test_attend_pages_given_up(binding, news, dtype):
    """Pages that are -1 or beyond the pool, also all of a sequence's: its rows are 0, their log sums minus infinity."""
    ref = paged(lens=[120, 100, 80], news=news, page_size=16, kv_heads=2, group=2, d=128, dtype=dtype, seed=3)
    ref.table[0, 1] = -1
    ref.table[0, 4] = ref.pages
    ref.table[0, 6] = -2147483648
    ref.table[1, :] = 2147483647
    out, lse = check_attend(ref.on_gpu(binding), ref, weigh=True)
    lo, hi = int(ref.starts[1]), int(ref.starts[2])
    assert not bool(out[lo:hi].any()) and bool((lse[lo:hi] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,group", [(1, 4), (6, 4), (40, 1), (150, 2)])
def test_what_is_not_attended_has_no_part(binding, new, group, dtype):
    """Infinities and NaNs behind the last token, in pages of nobody and in the chunk's later tokens: the rows before them come
    out bit for bit as without them, the rows that attend them are infinite or NaN where the formula is."""
    import torch

    ref = paged(lens=[201], news=[new], page_size=16, kv_heads=1, group=group, d=64, dtype=dtype, seed=5)
    kv = ref.on_gpu(binding)
    out0, lse0 = check_attend(kv, ref)
    used = torch.zeros(ref.pages, ref.ps, dtype=torch.bool)
    for s in range(201):
        page, r = ref.row(0, s)
        used[page, r] = True
    for pool, bad in ((kv.k, math.nan), (kv.v, math.inf)):
        pool.copy_(torch.where(used[:, None, :, None].cuda(), pool, torch.full((), bad, dtype=ref.t, device="cuda")))
    out, lse = kv.attend(ref.q.cuda(), ref.starts.cuda(), new), None
    assert torch.equal(out, out0)
    if new == 1:
        return
    for i, name, bad in ((new - 1, "k", math.nan), (new // 2, "v", math.inf), (new // 3, "v", math.nan), (0, "v", -math.inf)):
        kv2 = ref.on_gpu(binding)
        page, r = ref.row(0, 201 - new + i)
        getattr(kv2, name)[page, 0, r, 5] = bad
        lse = torch.empty_like(lse0)
        out = kv2.attend(ref.q.cuda(), ref.starts.cuda(), new, None, lse)
        assert torch.equal(out[:i], out0[:i]) and torch.equal(lse[:i], lse0[:i])
        got = out[i:].float()
        if name == "k":
            assert bool(got.isnan().all()) and bool(lse[i:].isnan().all())
        else:
            same = got[..., 5].isnan() if math.isnan(bad) else got[..., 5] == bad
            assert bool(same.all()) and bool(got[..., :5].isfinite().all()) and torch.equal(lse[i:], lse0[i:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 12, 20, 200])
@pytest.mark.parametrize("power", [22, 40])
def test_logits_of_any_size(binding, power, new, dtype):
    """Queries scaled by 2^22 and 2^40: one token has all of the weight, exactly, whatever its logit's last bits are."""
    import torch

    ref = paged(lens=[333], news=[new], page_size=16, kv_heads=1, group=2, d=64, dtype=dtype, seed=7)
    q = (ref.q.double() * 2.0 ** power).to(ref.t)
    kv = ref.on_gpu(binding)
    before = kv.weights.clone()
    lse = torch.empty(new, 2, device="cuda")
    out = kv.attend(q.cuda(), ref.starts.cuda(), new, None, lse, weigh=True).cpu()
    K, V = [ref.tokens(pool, 0, 0, 333)[0] for pool in (ref.k, ref.v)]
    s = (q.double() @ K.T) * ref.scale
    s = s.masked_fill(torch.arange(333) > (333 - new + torch.arange(new))[:, None, None], -math.inf)
    two = s.topk(2, dim=2).values
    sure = two[..., 0] - two[..., 1] > 2.0 ** -16 * two[..., 0].abs()       # no near tie: d + 8 roundings of 2^-24 of the terms' size
    top = s.argmax(dim=2)
    assert int(sure.sum()) > 0.9 * sure.numel()
    assert torch.equal(out[sure], V.to(ref.t)[top][sure])
    assert bool(((lse.cpu().double() - two[..., 0]).abs() <= 2.0 ** -16 * two[..., 0].abs())[sure].all())
    gain = (kv.weights - before)[0, 0, :333].cpu().double()
    want = torch.zeros(333, dtype=torch.float64)
    for t in top[sure].tolist():
        want[t] += 1
    doubt = int((~sure).sum())
    # (the weights began below 1: a gain is good to the roundings of sums up to 2 * new)
    room = (2 * new + 2) ** 2 * 2.0 ** -24
    assert bool((gain >= want - room).all()) and bool((gain <= want + doubt + room).all()) and abs(float(gain.sum()) - 2 * new) < 333 * room


@pytest.mark.parametrize("new", [1, 12, 20, 200])
@pytest.mark.parametrize("power", [0, 40])
def test_equal_tokens_share_the_weight(binding, power, new):
    """Three tokens with one key: their weights gain the same, bit for bit, of queries of any size; all together the rows' number."""
    import torch

    ref = paged(lens=[400], news=[new], page_size=16, kv_heads=1, group=2, d=64, seed=17)
    at = [ref.row(0, s) for s in (3, 77, 150)]
    for page, r in at:
        ref.k[page, 0, r] = 3 * ref.k[at[0][0], 0, at[0][1]] if (page, r) == at[0] else ref.k[at[0][0], 0, at[0][1]]
    kv = ref.on_gpu(binding)
    kv.weights.zero_()
    kv.attend((ref.q.double() * 2.0 ** power).to(ref.t).cuda(), ref.starts.cuda(), new, weigh=True)
    gain = kv.weights[0, 0].cpu()
    assert gain[3] == gain[77] == gain[150] and gain[3] > 0
    assert abs(float(gain.double().sum()) - 2 * new) < 2 * new * (2 * new + 464) * 2.0 ** -24 * 4


def test_weights_take_no_nan(binding):
    import torch

    ref = paged(lens=[50], news=[6], page_size=16, kv_heads=1, group=2, d=64, seed=6)
    q = ref.q.clone()
    q[2, 1, 3] = math.nan
    kv = ref.on_gpu(binding)
    before = kv.weights.clone()
    kv.attend(q.cuda(), ref.starts.cuda(), 6, weigh=True)
    gain = (kv.weights - before)[0, 0, :50].cpu().double()
    want = ref.attend()
    assert bool(gain.isfinite().all())
    # eleven of the twelve rows
    assert abs(float(gain.sum()) - 11.0) < 11 * 2.0 ** -10
    assert bool((gain <= want["gain"][0, 0, :50] + want["gain_room"][0, 0, :50] + 2.0 ** -23 * 8).all())


def test_refused_sequences_are_left_alone(binding):
    import torch

    ref = paged(lens=[40, 30, 60, 25], news=[5, 4, 7, 3], page_size=16, kv_heads=2, group=2, d=64, width=4, seed=8)
    kv = ref.on_gpu(binding)
    status = torch.full((4,), 9, dtype=torch.int32, device="cuda")

    def run(sequences, **kw):
        held_weights = kv.weights.clone()
        check_attend(kv, ref, weigh=True, sequences=sequences, status=status, **kw)
        for b in range(4):
            if b not in sequences:
                assert torch.equal(kv.weights[b], held_weights[b])
        assert status.tolist() == [0 if b in sequences else binding.TREEKV_EINVAL for b in range(4)]

    run([0, 1, 2, 3])
    run([0, 1, 3], longest=6)                              # the third has seven
    for b, bad in ((0, 65), (1, 3), (2, -1), (3, 2147483647)):
        kv.lens.copy_(ref.lens)
        kv.lens[b] = bad
        run([x for x in range(4) if x != b])
    kv.lens.copy_(ref.lens)
    starts = ref.starts.clone()
    for b, bad in ((0, -1), (4, 100), (4, 3)):
        odd = starts.clone()
        odd[b] = bad
        sequence = 0 if b == 0 else 3
        out = torch.full_like(ref.q, 7.0, device="cuda")
        kv.attend(ref.q.cuda(), odd.cuda(), 7, out, status=status)
        assert status.tolist() == [binding.TREEKV_EINVAL if x == sequence else 0 for x in range(4)]
        lo, hi = int(starts[sequence]), int(starts[sequence + 1])
        assert bool((out[lo:hi] == 7.0).all())


def test_rows_behind_the_last_sequence_stay(binding):
    import torch

    ref = paged(lens=[40, 30], news=[5, 4], page_size=16, kv_heads=1, group=2, d=64, seed=9)
    kv = ref.on_gpu(binding)
    q = torch.cat([ref.q, ref.q[:3]]).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    kv.attend(q, ref.starts.cuda(), 5, out, lse, weigh=True)
    want = ref.attend()
    held(out[:9], want["out"], want["room"])
    assert bool((out[9:] == 7.0).all()) and bool((lse[9:] == 7.0).all())
    k = torch.randn(12, 1, 64, device="cuda").to(ref.t)
    pool = kv.k.clone()
    kv.append(k, k, ref.starts.cuda(), torch.arange(12, dtype=torch.int32, device="cuda"))
    ref.append(k.cpu(), k.cpu(), torch.arange(12, dtype=torch.int32))
    assert torch.equal(kv.k.cpu(), ref.k) and not torch.equal(kv.k, pool)


def test_a_prefix_that_sequences_share(binding):
    import torch

    ref = paged(lens=[100, 100, 70], news=[3, 1, 2], page_size=16, kv_heads=2, group=2, d=64, seed=10)
    for b in (1, 2):
        ref.table[b, :4] = ref.table[0, :4]
    check_attend(ref.on_gpu(binding), ref, weigh=True)
    assert len(set(torch.unique(ref.table[:, :4]).tolist())) == 4


def test_far_pages(binding):
    """Rows more than 2^32 bytes into the pool, and into the weights."""
    import torch

    ref = paged(lens=[90, 35], news=[20, 1], page_size=16, kv_heads=2, group=2, d=128, seed=11)
    far = 600_000                                            # pages of 8192 bytes: 4.9 GB
    kv = binding.PagedKV(far + ref.pages, 16, 4, 128, kv_heads=2, batch=2, table_width=ref.width, tracked=True)
    kv.k[far:].copy_(ref.k)
    kv.v[far:].copy_(ref.v)
    kv.table.copy_(torch.where(ref.table >= 0, ref.table + far, ref.table))
    kv.lens.copy_(ref.lens)
    kv.weights.copy_(ref.weights)
    kv.positions.copy_(ref.positions)
    check_attend(kv, ref, weigh=True)
    rows = torch.randn(21, 2, 128).to(ref.t)
    kv.append(rows.cuda(), rows.cuda(), ref.starts.cuda(), torch.arange(21, dtype=torch.int32, device="cuda"))
    ref.append(rows, rows, torch.arange(21, dtype=torch.int32))
    ref.weights.copy_(kv.weights)
    kv.evict(30, 2, 10)
    ref.evict(30, 2, 10)
    assert torch.equal(kv.k[far:].cpu(), ref.k) and torch.equal(kv.v[far:].cpu(), ref.v) and torch.equal(kv.lens.cpu(), ref.lens)
    assert torch.equal(kv.weights.cpu(), ref.weights) and torch.equal(kv.positions.cpu(), ref.positions)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,news,hkv,d,ps", [([1], [1], 1, 64, 16), ([40, 33, 9], [40, 0, 9], 3, 64, 16), ([500, 20], [70, 20], 2, 128, 64),
                                                 ([1500] * 3, [1500, 1000, 700], 2, 64, 128)])
def test_append(binding, lens, news, hkv, d, ps, dtype):
    import torch

    ref = paged(lens=lens, news=news, page_size=ps, kv_heads=hkv, group=2, d=d, dtype=dtype, seed=12)
    if len(lens) > 1:
        ref.table[0, 1] = -1                                  # nothing is written there
    kv = ref.on_gpu(binding)
    packed = torch.randn(ref.total, 2 * hkv + 1, d, generator=ref.g).to(ref.t)
    k, v, positions = packed[:, :hkv], packed[:, hkv:2 * hkv], torch.randint(0, 1 << 30, (ref.total,), generator=ref.g).int()
    dev, status = packed.cuda(), torch.full((ref.B,), 9, dtype=torch.int32, device="cuda")
    kv.append(dev[:, :hkv], dev[:, hkv:2 * hkv], ref.starts.cuda(), positions.cuda(), status)
    ref.append(k, v, positions)
    for name in ("k", "v", "weights", "positions"):
        assert torch.equal(getattr(kv, name).cpu(), getattr(ref, name)), name
    assert not bool(status.any())
    bad = kv.lens.clone()
    bad[0] = news[0] - 1
    kv.lens.copy_(bad)
    held_k = kv.k.clone()
    only = ref.starts.clone()
    only[1:] = only[1]                                        # the first sequence's rows alone
    kv.append(dev[:, :hkv] + 1, dev[:, hkv:2 * hkv], only.cuda(), positions.cuda(), status)
    assert torch.equal(kv.k, held_k) and status.tolist() == [binding.TREEKV_EINVAL] + [0] * (ref.B - 1)


def evicted(binding, ref, *args, kv=None, **kw):
    import torch

    kv = kv or ref.on_gpu(binding)
    kv.evict(*args, **kw)
    ref.evict(*args)
    for name in ("k", "v", "weights", "positions", "lens"):
        x, y = getattr(kv, name).cpu(), getattr(ref, name)
        assert torch.equal(torch.nan_to_num(x, nan=-7.0) if x.is_floating_point() else x,
                           torch.nan_to_num(y, nan=-7.0) if y.is_floating_point() else y), name
    return kv


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("lens,budget,sink,recent,ps", [
    ([17], 16, 0, 0, 16), ([100, 16, 17, 0], 16, 4, 8, 16), ([300, 299, 31], 1, 0, 1, 16), ([2100, 1025, 40], 1024, 4, 512, 64),
    ([5000], 33, 0, 0, 128), ([70, 90], 64, 60, 4, 32), ([50], 40, 0, 40, 16), ([9000, 700], 4500, 2, 3, 256), ([8192, 8193, 6000], 5000, 4, 100, 128), ([4096, 4097], 4000, 4, 2000, 64),
    ([16384, 16385], 300, 4, 100, 256), ([32768, 32769], 20000, 4, 10000, 256)])
def test_evict(binding, lens, budget, sink, recent, ps, dtype, d):
    ref = paged(lens=lens, news=[0] * len(lens), page_size=ps, kv_heads=2, group=1, d=d, dtype=dtype, seed=20)
    import torch

    # positions in any order, as earlier evictions leave them
    for b in range(ref.B):
        for h in range(2):
            ref.positions[b, h] = torch.randperm(ref.positions.shape[2], generator=ref.g).int()
    kv = evicted(binding, ref, budget, sink, recent)
    evicted(binding, ref, budget, sink, recent, kv=kv)        # nothing is left to do
    ref.lens += 1                                             # a decode step later, over what lay there
    ref.lens.clamp_(max=ref.width * ps)
    kv.lens.copy_(ref.lens)
    evicted(binding, ref, budget, sink, recent, kv=kv)


@pytest.mark.parametrize("case", ["equal", "zeros", "nans", "infinite", "negative", "few values", "one bit"])
@pytest.mark.parametrize("lens", [[1500, 900], [10000, 5000], [30000, 33000]])
def test_evict_order(binding, case, lens):
    import torch

    ref = paged(lens=lens, news=[0, 0], page_size=256, kv_heads=2, group=1, d=64, seed=21)
    w, g = ref.weights, ref.g
    if case == "equal":
        w.fill_(0.25)
    elif case == "zeros":
        w.copy_(torch.where(torch.rand(w.shape, generator=g) < 0.5, 0.0, -0.0))
    elif case == "nans":
        w[torch.rand(w.shape, generator=g) < 0.7] = math.nan
        w[0, 0, :200] = -math.inf
    elif case == "infinite":
        w[torch.rand(w.shape, generator=g) < 0.3] = math.inf
    elif case == "negative":
        w.sub_(0.5)
    elif case == "few values":
        w.copy_((w * 5).floor())
    else:
        w.copy_((torch.full(w.shape, 1.0).view(torch.int32) + torch.randint(0, 3, w.shape, generator=g).int()).view(torch.float32))
    evicted(binding, ref, 400, 4, 100)
    if lens[0] > 2000:
        evicted(binding, ref, 399, 4, 100)


def test_evict_leaves_sequences_with_pages_given_up(binding):
    import torch

    ref = paged(lens=[100, 100, 300, 100], news=[0] * 4, page_size=16, kv_heads=2, group=1, d=64, width=8, seed=22)
    ref.table[2] = torch.arange(8)
    ref.table[0, 3] = -1
    ref.table[1, 7] = ref.pages + 5                           # behind its last token: not asked for
    status = torch.full((4,), 9, dtype=torch.int32, device="cuda")
    kv = evicted(binding, ref, 20, 2, 8, status=status)
    assert status.tolist() == [binding.TREEKV_EINVAL, 0, binding.TREEKV_EINVAL, 0] and kv.lens.tolist() == [100, 20, 300, 20]
    evicted(binding, ref, 100000, 0, 0, kv=kv, status=status)        # more than there are slots
    assert status.tolist() == [0, 0, binding.TREEKV_EINVAL, 0]


def test_layers_that_share_lengths(binding):
    """Each layer is evicted by the lengths that all of them had; a refused sequence and a short one keep theirs."""
    import torch

    ref = paged(lens=[100, 15, 90], news=[0] * 3, page_size=16, kv_heads=2, group=1, d=64, seed=23)
    ref.table[2, 1] = -1
    one = ref.on_gpu(binding)
    lens = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    two = binding.PagedKV(ref.pages, 16, 2, 64, batch=3, table_width=ref.width, table=one.table, lens=one.lens)
    other = paged(lens=[100, 15, 90], news=[0] * 3, page_size=16, kv_heads=2, group=1, d=64, seed=24)
    other.table.copy_(ref.table)
    for name in ("k", "v", "weights", "positions"):
        getattr(two, name).copy_(getattr(other, name))
    for kv in (one, two):
        kv.evict(40, 2, 10, lens_out=lens)
        assert one.lens.tolist() == [100, 15, 90] and lens.tolist() == [40, 15, 90]
    for kv, r in ((one, ref), (two, other)):
        r.evict(40, 2, 10)
        for name in ("k", "v", "weights", "positions"):
            assert torch.equal(getattr(kv, name).cpu(), getattr(r, name)), name
    one.lens.copy_(lens)
    one.evict(30, 2, 10, lens_out=one.lens)                   # as without it
    assert one.lens.tolist() == [30, 15, 90]
    with pytest.raises(ValueError):
        one.evict(30, 2, 10, lens_out=lens[:2])


def test_calls_beside_each_other(binding):
    """One cache read by calls on two streams at once, each with its own scratch; two sequences of one table (beams)."""
    import torch

    ref = paged(lens=[700, 700, 300], news=[20, 20, 9], page_size=16, kv_heads=2, group=3, d=128, seed=25)
    ref.table[1] = ref.table[0]
    kv, q, starts = ref.on_gpu(binding), ref.q.cuda(), ref.starts.cuda()
    q[20:40] = q[:20]
    want = kv.attend(q, starts, 20)
    assert torch.equal(want[:20], want[20:40])
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(want) for _ in range(2)]
    scratch = [kv.new_attend_scratch(49, 20) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, x in zip(streams, outs, scratch):
            with torch.cuda.stream(s):
                kv.attend(q, starts, 20, o, scratch=x)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_results_repeat_bit_for_bit_on_other_streams(binding):
    import torch

    ref = paged(lens=[900, 300, 77], news=[9, 1, 30], page_size=32, kv_heads=2, group=4, d=128, seed=30)
    a, b = ref.on_gpu(binding), ref.on_gpu(binding)
    q, starts = ref.q.cuda(), ref.starts.cuda()
    x = a.attend(q, starts, 30, weigh=True)
    a.evict(64, 4, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = b.attend(q, starts, 30, weigh=True)
        b.evict(64, 4, 16)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(x, y)
    for name in ("k", "v", "weights", "positions", "lens"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_arguments(binding):
    import torch

    ref = paged(lens=[40, 30], news=[5, 4], page_size=16, kv_heads=2, group=2, d=64, seed=31)
    kv = ref.on_gpu(binding)
    q, starts = ref.q.cuda(), ref.starts.cuda()
    for call in (lambda: kv.attend(q.float(), starts, 5), lambda: kv.attend(q[:, :2], starts, 5), lambda: kv.attend(q, starts.cpu(), 5),
                 lambda: kv.attend(q, starts[:2], 5), lambda: kv.attend(q, starts.long(), 5), lambda: kv.attend(q.cpu(), starts, 5),
                 lambda: kv.attend(q, starts, 5, torch.empty(9, 4, 64, device="cuda")), lambda: kv.attend(q.transpose(1, 2), starts, 5),
                 lambda: kv.append(q[:, :2], q[:8, :2], starts, starts), lambda: kv.append(q[:, :3], q[:, :2], starts, starts),
                 lambda: kv.evict(20, 1, 1, status=starts)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: kv.attend(q, starts, 0), lambda: kv.attend(q, starts, 10), lambda: kv.evict(20, 11, 10), lambda: kv.evict(0, 0, 0),
                 lambda: kv.append(q[:, :2], q[:, 2:], starts), lambda: kv.attend(q, starts, 5, q)):
        with pytest.raises(binding.TreeKVError):
            call()
    with pytest.raises(AttributeError):
        kv.lens = ref.lens.cuda()
    kv.lens += 1                                              # its values may change
    assert kv.lens.tolist() == [41, 31]
