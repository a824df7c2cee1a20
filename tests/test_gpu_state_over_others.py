"""GPU: a snapshot or a compressed prompt that replaces a state whose rows all held infinities and NaNs finds nothing of them: it
goes on bit for bit as it does in a context that never held anything else."""
import pytest

from tests.test_gpu_fork_over_others import BUDGET, STREAMS, binding, chunk, follow, make, rows, spoil  # noqa: F401 (binding: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["steps", "chunks"])
@pytest.mark.parametrize("fed", [0, 1, 17, 40, 77])
@pytest.mark.parametrize("stream", STREAMS, ids=str)
def test_snapshot(binding, stream, fed, kind):  # noqa: F811
    kv, fresh = [make(binding, 2, *stream) for _ in range(2)]
    spoil(kv)
    if fed:
        chunk(fresh, rows(fresh, fed, 2))
    kv.import_state(fresh.export_state())
    follow(binding, kv, fresh, [(0, 0), (1, 1)], kind)


@pytest.mark.parametrize("kind", ["steps", "chunks"])
def test_refused_snapshot(binding, kind):  # noqa: F811
    """A unit whose snapshot does not pass is as after a reset."""
    import torch

    kv, fresh = [make(binding, 2, *STREAMS[0]) for _ in range(2)]
    spoil(kv)
    buf = fresh.export_state()
    buf[:16].view(torch.int32).copy_(torch.tensor([5, 4, 1, 0]))           # more tokens kept than seen: unit 0 of sequence 0
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    kv.import_state(buf, status)
    assert status.tolist() == [-1, 0, 0, 0]
    follow(binding, kv, fresh, [(0, 0), (1, 1)], kind)


@pytest.mark.parametrize("kind", ["steps", "chunks"])
@pytest.mark.parametrize("length", [4, 24, 40, 96])
@pytest.mark.parametrize("stream", STREAMS, ids=str)
def test_prompt(binding, stream, length, kind):  # noqa: F811
    import torch

    kv, fresh = [make(binding, 2, *stream) for _ in range(2)]
    spoil(kv)
    q, k, v = [x.expand(2, *x.shape).contiguous() for x in rows(kv, length, 3)]
    for c in (kv, fresh):
        ret = torch.empty(2, 2, BUDGET, dtype=torch.int32, device="cuda")
        c.prefill_prompt(q[:, -4:].contiguous(), k, v, length, 4, ret)
    follow(binding, kv, fresh, [(0, 0), (1, 1)], kind)
