"""drafts.verify at the borders of its range."""
import pytest
import torch

import test_gpu_drafts as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def drafts(gpu_lib):
    from paper_2509_25689_amd import drafts
    return drafts


@pytest.mark.parametrize("own_stream", [False, True])
@pytest.mark.parametrize("max_new", [257, 1 << 20, (1 << 31) - 1])
def test_max_new_is_refused_before_memory_is_taken(drafts, max_new, own_stream):
    """The largest of these would want 16 GiB of results for each of the 400 requests."""
    from paper_2509_25689_amd import moeq
    R = 400
    ints = torch.zeros(R, dtype=torch.int32, device="cuda")
    rows = torch.ones((R, 1), device="cuda")
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    with pytest.raises(moeq.MoeqError) as e:
        drafts.verify(ints, ints, torch.arange(R + 1, device="cuda").int(), rows, None, rows[:, 0].contiguous(), rows[:, 0].contiguous(),
                      max_new=max_new, stream=torch.cuda.current_stream().cuda_stream if own_stream else None)
    assert e.value.status == moeq.MOEQ_ERR_UNSUPPORTED
    assert torch.cuda.max_memory_allocated() - before < 1 << 20


@pytest.mark.parametrize("sampled", [False, True])
@pytest.mark.parametrize("shape", ["chain", "star"])
@pytest.mark.parametrize("V", [128000, 262145, 300001, 1 << 20])
def test_wide_vocabularies(drafts, sampled, shape, V):
    """More than 64 and up to 256 chunks of a row of probabilities; the last tokens fall from the first chunk to the last."""
    sizes = [4, 1, 2, 1, 3]
    tokens = []
    for seed, keep in ((21, 0.3), (22, 0.0)):
        w = base._world(seed, sizes, V, shape, sampled, keep=keep)
        if keep == 0.0:  # no draft is kept: the residual of all of them
            w["uniform"][:] = 1 - 2.0 ** -24
        w["last"][:] = torch.tensor([0.001, 0.3, 0.55, 0.8, 0.999])
        base._check(drafts, w)
        path, counts, out = base._run(drafts, base._cuda(w), 4)
        tokens += [out[r, c - 1].item() for r, c in enumerate(counts.tolist())]
    chunks = [t // 4096 for t in tokens]
    assert min(chunks) < 64 and max(chunks) >= (V // 4096) * 3 // 4


def test_wide_vocabulary_ends(drafts):
    """A probability in the last place alone, and in a place of each 64 chunks, at the largest vocabulary."""
    V = 1 << 20
    places = [0, 4095, 4096, 64 * 4096 - 1, 64 * 4096, 128 * 4096 + 5, 192 * 4096, V - 1]
    R = len(places)
    target = torch.zeros((R, V))
    target[torch.arange(R), torch.tensor(places)] = 1.0
    w = dict(tokens=torch.zeros(R, dtype=torch.int32), parents=torch.full((R,), -1, dtype=torch.int32), cu=torch.arange(R + 1).int(),
             target=target, draft=None, uniform=torch.zeros(R), last=torch.linspace(0, 0.999, R))
    assert base._check(drafts, w) == [1] * R
    assert base._run(drafts, base._cuda(w), 1)[2].flatten().tolist() == places
