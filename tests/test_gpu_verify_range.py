"""drafts.verify at the borders of its range."""
import pytest
import torch

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
