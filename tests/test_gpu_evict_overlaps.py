"""dl_kv_evict into what it reads: refused, also where only a part is the same memory."""

import pytest
import torch

import paper_2511_06605_amd as dl

from test_gpu_decode_refusals import cache, refused

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    torch.cuda.set_device(0)
    dl.dl_init(0)
    yield
    dl.dl_shutdown()


BATCH, KEEP = 4, 3


def evict(room, lens, kept, kept_lens):
    """Lists of int32 at these places of room."""
    at = lambda place, n: room[place:place + n]  # noqa: E731
    r = dl.KvEvict(cache(), torch.ones((BATCH, 32), device="cuda"), torch.zeros((BATCH, 2), dtype=torch.int32, device="cuda"), at(lens, BATCH),
                   torch.arange(BATCH, dtype=torch.int32, device="cuda").view(BATCH, 1), at(kept, BATCH * KEEP).view(BATCH, KEEP), at(kept_lens, BATCH))
    r.use_workspace(torch.zeros(dl.dl_kv_evict_workspace(r), dtype=torch.uint8, device="cuda"))
    return r


@pytest.mark.parametrize("lens,kept,kept_lens", [
    (20, 0, 20), (20, 0, 21), (20, 0, 23), (20, 0, 17),     # lengths into lengths
    (20, 20, 40), (20, 23, 40), (20, 9, 40), (20, 14, 40),  # tokens into lengths
    (40, 0, 0), (40, 0, 11), (40, 3, 0)])                   # lengths into tokens
def test_refused(lens, kept, kept_lens):
    room = torch.zeros(60, dtype=torch.int32, device="cuda")
    refused(dl.dl_kv_evict, evict(room, lens, kept, kept_lens))
    assert not room.any()


@pytest.mark.parametrize("lens,kept,kept_lens", [(20, 0, 24), (20, 0, 16), (20, 24, 40), (20, 8, 40), (40, 0, 12), (40, 4, 0)])
def test_next_to_each_other(lens, kept, kept_lens):
    room = torch.full((60,), 7, dtype=torch.int32, device="cuda")
    room[lens:lens + BATCH] = torch.tensor([0, 2, 3, 0], dtype=torch.int32)
    want = room.clone()
    want[kept:kept + BATCH * KEEP] = torch.tensor([-1, -1, -1, 0, 1, -1, 0, 1, 2, -1, -1, -1], dtype=torch.int32)
    want[kept_lens:kept_lens + BATCH] = torch.tensor([0, 2, 3, 0], dtype=torch.int32)
    dl.dl_kv_evict(evict(room, lens, kept, kept_lens), torch.cuda.current_stream())
    assert torch.equal(room, want)


def test_no_tokens_overlap_nothing():
    """keep == 0: nothing is written to kept, wherever it points."""
    room = torch.full((60,), 7, dtype=torch.int32, device="cuda")
    r = evict(room, 20, 0, 40)
    r.desc.keep = 0
    for at in (20, 21, 40, 43):
        r.desc.kept = room.data_ptr() + 4 * at
        room[40:44] = 7
        dl.dl_kv_evict(r, torch.cuda.current_stream())
        assert room.tolist() == [7] * 40 + [0] * 4 + [7] * 16
