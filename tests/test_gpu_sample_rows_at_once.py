"""sample on more rows than go through its kernels at once, and in a workspace of just its size (MI355X)."""
import pytest
import torch

import paper_2502_00922_amd as hl
from test_gpu_sample import check, make

pytestmark = pytest.mark.gpu


def settings_of(rows):
    g = torch.Generator(device="cuda").manual_seed(5)
    pick = lambda values, dtype: torch.tensor(values, dtype=dtype, device="cuda")[  # noqa: E731
        torch.randint(0, len(values), (rows,), generator=g, device="cuda")]
    return dict(temperature=pick([0.0, 0.5, 1.0, 2.0], torch.float32), top_k=pick([0, 1, 10, 150, -3], torch.int32),
                top_p=pick([1.0, 0.9, 0.3, 0.0], torch.float32), min_p=pick([0.0, 0.05, 0.5], torch.float32))


@pytest.mark.parametrize("rows,vocab,dtype", [(4097, 200, torch.float32), (9000, 37, torch.bfloat16),
                                              (2050, 20001, torch.float16), (4096, 1, torch.float32)])
def test_more_rows(rows, vocab, dtype):
    x, u = make(rows, vocab, dtype)
    check(x, u, **settings_of(rows))


def test_more_rows_than_at_once_among_others():
    # rows of a wider tensor, one setting for all
    big, u = make(4200, 300)
    check(big[:, 7:291], u, top_k=40, top_p=0.9)


@pytest.mark.parametrize("rows,vocab", [(1, 5), (3, 40001), (4100, 33), (40, 131072)])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=3000, top_p=0.9), dict(top_k=20), dict(top_p=0.5)])
def test_workspace_of_just_its_size(rows, vocab, settings):
    x, u = make(rows, vocab)
    n = hl.lib().hl_sample_workspace_bytes(rows, vocab)
    room = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    want = hl.sample(x, u, **settings)
    for _ in range(2):  # what a call leaves there is no matter to the next
        got = hl.sample(x, u, workspace=room[:n], **settings)
        assert torch.equal(got.tokens, want.tokens) and torch.equal(got.logprobs, want.logprobs)
    assert (room[n:] == 0xA5).all()
    with pytest.raises(hl.HLError):
        hl.sample(x, u, workspace=room[:n - 1], **settings)
