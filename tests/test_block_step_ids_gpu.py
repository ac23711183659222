"""The training steps take token ids as they did when PyTorch looked the embeddings up: of either integer type, with any
stride."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2605_09825_b200 import api, block_step


@pytest.mark.parametrize("inner", [0, 272])
def test_ids_of_another_type_or_stride(inner):
    w = block_step.make_weights(128, 528, inner=inner)
    step = block_step.train_step_gated if inner else block_step.train_step
    ids = torch.arange(48, device="cuda") * 11 % 528
    want = step(w, ids, ids + 1)
    wide = torch.stack([ids, ids.flip(0)], 1)
    for other in (ids.int(), wide[:, 0], wide.int()[:, 0]):
        got = step(w, other, ids + 1)
        api.check()
        assert torch.equal(got[0], want[0])
        assert all(torch.equal(got[1][name], want[1][name]) for name in want[1])
