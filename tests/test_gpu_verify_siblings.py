"""What verification emits is distributed as the target where siblings are what the call's documentation asks for."""
import pytest
import torch

from tests.test_gpu_verify import clean_status  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

P = torch.tensor([0.1, 0.4, 0.05, 0.25, 0.2])


def emitted(tokens, draft):
    """Counts of the first token behind the root, of as many walks as tokens has rows (three children of the root each)."""
    from paper_2511_06010_b200 import speculative

    R, gen = tokens.shape[0], torch.Generator().manual_seed(8)
    parents = torch.tensor([-1, 0, 0, 0], dtype=torch.int32).repeat(R).cuda()
    tok = torch.cat([torch.zeros(R, 1, dtype=torch.int32), tokens.int()], 1).reshape(-1).cuda()
    target = P.expand(4 * R, 5).contiguous().cuda()
    d = None if draft is None else draft.expand(4 * R, 5).contiguous().cuda()
    u, un = torch.rand(4 * R, generator=gen).cuda(), torch.rand(R, generator=gen).cuda()
    path, n_path, nxt = speculative.verify(target, tok, parents, u, un, draft_probs=d, max_nodes=4)
    first = torch.where(n_path > 1, tok.view(R, 4).gather(1, path[:, 1:2].long().clamp(min=0)).squeeze(1), nxt)
    return torch.bincount(first.long(), minlength=5).double().cpu()


def follows(count):
    n = count.sum()
    return bool(((count - n * P).abs() < 5 * (n * P * (1 - P)).sqrt()).all())  # five standard deviations


@pytest.mark.parametrize("picked", [[1, 3, 4], [0, 2, 1], [3, 3, 1]])
def test_picked_siblings_without_draft_probabilities(picked):
    assert follows(emitted(torch.tensor(picked).expand(40000, 3), None))


def test_siblings_drawn_independently():
    q = torch.tensor([0.3, 0.1, 0.3, 0.1, 0.2])
    tokens = torch.multinomial(q.expand(120000, 5), 1, generator=torch.Generator().manual_seed(9)).view(40000, 3)
    assert follows(emitted(tokens, q))
