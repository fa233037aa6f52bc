"""The check of drafted tokens on the GPU over rows of few weights, as samplers that cut their probabilities leave them."""
import random

import pytest
import torch

from tests.test_verify_kernels_cpu import _fits, _sparse, _uniforms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2103_05288_amd import Context
    c = Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def _draw(ctx, rows, uniforms, left_of_a_draft):
    """The tokens drawn from rows [B, V]: as the target behind the last drafted token, or as what is left beside a draft whose token the
    target cannot have."""
    B, V = rows.shape
    h = ctx.register_verify("f32")
    drafts = 1 if left_of_a_draft else 0
    target, draft = rows[:, None], None
    u = torch.tensor(uniforms)[:, None]
    if left_of_a_draft:
        target, draft = torch.cat((target, torch.ones(B, 1, V)), 1), torch.zeros(B, 1, V)
        draft[:, 0, 77] = 1.0
        u = torch.cat((torch.full((B, 1), 0.75), u), 1)
    tokens = torch.full((B, drafts + 1), -9, dtype=torch.int32, device="cuda")
    accepted = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((h.workspace_bytes(B, V),), 255, dtype=torch.uint8, device="cuda")
    h.launch(target.contiguous().cuda(), torch.full((B, drafts), 77, dtype=torch.int32, device="cuda"), u.contiguous().cuda(), tokens, accepted,
             draft=None if draft is None else draft.cuda(), workspace=ws)
    assert accepted.tolist() == [0] * B and (tokens[:, 1:] == -1).all()
    return tokens[:, 0].tolist()


@pytest.mark.parametrize("left_of_a_draft", [False, True])
@pytest.mark.parametrize("V", [20480, 131072])
def test_verify_of_rows_of_few_weights(ctx, V, left_of_a_draft):
    g = random.Random(V)
    rows = [torch.zeros(V)]
    rows[0][0] = rows[0][4096] = 2.0 ** -54               # (the third chunk is empty, and its running sum a rounding above the second's)
    rows[0][8192] = rows[0][16384] = 0.5
    uniforms = [0.5]
    for _ in range(150):
        rows.append(_sparse(g, V, g.choice((2, 3, 4, 5, 8, 20))))
        rows[-1][77] = 0
        uniforms += _uniforms(g, rows[-1], 1)
    rows = torch.stack(rows)
    for row, u, t in zip(rows, uniforms, _draw(ctx, rows, uniforms, left_of_a_draft)):
        _fits(row, u, t)


def test_verify_with_a_last_uniform_of_one(ctx):
    g = torch.Generator().manual_seed(4)
    rows = torch.zeros(100, 32000)
    rows[:, :30000] = torch.softmax(2 * torch.randn(100, 30000, generator=g), -1)
    for row, t in zip(rows, _draw(ctx, rows, [1.0] * 100, False)):
        _fits(row, 1.0, t)


@pytest.mark.parametrize("V", [300001, 1000000])
def test_verify_of_several_chunks_a_lane_at_their_ends(ctx, V):
    """Vocabularies of more than 64 chunks: rows of few weights and dense ones, uniforms on the running sums and 1."""
    g = random.Random(V)
    rows, uniforms = [], []
    for i in range(24):
        rows.append(_sparse(g, V, g.choice((2, 5, 20, 60))))
        uniforms += [1.0] if i % 3 == 0 else _uniforms(g, rows[-1], 1)
    for first in (0, V // 2):
        rows.append(torch.zeros(V))
        rows[-1][first:V - 5000:701] = 0.25 + torch.rand(len(range(first, V - 5000, 701)), generator=torch.Generator().manual_seed(first))
        uniforms.append(1.0)
    rows = torch.stack(rows)
    for row, u, t in zip(rows, uniforms, _draw(ctx, rows, uniforms, False)):
        _fits(row, u, t)
