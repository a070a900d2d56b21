"""`python -m paper_2210_10108_amd.propose`: what it trains and how it proposes, by its
arguments."""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


def command(monkeypatch, *args):
    from paper_2210_10108_amd import propose
    monkeypatch.setattr(sys, "argv", ["propose", *args])
    propose.main()


@pytest.fixture
def seen(monkeypatch):
    """What the command's parts were called with."""
    from paper_2210_10108_amd import propose
    calls = {}
    train, encode = propose.train, propose.ProposalBlock.encode

    def watched_train(block, views, steps, **kw):
        losses = train(block, views, steps, **kw)
        calls.update(block=block, max_norm=kw.get("max_norm"), losses=losses, views=views)
        return losses

    def watched_encode(self, *a, **kw):
        calls["bits"] = kw.get("bits", 16)
        return encode(self, *a, **kw)
    monkeypatch.setattr(propose, "train", watched_train)
    monkeypatch.setattr(propose.ProposalBlock, "encode", watched_encode)
    return calls


@pytest.mark.parametrize("args,image,max_norm,bits", [
    ([], False, None, 16), (["--bits", "8"], False, None, 8), (["--max-norm", "5"], False, 5.0, 16),
    (["--image"], True, 100.0, 8), (["--image", "--max-norm", "inf", "--bits", "16"], True, float("inf"), 16)], ids=str)
def test_command(seen, monkeypatch, capsys, args, image, max_norm, bits):
    command(monkeypatch, "--steps", "3", *args)
    out = capsys.readouterr().out
    assert out.count("step ") == 3 and "hypotheses: " in out and "proposals: " in out and "nan" not in out
    assert seen["block"].image is image and seen["max_norm"] == max_norm and seen["bits"] == bits


def test_command_without_arguments_is_the_block_with_one_position_a_patch(seen, monkeypatch, capsys):
    # the same parameters as training it by hand, and the proposals of its forward pass
    from paper_2210_10108_amd import propose
    command(monkeypatch, "--steps", "4")
    out = capsys.readouterr().out
    views = propose.Views("tiny_bump")
    block = propose.ProposalBlock(state_dim=views.state_dim)
    losses = propose.train(block, views, 4)
    assert losses == seen["losses"]
    assert all(torch.equal(v, seen["block"].master[k]) for k, v in block.master.items())
    poses, states, q_pos, k_pos, _, hyps, gt = views.batch(4, 64, 10 ** 6, block.dtype)
    y = block.forward(poses, states, q_pos, k_pos)
    r, t = propose.errors(propose.corrected(hyps, y[..., :6].double().cpu().numpy()), gt[:, None])
    assert f"proposals: {r:.2f} degrees, {t:.4f} from the true pose" in out
