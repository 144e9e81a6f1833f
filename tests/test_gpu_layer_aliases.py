"""Results that a caller may leave where an operand was."""
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [100, 5000, 70000])
@pytest.mark.parametrize("which", ["old", "ref", "advantage", "weights"])
def test_log_probabilities_in_place_of_an_input(vocab, which):
    """The row's inputs are read before its log probability is written: new ones may take the place of those that they are compared with."""
    import torch
    from paper_2508_15706_amd import binding as sl
    rows = 9
    g = torch.Generator(device="cuda").manual_seed(vocab)
    z = 2.0 * torch.randn(rows, vocab, device="cuda", generator=g)
    targets = torch.randint(vocab, (rows,), device="cuda", generator=g)
    targets[4] = -1
    now = ref.token_loss(z, targets, None)[1].float()
    given = {"old": now + 0.4 * torch.randn(rows, device="cuda", generator=g), "ref": now + 0.4 * torch.randn(rows, device="cuda", generator=g),
             "advantage": torch.randn(rows, device="cuda", generator=g), "weights": torch.rand(rows, device="cuda", generator=g)}

    def call(t, logp):
        loss, dz = torch.empty(1, device="cuda"), torch.empty_like(z)
        sl.sl_token_loss(z, targets, t["weights"], loss, logp=logp, dlogits=dz, policy=sl.Policy(t["old"], t["advantage"], 0.2, 0.28, t["ref"], 0.1),
                         workspace=sl.alloc_token_loss_workspace(rows))
        return loss, logp, dz
    want = call(given, torch.empty(rows, device="cuda"))
    copies = {n: t.clone() for n, t in given.items()}
    got = call(copies, copies[which])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
