"""The vocabulary behind the network of gated blocks: a whole training step's losses and gradients against the definition in 64 bits, and the
command."""
import pytest
import torch

from tests import head_reference as R
from paper_1901_07988_amd import token_blocks as N
from paper_1901_07988_amd import token_head as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top,how", [(0, dict(smoothing=0.1)), (0, {}), (5, dict(temperature=2.0, label_weight=0.5)), (7, dict(label_weight=0.0))])
def test_a_step_of_the_network(top, how):
    """Rows from the blocks, their loss, the gradients of the table and back through the blocks, and the update."""
    M, C, F, V, layers = 96, 64, 96, 333, 2
    x = N.batch(M, C, 3)
    teacher = H.Teacher(layers, C, F, 2, V, M, seed=5)
    labels, ids, logits = teacher.look(x, max(top, 1))
    if not top:
        labels = torch.where(torch.arange(M, device="cuda") % 4 == 0, -100, labels)
    net = N.TokenNet(*N.random_parameters(layers, C, F, 2, seed=8), M, 8)
    head = H.VocabularyHead(H.random_table(V, C, 9), M, top=top, **how)
    extra = (ids, logits) if top else ()
    weight = torch.rand(M, device="cuda") / M
    n = net.forward(x)
    rows = n.clone()
    loss = head.forward(n, labels, *extra)
    dn = head.backward(n, labels, weight, *extra)
    settings = R.Settings(**dict(dict(teacher_weight=1.0) if top else {}, **how))
    cpu = [t.cpu() if t is not None else None for t in (rows, head.half, labels, ids if top else None, logits if top else None)]
    want = R.forward(cpu[0], cpu[1], cpu[2], settings, *cpu[3:])
    R.assert_within(loss, want["loss"], want["bound"]["loss"], "loss")
    want = R.backward(cpu[0], cpu[1], cpu[2], head.lse.cpu(), weight.cpu(), settings, torch.bfloat16, torch.float32, ids=cpu[3], t=cpu[4],
                      lse_t=head.lse_t.cpu() if top else None)
    R.assert_within(dn, want["dh"], want["bound"]["dh"], "dn")
    R.assert_within(head.grad, want["dW"], want["bound"]["dW"], "table")
    dx = net.backward(dn)
    assert bool(dx.isfinite().all()) and all(bool(g["W1"].isfinite().all()) and bool((g["W1"] != 0).any()) for g in net.grads)
    before = head.master.clone()
    head.update(0.1)
    torch.testing.assert_close(head.master, before - 0.1 * head.grad, rtol=2.0 ** -22, atol=0.0 + 2.0 ** -24 * float(before.abs().max()))
    assert torch.equal(head.half, head.master.bfloat16())


def test_a_batch_in_parts():
    """The table's gradient of two halves, added, and each half's gradient of its rows, are within the whole batch's bounds."""
    M, C, V = 64, 32, 200
    n = N.batch(M, C, 1)
    labels = torch.randint(0, V, (M,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    weight = torch.full((M,), 1 / M, device="cuda")
    half = H.VocabularyHead(H.random_table(V, C, 4), M // 2)
    parts, lse = [], []
    for i in range(2):
        s = slice(i * M // 2, (i + 1) * M // 2)
        half.forward(n[s], labels[s])
        lse.append(half.lse.clone())
        parts.append(half.backward(n[s], labels[s], weight[s], accumulate=i > 0))
    want = R.backward(n.cpu(), half.half.cpu(), labels.cpu(), torch.cat(lse).cpu(), weight.cpu(), R.Settings(), torch.bfloat16, torch.float32)
    R.assert_within(torch.cat(parts), want["dh"], want["bound"]["dh"], "dn")
    R.assert_within(half.grad, want["dW"], want["bound"]["dW"] + R.F32 * want["dW"].abs(), "table")


def test_the_command_runs():
    curves, after = H.main(["--layers", "1", "--tokens", "128", "--samples", "2", "--channels", "64", "--width", "96", "--vocab", "300", "--top", "4",
                            "--steps", "3"])
    assert set(curves) == {"labels", "logits", "both"}
    assert all(len(c) == 3 and all(v == v and v >= 0 for v in c) for c in curves.values()) and all(v > 0 for v in after.values())
