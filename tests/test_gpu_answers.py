"""The network's answers, and a teacher's answers on their way into a student's loss: the operators behind the classifier where the framework itself
calls them."""
import numpy as np
import pytest
import torch

from paper_1805_12549_amd import binding as B
from paper_1805_12549_amd import resnet18 as R
from tests import logits_oracle as O

pytestmark = pytest.mark.gpu


def test_answers_and_distillation_of_a_network():
    n, size, classes = 3, 64, 40
    student, teacher = R.GatedResNet18(4, size, classes=classes, rho=0.3, calib_images=4), R.GatedResNet18(4, size, classes=classes, rho=0.0, calib_images=4)
    x = R._t(student.calib_input[:n])
    labels = torch.arange(n, device="cuda")
    logits, logprob, entropy, top_ids, top_logprobs = teacher.answers(x, labels, top=100)      # (no more than there are)
    assert torch.equal(logits, teacher.forward(x)) and top_ids.shape == (n, classes)
    z = logits.double().cpu().numpy()
    for r in range(n):
        want = O.logprobs(z[r], [r], classes, 1.0)
        O.check(logprob[r:r + 1].cpu().numpy(), *want["logprob"], "logprob")
        O.check(entropy[r].item(), *want["entropy"], "entropy")
        assert np.array_equal(top_ids[r].cpu().numpy(), want["top_ids"])
    # a step of the student's logits on the teacher's first answers, captured with the forward passes of both
    def step():
        _, _, _, ids, logp = teacher.answers(x, top=8)
        mine = student.forward(x)
        loss, _, grad = B.distill(mine, ids, logp, labels, teacher_weight=0.5, label_weight=0.5, grad=True)
        return mine, ids, logp, loss, grad

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    for _ in range(3):
        for g in got:
            g.zero_()
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for w, g, e in zip(want, got, eager):
            assert torch.equal(w, g) and torch.equal(w, e)
    mine, ids, logp, loss, grad = [t.double().cpu().numpy() for t in want]
    for r in range(n):
        (lv, lb), (gv, gb) = O.distill(mine[r], ids[r], logp[r], r, 0.5, 0.5, 1.0)
        O.check(loss[r], lv, lb, "loss")
        O.check(grad[r], gv, gb, "gradient")
    # a teacher that is the student has nothing to teach beyond its first classes
    _, _, _, ids, logp = student.answers(x, top=classes)
    own, _, grad = B.distill(student.forward(x), ids, logp, grad=True)
    for r in range(n):
        (lv, lb), (gv, gb) = O.distill(mine[r], ids[r].cpu().numpy(), logp[r].cpu().numpy(), -1, 1.0, 0.0, 1.0)
        O.check(own[r].item(), lv, lb, "own loss")
        O.check(grad[r].cpu().numpy(), gv, gb, "own gradient")
    student.close()
    teacher.close()
