"""What the operators behind the classifier return, as tensors like any other: each has memory of its own, is saved and loaded alone and with the others."""
import io

import pytest
import torch

from paper_1805_12549_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["extension", "ctypes"])
def way(request, monkeypatch):
    """Both ways of marshalling."""
    if request.param == "ctypes":
        monkeypatch.setattr(B, "_calls", None)
    elif B._calls is None:
        pytest.skip("the extension is not built")
    return request.param


def outputs(rows, classes, top):
    z = torch.randn(rows, classes, device="cuda")
    labels = torch.randint(0, classes, (rows, 2), device="cuda")
    logprob, entropy, top_ids, top_logprobs = B.logprobs(z, labels, top=top)
    loss, stats, grad = B.distill(z, top_ids, top_logprobs, labels[:, 0].contiguous(), label_weight=0.5, grad=True)
    return dict(logprob=logprob, entropy=entropy, top_ids=top_ids, top_logprobs=top_logprobs, loss=loss, stats=stats, grad=grad)


def loaded(what):
    f = io.BytesIO()
    torch.save(what, f)
    size = f.tell()
    f.seek(0)
    return torch.load(f, weights_only=True), size


@pytest.mark.parametrize("rows,classes,top", [(1, 1000, 5), (256, 1000, 5), (64, 777, 128), (2000, 130, 100)])
def test_outputs_are_saved_and_loaded(way, rows, classes, top):
    outs = outputs(rows, classes, top)
    again, _ = loaded(outs)
    for k, t in outs.items():
        assert torch.equal(again[k], t) and again[k].dtype == t.dtype and again[k].shape == t.shape, k
    top_lists, _ = loaded((outs["top_ids"], outs["top_logprobs"]))
    assert torch.equal(top_lists[0], outs["top_ids"]) and torch.equal(top_lists[1], outs["top_logprobs"])
    _, least = loaded(torch.zeros(1, device="cuda"))
    for k, t in outs.items():
        one, size = loaded(t)
        assert torch.equal(one, t), k
        assert size <= least + t.numel() * t.element_size() + 256, "%s alone takes %d bytes for %d" % (k, size, t.numel() * t.element_size())


@pytest.mark.parametrize("rows", [1, 300])
def test_an_output_that_is_kept_holds_no_other(way, rows):
    outs = outputs(rows, 900, 100)
    places = set()
    for k, t in outs.items():
        assert t.untyped_storage().nbytes() == t.numel() * t.element_size(), k
        places.add(t.untyped_storage().data_ptr())
    assert len(places) == len(outs)
    held = torch.cuda.memory_allocated()
    kept = outs.pop("entropy")
    freed = sum(max(512, t.numel() * t.element_size()) for t in outs.values())       # (the allocator rounds up, to 512 bytes at least)
    outs.clear()
    del t
    assert held - torch.cuda.memory_allocated() >= freed and kept.shape == (rows,)


def test_memory_is_the_allocators_own(way):
    """What a stream that was told of still reads is not given to the next call; outputs are on the logits' device."""
    side = torch.cuda.Stream()
    a, b = torch.randn(4096, 4096, device="cuda"), torch.empty(4096, 4096, device="cuda")
    outs = outputs(700, 900, 100)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.mm(a, a, out=b)
        places = set()
        for k, t in outs.items():
            assert t.device == a.device and t.is_contiguous() and not t._is_view() and not t.requires_grad, k
            t.record_stream(side)
            places.add(t.data_ptr())
    waits = not side.query()
    outs.clear()
    del t
    again = outputs(700, 900, 100)
    if waits and not side.query():          # (the products still run)
        assert not places & {t.data_ptr() for t in again.values()}
    torch.cuda.synchronize()
    again.clear()
