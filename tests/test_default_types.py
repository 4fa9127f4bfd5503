"""Whatever type a program has made torch's default: the package's own tensors have theirs.

A kernel writes float32 through the address of an output; of a narrower default type the tensor would end before the
kernel does."""

import ast
import glob
import os

import pytest

PKG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_28726_amd")
# Factories of torch whose type is the default one where none is named.
FACTORIES = ("empty", "zeros", "ones", "full", "rand", "randn", "linspace", "empty_strided", "tensor")


def untyped(path):
    with open(path) as f:
        tree = ast.parse(f.read())
    for node in ast.walk(tree):
        if (isinstance(node, ast.Call) and isinstance(node.func, ast.Attribute) and node.func.attr in FACTORIES
                and isinstance(node.func.value, ast.Name) and node.func.value.id == "torch"
                and not any(k.arg == "dtype" for k in node.keywords)):
            yield f"{os.path.basename(path)}:{node.lineno}"


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(PKG, "*.py"))), ids=os.path.basename)
def test_every_tensor_that_is_made_names_its_type(path):
    assert list(untyped(path)) == []


@pytest.mark.gpu
@pytest.mark.parametrize("default", ["float64", "bfloat16", "float16"])
@pytest.mark.parametrize("own_scratch", [False, True])
def test_calls_under_another_default_type(default, own_scratch):
    """The beam and training entry points, and the examples that call them, under each default type."""
    import torch

    import paper_2608_28726_amd as pr
    from paper_2608_28726_amd import beam_search as bs
    from paper_2608_28726_amd import post_train as pt
    from tests.gpu_common import require_gpu
    require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    f32 = dict(dtype=torch.float32, device="cuda")
    n, B, V, k = 24, 4, 5003, 9
    z = torch.empty(n, V, **f32).normal_(generator=g)
    scores = torch.zeros(n // B, B, **f32)
    w, ids = torch.full((n,), 1.0 / n, **f32), torch.arange(n, dtype=torch.int32, device="cuda")
    hidden = torch.empty(3, 16, **f32).normal_(generator=g).bfloat16()
    weight = torch.empty(40, 16, **f32).normal_(generator=g).bfloat16()
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda") if own_scratch else None

    def calls():
        top = pr.top_logits(z, k, 0.9, workspace=scratch)
        out = {"top " + name: x for name, x in top.items()}
        for name, x in (("select ", pr.beam_select(z, scores, 0.9, k, workspace=scratch)),
                        ("distill ", pr.distill_loss(z, top["ids"], top["logprob"], 0.8, w, workspace=scratch)),
                        ("policy ", pr.policy_loss(z, ids, 0.8, w, w, w, workspace=scratch)),
                        ("search ", bs.search(lambda h: h @ weight.t(), hidden, 40, 3, 4, 5))):
            out.update({name + key: value for key, value in x.items()})
        out["post train"] = torch.tensor(pt.post_train("distill", 2, vocab=64, width=16, requests=4, length=2)["loss"],
                                         dtype=torch.float64)
        torch.cuda.synchronize()
        return out

    want = calls()
    before = torch.get_default_dtype()
    torch.set_default_dtype(getattr(torch, default))
    try:
        got = calls()
    finally:
        torch.set_default_dtype(before)
    for name, x in want.items():
        assert got[name].dtype == x.dtype and torch.equal(got[name], x), name
