"""Reordering of states beyond the last-level cache and of more requests than a launch takes."""

import pytest
import torch

import paper_2608_28726_amd as pr
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def parents(n_req, B, seed):
    """Any beam after any other; some entries leave their beam as it is."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    p = torch.randint(0, B, (n_req, B), dtype=torch.int32, device="cuda", generator=g)
    p[torch.rand(n_req, B, device="cuda", generator=g) < 0.05] = -1
    p[torch.rand(n_req, B, device="cuda", generator=g) < 0.05] = B
    return p, g


def rows_of(p):
    """Which row each row becomes."""
    n_req, B = p.shape
    own = torch.arange(B, device="cuda").expand(n_req, B)
    p = torch.where((p >= 0) & (p < B), p.long(), own)
    return (p + B * torch.arange(n_req, device="cuda")[:, None]).view(-1)


@pytest.mark.parametrize("B", [2, 3, 4, 5, 64])
def test_states_beyond_the_cache(B):
    """1.1 GB of states, with odd row lengths among them (up to 4 beams are moved past the caches)."""
    n_req = 256 // B
    n = n_req * B
    p, g = parents(n_req, B, B)
    sizes = (1_048_576, 1_048_577, 1_048_591, 1_000_000, 17, 3)
    states = [torch.randint(0, 256, (n, size), dtype=torch.uint8, device="cuda", generator=g) for size in sizes]
    assert sum(x.numel() for x in states) > 1_000_000_000
    at = rows_of(p)
    want = [x[at] for x in states]
    pr.beam_reorder(states, p)
    torch.cuda.synchronize()
    for x, y in zip(want, states):
        assert torch.equal(x, y), x.shape


@pytest.mark.parametrize("n_req,B", [(32768, 2), (32769, 4), (70000, 3)])
def test_more_requests_than_a_launch_takes(n_req, B):
    n = n_req * B
    p, g = parents(n_req, B, n)
    states = [torch.randint(0, 2 ** 31 - 1, (n, size), dtype=torch.int32, device="cuda", generator=g) for size in (1, 9, 33)]
    at = rows_of(p)
    want = [x[at] for x in states]
    pr.beam_reorder(states, p)
    torch.cuda.synchronize()
    for x, y in zip(want, states):
        assert torch.equal(x, y), x.shape


@pytest.mark.parametrize("max_len", [0, 3])
def test_the_verifier_of_more_requests_than_a_launch_takes(max_len):
    n_req, B, V = 40000, 2, 8
    n = n_req * B
    p, g = parents(n_req, B, 7)
    slots = torch.randperm(n, device="cuda", generator=g).int()
    z = torch.empty(n, V, device="cuda").normal_(generator=g)
    ids = torch.randint(0, V, (n,), dtype=torch.int32, device="cuda", generator=g)
    verdicts = []
    for move in (False, True):
        state = pr.StreamState(n, max_len)
        state.step(z, slots, ids, 1.0)
        state.step(z.flip(0), slots, ids, 1.0)
        if move:
            state.reorder(slots.view(n_req, B), p)
        verdicts.append(state.finish(slots, 0.5))
        torch.cuda.synchronize()
        state.close()
    at = rows_of(p)
    for name, x in verdicts[0].items():
        assert torch.equal(x[at], verdicts[1][name]), name
