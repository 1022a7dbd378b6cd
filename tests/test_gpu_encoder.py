"""The prompt encoder as a whole: its embeddings and gradients against the same
network in 64 bits, its decision against the store's own on the same embeddings.

An e4m3 value is off by at most 2^-4 of its magnitude, 2^-4 / sqrt(3) in the root
mean square. A layer's forward pass rounds four operands and its backward pass
five more on the way to a weight; taken as independent, the errors of two layers
add to sqrt(2 * 9) * 2^-4 / sqrt(3) = 0.153 of a gradient's norm, and those of the
forward pass to sqrt(2 * 4) * 2^-4 / sqrt(3) = 0.102 of a layer's branch. bf16
roundings (2^-8) are small beside them."""
import pytest
import torch

from paper_2603_07917_amd import sage, workloads
from paper_2603_07917_amd.encoder import PromptEncoder

pytestmark = pytest.mark.gpu


def prompts(vocab, lengths, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    off = torch.tensor([0] + list(torch.tensor(lengths).cumsum(0)), dtype=torch.int32)
    return torch.randint(0, vocab, (int(off[-1]),), generator=g, dtype=torch.int32).cuda(), off.cuda()


def plain(enc, tokens, offsets, sides=None):
    """The network in 64 bits with gradients; its weights and its output. `sides`:
    per layer, on which side of the ReLU each hidden value of a run is (the
    gradient is that of the piece of the network that the run was on)."""
    leaf = lambda t: t.double().cpu().requires_grad_()
    table = leaf(enc.table)
    layers = [{k: leaf(getattr(l, k)) for k in ("gain", "w1", "b1", "w2", "b2")} for l in enc.layers]
    off = offsets.cpu().tolist()
    x = torch.stack([table[tokens.cpu().long()[b:e]].sum(0) / max(e - b, 1) for b, e in zip(off, off[1:])])
    norm = lambda v, eps: v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    for i, l in enumerate(layers):
        h = norm(x, enc.eps) * l["gain"] @ l["w1"].t() + l["b1"]
        h = torch.relu(h) if sides is None else h * sides[i]
        x = x + h @ l["w2"].t() + l["b2"]
    return table, layers, norm(x, 1e-12) / enc.d ** 0.5


def encoder(vocab=300, d=96, hidden=200, layers=2):
    enc = PromptEncoder(vocab, d, hidden, layers, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    for l in enc.layers:
        l.b1 += 0.1 * torch.randn(hidden, generator=g, device="cuda")
        l.b2 += 0.1 * torch.randn(d, generator=g, device="cuda")
    return enc


LENGTHS = [1, 7, 40, 0, 3, 129, 1, 18] * 5 + [2000]


def test_embeddings():
    enc = encoder()
    tokens, offsets = prompts(300, LENGTHS, 1)
    e = enc.encode(tokens, offsets).cpu().double()
    want = plain(enc, tokens, offsets)[2].detach()
    assert torch.allclose(e.norm(dim=1), torch.ones(len(LENGTHS), dtype=torch.float64), atol=1e-5)
    assert float((e - want).norm() / want.norm()) < 0.102


def test_one_prompt_is_the_batch_of_one():
    enc = encoder()
    tokens, offsets = prompts(300, LENGTHS, 1)
    e = enc.encode(tokens, offsets)
    for q in (0, 2, 40):
        b, n = int(offsets[q]), LENGTHS[q]
        one = enc.encode(tokens[b:b + n].clone(), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
        # few rows take the exact sums, many the fast ones: rounding apart the same
        assert float((one[0] - e[q]).norm()) < 0.01


def test_gradients():
    enc = encoder()
    tokens, offsets = prompts(300, LENGTHS, 1)
    saved = []
    e = enc.encode(tokens, offsets, saved)
    c = torch.randn(e.shape, generator=torch.Generator().manual_seed(2))
    held = torch.ones_like(enc.table)
    grads = enc.gradients(tokens, offsets, saved, c.cuda(), add=held)
    assert grads["table"] is held
    table, layers, out = plain(enc, tokens, offsets, [(h > 0).cpu() for _, h in saved[:-1]])
    (out * c.double()).sum().backward()
    pairs = [("table", held - 1.0, table.grad)]
    pairs += [(f"{k}{i}", grads["layers"][i][k], l[k].grad) for i, l in enumerate(layers) for k in l]
    for name, got, want in pairs:
        rel = float((got.cpu().double() - want).norm() / want.norm())
        assert rel < 0.153, (name, rel)


def test_a_prompt_without_a_direction_has_no_gradient():
    enc = PromptEncoder(300, 96, 200, 2, seed=3)         # zero biases: an empty prompt's vector is zero
    full, cuts = prompts(300, [20] * 24, 4)
    target = torch.nn.functional.normalize(torch.randn(25, 96, generator=torch.Generator().manual_seed(1)), dim=1).cuda()
    saved, with_empty = [], torch.cat([cuts, cuts[-1:]])
    out = enc.encode(full, with_empty, saved)
    assert int(out[24].count_nonzero()) == 0
    got = enc.gradients(full, with_empty, saved, -target)
    target[24] = 0.0
    want = enc.gradients(full, with_empty, saved, -target)
    assert torch.equal(got["table"], want["table"])
    for a, b in zip(got["layers"], want["layers"]):
        for k in a:
            assert torch.equal(a[k], b[k]) and bool(torch.isfinite(a[k]).all())


def test_descent_brings_prompts_to_their_targets():
    enc = encoder()
    tokens, offsets = prompts(300, [20] * 24, 4)
    target = torch.nn.functional.normalize(torch.randn(24, 96, generator=torch.Generator().manual_seed(1)), dim=1).cuda()
    losses = []
    for _ in range(12):
        saved = []
        e = enc.encode(tokens, offsets, saved)
        losses.append(float((1 - (e * target).sum(1)).mean()))
        enc.step(enc.gradients(tokens, offsets, saved, -target / 24), 2.0)
    assert losses[-1] < 0.5 * losses[0]


def test_decide_is_the_stores_decision_on_the_embeddings():
    enc = encoder()
    past_tokens, past_offsets = prompts(300, [5, 30, 60, 2] * 100, 7)
    edges, reprs = (torch.from_numpy(a).cuda() for a in workloads.log_bins(4096, 64))
    lens = torch.randint(1, 4096, (400,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    store = sage.Store(enc.encode(past_tokens, past_offsets), lens, edges, reprs, k=16, tau=0.2)
    tokens, offsets = prompts(300, LENGTHS, 8)
    got = enc.decide(store, tokens, offsets)
    want = store.decide(enc.encode(tokens, offsets), (offsets[1:] - offsets[:-1]).contiguous())
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # a prompt of the store finds itself
    ids = enc.decide(store, past_tokens, past_offsets)[0]
    assert float((ids[:, 0].cpu() == torch.arange(400)).float().mean()) > 0.99
