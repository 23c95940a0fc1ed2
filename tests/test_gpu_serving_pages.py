"""The example server with a pool of 8 bits, a window, forks and compactions."""
import os
import sys

import pytest
import torch

import pages_reference as pages

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain_logits(s, tokens):
    """The same model over one sequence, no cache, float32 on the CPU; where the server's pool is in 8 bits, so are keys and values here, rounded block by block."""
    f = lambda t: t.detach().float().cpu()  # noqa: E731
    n, h, kv, d = len(tokens), s.heads, s.kv_heads, s.head_dim
    x = f(s.embedding)[torch.tensor(tokens)]
    cos, sin = f(s.table)[:n, None, :d // 2], f(s.table)[:n, None, d // 2:]
    norm = lambda t: t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    i = torch.arange(n)
    hidden = i[None] > i[:, None]
    if s.window:
        hidden = hidden | ((i[None] <= i[:, None] - s.window) & (i[None] >= s.sinks))

    def turn(t):
        a, b = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    def held(t):
        if s.scales is None:
            return t
        out = t.clone()
        for b in range(0, n, 16):
            for j in range(kv):
                e = pages.scale_for(float(t[b:b + 16, j].abs().max()))
                out[b:b + 16, j] = pages.codes_of(t[b:b + 16, j].double() * 2.0 ** -e) * 2.0 ** e
        return out

    for l in range(s.layers):
        q, k, v = (norm(x) @ f(s.qkv[l])).view(n, h + 2 * kv, d).split([h, kv, kv], 1)
        q, k = turn(norm(q) * f(s.q_norm[l])), turn(norm(k) * f(s.k_norm[l]))
        k, v = held(k).repeat_interleave(h // kv, 1), held(v).repeat_interleave(h // kv, 1)
        scores = torch.einsum("ihd,jhd->hij", q, k) / d ** 0.5
        x = x + torch.einsum("hij,jhd->ihd", torch.softmax(scores.masked_fill(hidden, float("-inf")), -1), v).reshape(n, -1) @ f(s.out[l])
    return x[-1] @ f(s.embedding).T


@pytest.mark.parametrize("in_8_bits, window, sinks", [(False, 40, 4), (True, 0, 0), (True, 40, 4)])
def test_forks_and_compactions_keep_what_requests_see(in_8_bits, window, sinks):
    from prefix_serving import Request, Server
    s = Server(layers=2, heads=8, kv_heads=2, head_dim=64, width=128, vocab=50, blocks=64, max_tokens=512, in_8_bits=in_8_bits, window=window, sinks=sinks)
    gen = torch.Generator().manual_seed(4)
    draw = lambda n: torch.randint(0, 50, (n,), generator=gen).tolist()  # noqa: E731
    # the roundings of bfloat16 in a row, as for a pool of 16 bits: embedding, six in each of two layers.  In 8 bits, a key or value whose roundings up to there (2^-8 and
    # more of it) are put on the other side of a border between codes is off by a step, 2^-3 of it; with steps of 2^-4 to 2^-3 that is about one in eight, 2^-3 / sqrt(8)
    # = 2^-4.5 in the mean square, for keys and for values of each layer
    most = (1 + 2 * 6) * torch.finfo(torch.bfloat16).eps / 2 + (2 * 2 * 2.0 ** -4.5 if in_8_bits else 0.0)

    def check(logits, requests):
        for got, r in zip(logits.cpu(), requests):
            want = plain_logits(s, r.tokens)
            assert float((got - want).norm() / want.norm()) < most

    shared = draw(70)
    batch = [Request(shared + draw(9)), Request(draw(5)), Request(shared + draw(40)), Request(draw(64))]
    check(s.prefill(batch), batch)
    ways = [batch[0]] + s.fork(batch[0], 3)           # 79 tokens: four whole blocks shared, fifteen tokens copied
    assert len({r.blocks[-1] for r in ways}) == 4 and all(r.blocks[:4] == batch[0].blocks[:4] for r in ways)
    ways += s.fork(batch[3], 1)                       # whole blocks alone: nothing to copy
    assert ways[-1].blocks == batch[3].blocks
    for step in range(3):
        logits = s.decode(ways, [step + 7 * i for i in range(5)])
    check(logits, ways)
    assert len({tuple(r.tokens) for r in ways}) == 5
    before, held = len(s.free), len(s.held)
    go_on = [ways[1], ways[4], batch[1]]
    n = s.compact(go_on)
    assert n == len({b for r in go_on for b in r.blocks} | set(s.held.values())) and len(s.held) == held
    assert before < len(s.free) == 64 - n and max(b for r in go_on for b in r.blocks) < n and max(s.held.values()) < n
    logits = s.decode(go_on, [1, 2, 3])
    check(logits, go_on)
    # the index still finds the blocks, where they are now
    later = [Request(shared + draw(12)), Request(list(batch[3].tokens) + draw(3))]
    check(s.prefill(later), later)
    assert [r.found for r in later] == [64, 64]
    assert s.compact([]) == len(set(s.held.values()))


def test_forks_that_cannot_be_are_refused():
    from prefix_serving import Request, Server
    s = Server(layers=1, heads=2, kv_heads=1, head_dim=64, width=32, vocab=20, blocks=5, max_tokens=96)
    r = Request([1] * 20)
    with pytest.raises(ValueError):
        s.fork(r, 1)  # not run yet
    s.prefill([r])
    with pytest.raises(ValueError):
        s.fork(r, 4)  # three blocks are free
    assert len(s.free) == 3 and len(s.fork(r, 3)) == 3 and not s.free
