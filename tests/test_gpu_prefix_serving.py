"""The example server: batches behind cached prefixes give what a plain 32-bit forward pass over all tokens gives."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain_logits(s, tokens):
    """The same model over one sequence, no cache, float32 on the CPU."""
    f = lambda t: t.detach().float().cpu()  # noqa: E731
    n, h, kv, d = len(tokens), s.heads, s.kv_heads, s.head_dim
    x = f(s.embedding)[torch.tensor(tokens)]
    cos, sin = f(s.table)[:n, None, :d // 2], f(s.table)[:n, None, d // 2:]
    norm = lambda t: t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6)  # noqa: E731

    def turn(t):
        a, b = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    for l in range(s.layers):
        q, k, v = (norm(x) @ f(s.qkv[l])).view(n, h + 2 * kv, d).split([h, kv, kv], 1)
        q, k = turn(norm(q) * f(s.q_norm[l])), turn(norm(k) * f(s.k_norm[l]))
        k, v = k.repeat_interleave(h // kv, 1), v.repeat_interleave(h // kv, 1)
        scores = torch.einsum("ihd,jhd->hij", q, k) / d ** 0.5
        scores = scores.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), float("-inf"))
        x = x + torch.einsum("hij,jhd->ihd", torch.softmax(scores, -1), v).reshape(n, -1) @ f(s.out[l])
    return x[-1] @ f(s.embedding).T


@pytest.mark.parametrize("dtype, head_dim", [(torch.bfloat16, 64), (torch.float16, 128)])
def test_served_batches_agree_with_a_plain_forward_pass(dtype, head_dim):
    from prefix_serving import Request, Server
    s = Server(layers=2, heads=8, kv_heads=2, head_dim=head_dim, width=128, vocab=50, blocks=256, max_tokens=512, dtype=dtype)
    gen = torch.Generator().manual_seed(3)
    draw = lambda n: torch.randint(0, 50, (n,), generator=gen).tolist()  # noqa: E731
    shared, other = draw(70), draw(33)
    # roundings in a row: embedding, and in each of two layers the norm, projection, rotation, weights, attention and the projection back
    most = (1 + 2 * 6) * torch.finfo(dtype).eps / 2

    def check(logits, requests):
        for got, r in zip(logits.cpu(), requests):
            want = plain_logits(s, r.tokens)
            assert float((got - want).norm() / want.norm()) < most

    first = [Request(shared + draw(9)), Request(draw(5)), Request(other + draw(40))]
    check(s.prefill(first), first)
    assert [r.found for r in first] == [0, 0, 0]
    second = [Request(shared + draw(30)), Request(other[:16] + draw(17)), Request(shared[:48] + draw(1)), Request(first[0].tokens[:64]), Request(draw(20)), Request(shared + draw(3))]
    logits = s.prefill(second)
    check(logits, second)
    assert [r.found for r in second] == [64, 16, 48, 48, 0, 64]  # whole blocks, and never all of a request's tokens
    for _ in range(3):
        logits = s.decode(second, logits.argmax(-1).tolist())
    check(logits, second)
    third = [Request(list(second[0].tokens) + draw(4)), Request(list(second[1].tokens))]
    check(s.prefill(third), third)
    assert third[0].found == 96 and third[1].found == 32  # the prompt's own complete blocks


def test_requests_that_cannot_be_served_are_refused_before_anything_is_taken():
    """Without tokens, of more than there are angles for, or of more blocks than there are free: such batches gave logits of other tokens or NaN."""
    from prefix_serving import Request, Server
    s = Server(layers=1, heads=2, kv_heads=1, head_dim=64, width=32, vocab=20, blocks=5, max_tokens=96)
    for tokens in ([], [1] * 97, [1] * 81):
        requests = [Request([1, 2, 3]), Request(tokens)]
        with pytest.raises(ValueError):
            s.prefill(requests)
        assert len(s.free) == 5 and not any(r.blocks for r in requests)
    assert bool(torch.isfinite(s.prefill([Request([1] * 60), Request([2])])).all())
