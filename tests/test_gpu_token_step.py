"""The operators of a training step together, as examples/token_step.py runs
them: from the planned streams to weights that learn, and one step's gradients
against plain torch in 32 bits."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("token_step",
                                                  os.path.join(ROOT, "examples", "token_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_loss_falls(example):
    losses = example.main(steps=40)
    assert len(losses) == 40 and all(x == x for x in losses)
    assert losses[-1] < 0.8 * losses[0]


def test_gradients_of_a_step(example):
    """Weights of 16 bits on both sides; the kernels round P, dS, the outputs
    and gradients to 8 bits (2^-8 each), the plain form nothing: within 4 * 2^-8
    of the gradients' norm."""
    ex = example
    g = torch.Generator().manual_seed(3)
    T, start = 200, [0, 37, 38, 38, 150, 190]
    tokens = torch.randint(0, ex.VOCAB, (T,), generator=g).cuda()
    index, teacher = ex.teacher_entries(tokens, tokens.roll(1))
    weight = (torch.arange(T) < 190).float().cuda() / 190
    model = ex.Model().cuda()
    with torch.no_grad():
        for p in model.parameters():
            p.copy_(p.bfloat16())
    st = torch.tensor(start, dtype=torch.int32, device="cuda")
    ex.Distill.apply(model(tokens, st), index, teacher, 1.5, weight).backward()
    got = [p.grad.clone() for p in model.parameters()]
    model.zero_grad()

    x = model.embed[tokens]
    qkv = (x @ model.qkv).view(T, -1, ex.WIDTH)
    q, k, v = ex._heads(qkv)
    parts = []
    for a, b in zip(start[:-1], start[1:]):
        heads = []
        for h in range(ex.HEADS):
            kh = h // (ex.HEADS // ex.KV_HEADS)
            s = (q[a:b, h] @ k[a:b, kh].T) * ex.WIDTH ** -0.5
            s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), float("-inf"))
            heads.append(torch.softmax(s, 1) @ v[a:b, kh])
        parts.append(torch.stack(heads, 1))
    parts.append(torch.zeros((T - start[-1], ex.HEADS, ex.WIDTH), device="cuda"))
    o = torch.cat(parts).reshape(T, -1)
    logits = (x + o @ model.out) @ model.head
    logq = torch.log_softmax(logits / 1.5, 1)
    logp = torch.log_softmax(teacher.float() / 1.5, 1)
    kl = (logp.exp() * (logp - torch.gather(logq, 1, index.long()))).sum(1)
    (weight * 1.5**2 * kl).sum().backward()
    for a, p in zip(got, model.parameters()):
        assert float((a - p.grad).norm()) <= 4 * 2.0**-8 * float(p.grad.norm())
