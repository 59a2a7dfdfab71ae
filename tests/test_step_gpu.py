"""The example step: its gradients, its rematerialized form, and its trace in the simulator."""
import pytest
import torch

from paper_2006_09616_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def step():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2006_09616_amd import step as S
    return S.Step(layers=2, batch=2, seq=96, hidden=128, heads=2, vocab=500)


def test_rematerialized_step_gives_the_same_gradients(step):
    loss, grads = step.run()
    again, regrads = step.run_rematerialized()
    assert torch.equal(loss, again)
    for k, g in grads.items():
        # the weights' gradients are library products over 192 rows in bf16: the operators of the
        # framework repeat their bits, a library product may be summed in another order
        assert torch.isfinite(g).all() and g.any()
        err = (g.float() - regrads[k].float()).norm() / g.float().norm()
        assert err < 2.0 ** -8, k


def test_step_against_plain_torch(step):
    """The loss against the same layers in 32 bits with stored masks and probabilities."""
    w = {k: v.detach().float() for k, v in step.weights.items()}
    B, S, H, N = step.batch, step.seq, step.hidden, step.heads
    from paper_2006_09616_amd import ops
    x = torch.nn.functional.embedding(step.tokens, w["embedding"])
    pos = torch.arange(S, device="cuda")
    seen = (pos[None] <= pos[:, None])[None] & (step.docs[:, :, None] == step.docs[:, None])
    bias = step.slopes[:, None, None] * (pos[:, None] - pos[None]).abs()

    def drop(t, r, number):
        kept = ops.dropout_add(torch.ones_like(t), p=step.p, seed=step.seed, offset=number * (t.numel() // 2 + 1))
        return r + t * kept

    for i in range(step.layers):
        q, k, v = (t.transpose(1, 2).contiguous() for t in (step.norm(x) @ w[f"qkv{i}"].t()).view(B, S, 3, N, -1).unbind(2))
        s = step.cap * torch.tanh(torch.matmul(q, k.transpose(2, 3).contiguous()) * q.shape[-1] ** -0.5 / step.cap) - bias
        p = torch.softmax(s.masked_fill(~seen[:, None], -torch.inf), 3)
        a = torch.matmul(p, v).transpose(1, 2).reshape(-1, H)
        x = drop(a @ w[f"proj{i}"].t(), x, 2 * i)
        x = drop(torch.nn.functional.gelu(step.norm(x) @ w[f"up{i}"].t()) @ w[f"down{i}"].t(), x, 2 * i + 1)
    z = torch.log_softmax(step.norm(x) @ w["head"].t(), 1)
    want = -z.gather(1, step.targets[:, None]).mean()
    # about 30 roundings to bf16 (2^-9 each, relative to values of size 1) on the way to logits of size 1,
    # averaged over 192 tokens
    assert abs(float(step.run()[0]) - float(want)) < 30 * 2.0 ** -9


def test_step_trace_in_the_simulator(step, oracle_lib):
    from paper_2006_09616_amd import step as S
    trace = step.trace(repeats=1)
    assert trace.n_ops == 2 * (4 + 9 * step.layers)
    got = S.simulate(trace, percents=(100, 60, 40))
    rows = [(0, h, max(1, W.natural_peak(trace) * p // 100), 1) for h in (W.H_DTR, W.H_EQ, W.H_LRU) for p in (100, 60, 40)]
    want = oracle_lib.run([trace], W.make_specs(rows))
    for (name, pct, r), o in zip(got, want):
        for f in ("total_cost", "n_remats", "peak_memory", "status"):
            assert int(r[f]) == int(o[f]), (name, pct, f)
        if pct == 100:
            assert r["status"] == 0 and r["n_remats"] == 0
