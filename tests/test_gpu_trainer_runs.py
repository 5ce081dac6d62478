"""A trainer's calls as they run together: a teacher's rows through the lm-head, their top logits, distillation; a routed rollout whose metadata
go to the loss from hidden states; each against the library's own path over full logits, or the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _models(N, d, V, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    weight = (2.0 / d ** 0.5 * torch.randn((V, d), generator=g, device=DEV)).to(BF16)
    hidden = (1.5 * torch.randn((N, d), generator=g, device=DEV)).to(BF16)
    other = (hidden.float() + 0.3 * torch.randn((N, d), generator=g, device=DEV)).to(BF16)
    return hidden, other, weight, g


@pytest.mark.parametrize("reverse", [False, True])
def test_a_teacher_s_top_logits_teach_a_student(reverse):
    N, d, V, k = 200, 256, 8192, 48
    hidden, teacher, weight, g = _models(N, d, V, 1)
    t_logits, _, t_lse = P.lmhead_lse(teacher, weight)
    top = P.top_logits(t_logits, k)
    assert torch.allclose(top["lse"], t_lse, rtol=1e-5, atol=1e-5) and (top["row_status"] == 0).all()
    s_logits, _, s_lse = P.lmhead_lse(hidden, weight)
    mask = (torch.rand(N, generator=g, device=DEV) < 0.9).to(torch.uint8)
    n = int(mask.sum())
    out, dlogits = P.distill_top(s_logits, top["token"], top["logit"], top["lse"], reverse=reverse, mask=mask, grad_scale=1.0 / n)
    assert torch.allclose(out["lse"][mask != 0], s_lse[mask != 0], rtol=1e-5, atol=1e-5)
    # the same from all of the teacher's row: what the list leaves out is one event, so the divergence over the list is at most that over the row
    p, t = (torch.log_softmax(x.double(), 1) for x in (s_logits, t_logits))
    full = (p.exp() * (p - t)).sum(1) if reverse else (t.exp() * (t - p)).sum(1)
    m = mask != 0
    assert bool((out["loss"][m].double() <= full[m] + 1e-4).all()) and bool((out["loss"][m] > 0).all())
    # a small step against the gradient lowers the loss by about its square
    step = 0.02 * n
    after, _ = P.distill_top((s_logits.float() - step * dlogits.float()).contiguous(), top["token"], top["logit"], top["lse"], reverse=reverse, mask=mask, dlogits=None)
    fall = float((out["loss"] - after["loss"]).sum() / n)
    want = float(step * (dlogits.double() ** 2).sum())
    assert 0.8 * want <= fall <= 1.05 * want
    assert P.check() == 0


def test_a_list_of_everything_is_the_full_divergence():
    N, V = 60, 100
    g = torch.Generator(device=DEV).manual_seed(2)
    s, t = (2 * torch.randn((N, V), generator=g, device=DEV) for _ in range(2))
    top = P.top_logits(t, V)
    for lse, reverse in ((None, False), (top["lse"], False), (top["lse"], True)):
        out, grad = P.distill_top(s, top["token"], top["logit"], lse, reverse=reverse)
        p, q = torch.log_softmax(s.double(), 1).requires_grad_(), torch.log_softmax(t.double(), 1)
        z = s.double().requires_grad_()
        p = torch.log_softmax(z, 1)
        loss = (p.exp() * (p - q)).sum(1) if reverse else (q.exp() * (q - p)).sum(1)
        loss.sum().backward()
        assert torch.allclose(out["loss"].double(), loss, rtol=1e-5, atol=2e-6) and torch.allclose(grad.double(), z.grad, rtol=2e-5, atol=2e-6)


def test_routed_training_from_hidden_states():
    """The routing call's metadata through linear_ce is what route_bwd_from_meta makes of the full logits, and the lm-head's two products of that."""
    N, d, V = 300, 192, 6000
    hidden, other, weight, g = _models(N, d, V, 3)
    s, _, _ = P.lmhead_lse(hidden, weight)
    t, _, _ = P.lmhead_lse(other, weight)
    x = P.sample_proposal(s, seed=5)
    mask = (torch.rand(N, generator=g, device=DEV) < 0.85).to(torch.uint8)
    n = int(mask.sum())
    out = P.route_fwd(s, t, x, 0.05, seed=7, mask=mask)
    advantage = out["logT_x"] - out["logp_x"]
    assert 0 < int(out["corrected"].sum()) < N
    meta = dict(advantage=advantage, corrected=out["corrected"], teacher_top1=out["teacher_top1"], mask=mask, rollout_status=out["row_status"])
    linear = P.linear_ce(hidden, weight, x, **meta)
    dh, dw = P.linear_ce_bwd(hidden, weight, x, linear["lse"], grad_scale=1.0 / n, **meta)
    ref, dlogits = P.route_bwd_from_meta(s, out["corrected"], x, out["teacher_top1"], advantage, mask=mask, rollout_status=out["row_status"], grad_scale=1.0 / n)
    torch.cuda.synchronize()
    assert torch.equal(linear["row_status"], ref["row_status"])
    # the stored logits are rounded to bf16 (2^-8 of up to 16), those of the products are not; and the log-sum-exp with them
    assert float((linear["logp_tok"] - ref["logp_tok"]).abs().max()) <= 2 * 16 * 2.0 ** -8
    for got, want in ((dh, dlogits.double() @ weight.double()), (dw, dlogits.double().t() @ hidden.double())):
        assert float((got.double() - want).norm() / want.norm()) < 0.02
    h64, w64 = hidden.double().cpu().numpy(), weight.double().cpu().numpy()
    rows = O.supervised(V, x.cpu().numpy(), **{k: v.cpu().numpy() for k, v in meta.items()})
    exact = O.linear_ce(h64, w64, rows, 1.0, 1.0 / n)
    assert np.max(np.abs(linear["loss"].cpu().numpy() - exact["loss"])) <= 1e-4
    for got, name in ((dh, "dhidden"), (dw, "dweight")):
        err = np.linalg.norm(got.double().cpu().numpy() - exact[name]) / np.linalg.norm(exact[name])
        assert err < 2.0 ** -8, (name, err)
    assert P.check() == 0


def test_the_whole_step_captured():
    """Teacher's list, distillation and the loss from hidden states in one graph, replayed on new hidden states, beside calls on another stream."""
    N, d, V, k = 96, 128, 5000, 20
    hidden, teacher, weight, g = _models(N, d, V, 4)
    target = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)

    def step():
        t_logits, _, _ = P.lmhead_lse(teacher, weight)
        top = P.top_logits(t_logits, k)
        s_logits, _, _ = P.lmhead_lse(hidden, weight)
        out, dlogits = P.distill_top(s_logits, top["token"], top["logit"], top["lse"], grad_scale=1.0 / N)
        ce = P.linear_ce(hidden, weight, target)
        return (top["token"], out["loss"], dlogits, ce["loss"], *P.linear_ce_bwd(hidden, weight, target, ce["lse"], grad_scale=1.0 / N))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    other = torch.cuda.Stream()
    for i in range(3):
        hidden.copy_(torch.randn((N, d), generator=g, device=DEV).to(BF16))
        teacher.copy_(torch.randn((N, d), generator=g, device=DEV).to(BF16))
        other.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(other):
            want = step()                     # at the same time, with scratch of its own
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    assert P.check() == 0
