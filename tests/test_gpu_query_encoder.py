"""The encoder's operators together: its gradients against differences of its own loss, training, serving, search."""
import numpy as np
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from paper_2506_00812_amd.query_encoder import QueryEncoder

pytestmark = pytest.mark.gpu


def batch(m, width, dim, n_labels, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((m, width), generator=g, device="cuda")
    y = torch.randn((m, dim), generator=g, device="cuda")
    t = torch.randint(0, n_labels, (m,), generator=g, device="cuda", dtype=torch.int32)
    t[0] = -1
    return x, y, t


def test_gradients_against_a_float64_model():
    """All twelve gradients against torch's own differentiation of the formula in 64 bits, on the CPU.  Each passes up to eight
    float32 operators with sums of up to 48 terms, errors of some 100 x 2^-24 of the largest gradient: 2e-5."""
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=torch.float32)
    x, y, t = batch(16, 24, 12, 10)
    loss, grads = enc.gradients(x, y, t, label_weight=0.7, entropy_weight=0.2)
    p = {k: v.double().cpu().requires_grad_() for k, v in enc.params.items()}
    X, Y, T = x.double().cpu(), y.double().cpu(), t.long().cpu()
    ln = lambda v, w, b: torch.nn.functional.layer_norm(v, (24,), w, b)   # noqa: E731
    z = ln(X, p["n1w"], p["n1b"]) @ p["w1"].t() + p["b1"]
    h = X + z * torch.special.ndtr(z) @ p["w2"].t() + p["b2"]
    g = ln(h, p["n2w"], p["n2b"])
    lp = torch.log_softmax(g @ p["wl"].t() + p["bl"], 1)
    picked = lp.gather(1, T.clamp_min(0)[:, None])[:, 0] * (T >= 0)
    want = ((g @ p["wv"].t() + p["bv"] - Y) ** 2).sum(1).mean() - 0.7 * picked.mean() + 0.2 * (lp.exp() * lp).sum(1).mean()
    want.backward()
    assert abs(loss.item() - want.item()) < 2e-5 * abs(want.item())
    for k, v in p.items():
        assert (grads[k].double().cpu() - v.grad).abs().max() <= 2e-5 * v.grad.abs().max(), k


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 32), (torch.bfloat16, 8), (torch.bfloat16, 32), (torch.float16, 8)])
def test_training_learns(dtype, bits):
    enc = QueryEncoder(64, 16, 30, dtype=dtype, state_bits=bits, absent=[3, 29])
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    lift, mark = torch.randn((16, 64), generator=g, device="cuda") / 4, torch.randn((30, 64), generator=g, device="cuda")
    first = last = None
    for i in range(150):
        y = torch.randn((256, 16), generator=g, device="cuda")
        t = torch.randint(0, 29, (256,), generator=g, device="cuda", dtype=torch.int32)
        t[t == 3] = 4
        x = (y @ lift + mark[t.long()]).to(dtype)
        last = enc.train_step(x, y, t, lr=3e-3).item()
        first = last if first is None else first
    assert np.isfinite(last) and last < 0.3 * first
    _, ids, logp, entropy = enc.encode(x, top=30)
    assert not ((ids == 3) | (ids == 29)).any() and (ids[:, 28:] == -1).all()      # labels that nothing carries
    assert (ids[:, 0] == t).float().mean() > 0.9 and torch.isfinite(entropy).all()
    # one query as it is served, against its row of the batch: other tiles, the same sums up to their order and one rounding each
    one = enc.encode(x[5:6], top=4)
    assert (one[1][0, 0] == ids[5, 0]) and (one[2][0] - logp[5, :4]).abs().max() < 0.1
    assert (one[0].float() - enc.encode(x)[0][5:6].float()).abs().max() < 0.1


def test_search_with_predicted_labels(tiny):
    s = tiny.spec
    X = torch.from_numpy(tiny.vectors.astype(np.float32)).cuda()
    index = vf.build_index(X, tiny.label_offsets, tiny.label_ids, s.n_labels, s.T, s.graph_degree)
    enc = QueryEncoder(64, s.dim, s.n_labels, dtype=torch.float32)
    x = torch.randn((50, 64), device="cuda")
    ids, dists, labels = enc.search(index, x, 10, itopk=32, width=1, iters=20, n_seeds=128)
    vectors, top, _, _ = enc.encode(x)
    assert torch.equal(top[:, 0], labels)
    want = vf.search(index, vectors, np.arange(51), labels.cpu().numpy(), 10, itopk=32, width=1, iters=20, n_seeds=128)
    assert torch.equal(ids, want[0]) and torch.equal(dists, want[1])
    found = ids[ids >= 0].cpu().numpy()
    rows = torch.nonzero(ids >= 0)[:, 0].cpu().numpy()
    lab = labels.cpu().numpy()
    assert len(found) and all(lab[r] in tiny.point_labels(i) for r, i in zip(rows, found))
