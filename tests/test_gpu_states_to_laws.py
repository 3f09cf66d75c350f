"""The operators between states and laws as they are used together: a student's step, forward and back, against one without them, in
place of tolerances by the bounds of what 8 bits hold; the command that uses them."""
import numpy as np
import pytest
import torch

from oracle import block8_oracle as orc
from paper_2206_05279_amd import binding as pb
from paper_2206_05279_amd import fit_laws

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def up(t):
    return t.detach().cpu().double().numpy()


def held(h, kind):
    m = h.block
    return orc.values(m.codes.view(torch.uint8).cpu().numpy(), m.scales.cpu().numpy(), kind, m.record.block_rows)


@pytest.mark.parametrize("width", [32, 130])
def test_a_step_is_its_operators_one_after_the_other(width):
    """Each matrix in 8 bits holds its values to half a step, 2^-4 or 2^-3 of them or of the smallest normal value under the block's
    scale; the products, the loss and the norm's way back are those of what is held."""
    net = fit_laws.StudentNetwork(width, seed=3)
    logits = net.forward().clone()
    y, w = up(net.y), up(net.params["head"])
    y8, w8 = held(net.y8, "e4m3"), held(net.head8, "e4m3")

    def near(v, h, block_rows, kind, extra):
        digits, low = (4, -6) if kind == "e4m3" else (3, -14)
        p = orc.powers(h.block.scales.cpu().numpy(), v.shape, block_rows)
        return (np.abs(held(h, kind) - v) <= 2.0 ** -digits * np.maximum(np.abs(v), 2.0 ** low * p) + extra * np.abs(v)).all()

    assert near(y, net.y8, 1, "e4m3", 2.0 ** -7) and near(w, net.head8, 128, "e4m3", 0)      # y itself is rounded to bfloat16
    assert np.array_equal(held(net.turned_head8, "e4m3"), w8.T)
    want, err = orc.product(y8, w8, True)
    assert (np.abs(up(logits) - want) <= err + 2.0 ** -8 * np.abs(want) * 1.01).all()
    # the loss and its gradient, from the logits as they are
    rng = np.random.default_rng(0)
    teacher = torch.from_numpy(rng.normal(size=(fit_laws.LAWS, 256)) * 2).float().to(DEV)
    sym, logp = torch.empty(fit_laws.LAWS, 16, dtype=torch.int32, device=DEV), torch.empty(fit_laws.LAWS, 16, device=DEV)
    ws = torch.empty(pb.pilc_logprobs_workspace_size(fit_laws.LAWS, 256, 16), dtype=torch.uint8, device=DEV)
    pb.pilc_logprobs(teacher, None, top_sym=sym, top_logp=logp, workspace=ws)
    before = {k: v.clone() for k, v in net.params.items()}
    loss = net.step(sym, logp, lr=0.0)
    wl, wg, le, ge = orc.distill(up(logits), sym.cpu().numpy(), up(logp), np.full(fit_laws.LAWS, np.float32(1.0 / fit_laws.LAWS)), 1.0, True)
    assert (np.abs(up(loss) - wl) <= le + 2.0 ** -23 * np.abs(wl) + 1e-30).all()
    d = up(net.logits)
    assert (np.abs(d - wg) <= ge + 2.0 ** -8 * np.abs(wg) * 1.01 + 1e-30).all()
    assert near(d, net.back8, 1, "e5m2", 0) and near(d.T, net.turned_back8, 1, "e5m2", 0) and near(y.T, net.turned_y8, 1, "e4m3", 0)
    # the way back, from what is held
    wh, eh = orc.product(held(net.turned_back8, "e5m2"), held(net.turned_y8, "e4m3"), False)
    assert (np.abs(up(net.grads["head"]) - wh) <= eh + 2.0 ** -23 * np.abs(wh)).all()
    wy, ey = orc.product(held(net.back8, "e5m2"), held(net.turned_head8, "e4m3"), True)
    hsum, rstd, nw = up(net.sum), up(net.rstd), up(net.params["norm_weight"])
    dx, dw, xe, _ = orc.rms_backward(wy, hsum, nw, rstd, None)
    dy_off = ey + 2.0 ** -8 * np.abs(wy) * 1.01
    hh = np.abs(hsum * rstd[:, None])
    spread = np.abs(rstd[:, None]) * (dy_off * np.abs(nw) + hh * (dy_off * np.abs(nw) * hh).mean(1, keepdims=True))
    assert (np.abs(up(net.dy) - dx) <= xe + spread + 2.0 ** -8 * (np.abs(dx) + spread) * 1.01).all()
    assert (np.abs(up(net.grads["norm_weight"]) - dw) <= (dy_off * hh).sum(0) + 2.0 ** -20 * np.abs(wy * hsum * rstd[:, None]).sum(0)).all()
    assert all(torch.equal(before[k], v) for k, v in net.params.items())       # a rate of 0 moves nothing


def test_a_step_in_a_graph():
    net = fit_laws.StudentNetwork(64, seed=5)
    rng = np.random.default_rng(1)
    sym = torch.from_numpy(np.argsort(rng.random((fit_laws.LAWS, 256)))[:, :8].astype(np.int32)).to(DEV)
    logp = torch.log(torch.rand(fit_laws.LAWS, 8, device=DEV) / 8)
    x = torch.randn(fit_laws.LAWS, 64, device=DEV).bfloat16()
    add = torch.randn_like(x)
    one = torch.ones(fit_laws.LAWS, device=DEV)

    def go():
        pb.pilc_rms_forward(x, net.params["norm_weight"], y=net.y, y8=net.y8.block, add=add, sum=net.sum, rstd=net.rstd)
        pb.pilc_block8_quantize(net.params["head"], net.head8.block, net.turned_head8.block)
        pb.pilc_block8_product(net.y8.block, net.head8.block, net.logits, workspace=net.workspace)
        pb.pilc_distill(net.logits, sym, logp, net.loss, up=one, grad=net.logits, rest=True, workspace=net.workspace)
        pb.pilc_block8_quantize(net.logits, net.back8.block, net.turned_back8.block)
        pb.pilc_block8_quantize(net.y, None, net.turned_y8.block)
        pb.pilc_block8_product(net.back8.block, net.turned_head8.block, net.dy, workspace=net.workspace)
        pb.pilc_block8_product(net.turned_back8.block, net.turned_y8.block, net.grads["head"], workspace=net.workspace)
        pb.pilc_rms_backward(net.dy, net.sum, net.params["norm_weight"], net.rstd, dx=net.dy, dweight=net.grads["norm_weight"], workspace=net.workspace)

    outs = (net.sum, net.y, net.rstd, net.logits, net.loss, net.dy, net.grads["head"], net.grads["norm_weight"])
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        go()
    for _ in range(4):
        x.normal_()
        go()
        torch.cuda.synchronize()
        first = [t.clone() for t in outs]
        net.workspace.fill_(0x5A)
        for t in outs:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, outs))


def test_a_student_codes_the_stream():
    out = fit_laws.fit(images=500, steps=60, batch=4096, say=lambda s: print(s, flush=True), student=48)
    assert out["lossless"] and np.isfinite(out["student"])
