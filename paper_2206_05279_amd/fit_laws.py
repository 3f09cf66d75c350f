"""Learns the laws of a stream of vector indices and codes the stream under them.

    python -m paper_2206_05279_amd.fit_laws [--images N] [--steps K]

An image of 32 x 32 pixels is 16 x 16 indices out of 256 (arXiv 2206.05279, Sec. 3.1).  One static law
for all of them costs what their histogram does.  Here the law of an index hangs on what both sides know
beforehand, its place (8 x 8 cells) and the class of its image (one of 3): 192 laws, which a small network
answers with as logits.  A training step takes a batch of indices through an embedding, layer norm and a
linear layer, lets `pilc_logprobs_train` say what the indices cost and how the logits should move, and goes
back through `pilc_norm_backward` to `pilc_adamw_step`, whose states are held in 8 bits.  At the end the laws
become the integer masses of the table-driven coder, which codes the stream and gives it back.

The indices are synthetic, drawn from laws of low rank.
"""
from __future__ import annotations

import argparse
import math
from dataclasses import dataclass

import numpy as np
import torch

from . import binding as pb

NUM_SYM, CELLS, CLASSES, SIDE = 256, 64, 3, 16
LAWS = CELLS * CLASSES
PREC_BITS = 12


def law_numbers(classes: torch.Tensor) -> torch.Tensor:
    """uint8 [images, 256]: which of the 192 laws each index of an image has."""
    row, col = torch.meshgrid(torch.arange(SIDE), torch.arange(SIDE), indexing="ij")
    cell = ((row // 2) * (SIDE // 2) + col // 2).reshape(-1).to(classes.device)
    return (classes.long()[:, None] * CELLS + cell[None]).to(torch.uint8)


def make_stream(images: int, seed: int, device: str = "cuda:0"):
    """(indices, law numbers) uint8 [images, 256], drawn from 192 seeded laws of rank 8."""
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn(LAWS, 8, generator=g) @ torch.randn(8, NUM_SYM, generator=g) * 0.9
    cum = torch.softmax(logits, 1).cumsum(1).to(device)
    laws = law_numbers(torch.randint(0, CLASSES, (images,), generator=g).to(device))
    d = torch.Generator(device=device).manual_seed(seed + 1)
    out = torch.empty(images, SIDE * SIDE, dtype=torch.uint8, device=device)
    for a in range(0, images, 4096):
        u = torch.rand(laws[a:a + 4096].shape, generator=d, device=device)
        rows = cum[laws[a:a + 4096].long()]
        out[a:a + 4096] = (rows < u[..., None]).sum(-1).clamp(max=NUM_SYM - 1).to(torch.uint8)
    return out, laws


def masses_of(p: np.ndarray, prec_bits: int = PREC_BITS) -> np.ndarray:
    """Integer masses, 1 at least and 2^prec_bits in all a row, near the probabilities p [laws, symbols]."""
    top = (1 << prec_bits) - p.shape[1]
    cut = np.rint(np.concatenate([np.zeros((len(p), 1)), np.cumsum(p / p.sum(1, keepdims=True), 1)], 1) * top).astype(np.int64)
    cut[:, -1] = top
    return (1 + np.diff(cut, axis=1)).astype(np.uint32)


@dataclass
class LawNetwork:
    """Logits of a law: embedding of its cell and class, layer norm, linear layer."""

    width: int = 128
    device: str = "cuda:0"
    seed: int = 0

    def __post_init__(self):
        g = torch.Generator().manual_seed(self.seed)
        new = lambda *shape, scale: (torch.randn(*shape, generator=g) * scale).to(self.device)  # noqa: E731
        self.params = {"cell": new(CELLS, self.width, scale=0.5), "class": new(CLASSES, self.width, scale=0.5),
                       "norm_weight": torch.ones(self.width, device=self.device), "norm_bias": torch.zeros(self.width, device=self.device),
                       "head": new(self.width, NUM_SYM, scale=self.width ** -0.5)}
        self.grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        codes = lambda v, each=1: torch.zeros(-(-v.numel() // each), dtype=torch.uint8, device=self.device)  # noqa: E731
        state = lambda each: [codes(v, each) for v in self.params.values()]  # noqa: E731
        self.state = {"m": state(1), "v": state(1), "m_scale": state(256), "v_scale": state(256)}
        self.list = pb.make_adamw_tensors(list(self.params.values()), list(self.grads.values()), self.state["m"], self.state["v"],
                                          self.state["m_scale"], self.state["v_scale"],
                                          decay=[0.01 if v.dim() == 2 else 0.0 for v in self.params.values()])
        self.steps = 0

    def logits(self, laws: torch.Tensor):
        """Logits (bfloat16) of the laws, and what the way back needs."""
        p, rows = self.params, laws.numel()
        h = (p["cell"][laws % CELLS] + p["class"][laws // CELLS]).to(torch.bfloat16)
        y, mean, rstd = torch.empty_like(h), torch.empty(rows, device=h.device), torch.empty(rows, device=h.device)
        pb.pilc_norm_forward(h, p["norm_weight"], p["norm_bias"], y, mean=mean, rstd=rstd)
        return y @ p["head"].to(torch.bfloat16), (h, y, mean, rstd)

    def step(self, symbols: torch.Tensor, laws: torch.Tensor, lr: float) -> torch.Tensor:
        """One step on a batch of indices; returns ln p of each before it."""
        p, g, rows = self.params, self.grads, symbols.numel()
        logits, (h, y, mean, rstd) = self.logits(laws)
        logp = torch.empty(rows, device=h.device)
        up = torch.full((rows,), -1.0 / rows, device=h.device)     # the mean length, downwards
        workspace = torch.empty(max(pb.pilc_logprobs_workspace_size(rows, NUM_SYM), pb.pilc_norm_workspace_size(rows, self.width)),
                                dtype=torch.uint8, device=h.device)
        pb.pilc_logprobs_train(logits, symbols, up, logp, logits, workspace=workspace)      # the gradient takes the logits' place
        g["head"].copy_(y.t() @ logits)
        dy = logits @ p["head"].to(torch.bfloat16).t()
        pb.pilc_norm_backward(dy, h, p["norm_weight"], mean, rstd, dy, g["norm_weight"], g["norm_bias"], workspace=workspace)
        dh = dy.float()
        g["cell"].zero_().index_add_(0, laws % CELLS, dh)
        g["class"].zero_().index_add_(0, laws // CELLS, dh)
        self.steps += 1
        pb.pilc_adamw_step(self.list, lr=lr, beta1=0.9, beta2=0.99, eps=1e-8, step=self.steps, dither=self.steps)
        return logp

    def laws(self) -> np.ndarray:
        """Probabilities [192, 256] of all laws."""
        x, _ = self.logits(torch.arange(LAWS, device=self.device))
        return torch.softmax(x.float(), 1).cpu().numpy()


def _bits(nats: torch.Tensor) -> float:
    return float(-nats.double().mean()) / math.log(2)


def code(symbols: torch.Tensor, laws: torch.Tensor, masses: np.ndarray):
    """(bytes of the container, whether the stream came back) of the table-driven coder, a piece an image."""
    dev = symbols.device
    shape = pb.make_ansai_shape(*symbols.shape, PREC_BITS, *masses.shape)
    tables = torch.empty(pb.pilc_ansai_table_bytes(PREC_BITS, *masses.shape), dtype=torch.uint8, device=dev)
    pb.pilc_ansai_build_tables(PREC_BITS, *masses.shape, torch.from_numpy(masses).to(dev), tables)
    ws_bytes, most = pb.pilc_ansai_workspace_size(shape)
    workspace, coded = (torch.empty(n, dtype=torch.uint8, device=dev) for n in (ws_bytes, most))
    _, nbytes = pb.pilc_ansai_encode(shape, symbols, laws, tables, workspace, coded)
    back = torch.empty_like(symbols)
    pb.pilc_ansai_decode(shape, coded, nbytes, laws, tables, workspace, back)
    return nbytes, torch.equal(back, symbols)


def fit(images: int = 20000, steps: int = 300, batch: int = 16384, lr: float = 5e-3, seed: int = 0, say=print) -> dict:
    """Learns, codes and compares; returns the figures, bits an index."""
    symbols, laws = make_stream(images, seed)
    flat_s, flat_l = symbols.reshape(-1), laws.reshape(-1).long()
    net = LawNetwork(seed=seed)
    pick = torch.Generator(device=symbols.device).manual_seed(seed)
    for k in range(steps):
        at = torch.randint(0, flat_s.numel(), (batch,), generator=pick, device=symbols.device)
        logp = net.step(flat_s[at], flat_l[at], lr * min(1.0, 4.0 * (1 - k / steps)))
        if say and (k % 50 == 0 or k == steps - 1):
            say("step %3d: %.4f bits an index" % (k, _bits(logp)))
    # what the whole stream costs under the laws learned, and what the laws expect of themselves
    table, _ = net.logits(torch.arange(LAWS, device=symbols.device))
    workspace = torch.empty(pb.pilc_logprobs_workspace_size(LAWS, NUM_SYM, 4), dtype=torch.uint8, device=symbols.device)
    lse, entropy = (torch.empty(LAWS, device=symbols.device) for _ in range(2))
    best, best_logp = torch.empty(LAWS, 4, dtype=torch.int32, device=symbols.device), torch.empty(LAWS, 4, device=symbols.device)
    pb.pilc_logprobs(table, None, entropy=entropy, lse=lse, top_sym=best, top_logp=best_logp, workspace=workspace)
    learned = _bits(table.float()[flat_l, flat_s.long()] - lse[flat_l])
    expected = float(entropy[flat_l].double().mean()) / math.log(2)
    # one static law against the learned ones, in the same coder
    counts = torch.bincount(flat_s.long(), minlength=NUM_SYM).cpu().numpy().astype(np.float64)
    static_bytes, static_back = code(symbols, torch.zeros_like(laws), masses_of(counts[None]))
    nbytes, back = code(symbols, laws, masses_of(net.laws()))
    out = {"learned": learned, "expected": expected, "coded": 8.0 * nbytes / symbols.numel(), "static": 8.0 * static_bytes / symbols.numel(),
           "lossless": back and static_back, "best": best.cpu(), "best_logp": best_logp.cpu()}
    if say:
        say("learned laws: %.4f bits an index (they expect %.4f), coded %.4f; one static law, coded %.4f; lossless: %s" % (
            learned, expected, out["coded"], out["static"], out["lossless"]))
        say("law 0 answers with %s at %s bits" % (best[0].tolist(), ["%.2f" % b for b in (-best_logp[0] / math.log(2)).tolist()]))
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--images", type=int, default=20000)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    fit(a.images, a.steps, seed=a.seed)
