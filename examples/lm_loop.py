"""A small language model around EAT layers, on synthetic tokens: every operator of the library in the
place where a model uses it.

    python examples/lm_loop.py [--steps 12]

Scoring (`score`): embedding -> per layer [residual + RMS norm -> EAT layer] -> residual + RMS norm to
e4m3 -> e4m3 vocabulary head -> token NLLs -> perplexity sign, which the layers' routing reads on the
device at the next step.
Training (`train_step`): the same in bf16; the head's gradient, the final norm's gradient, and for each
router the balance loss with its gradient.  The experts stay frozen (the library runs them forward
only), so the head, the final gain and the routers learn.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_33614_gb300 import eat, workloads as W  # noqa: E402

EPS = 1e-6
SHAPE = W.scaled(W.OLMOE, "olmoe-lm", d_model=512, d_ff=256, n_experts=16, max_k=4)
VOCAB, BATCH, LAYERS = 5003, 384, 2


def e4m3_rows(w):
    """Rows as e4m3 with one fp32 scale each."""
    top = w.float().abs().amax(1)
    scale = torch.where(top > 0, top / 448.0, 1.0)
    return (w.float() / scale[:, None]).to(torch.float8_e4m3fn), scale


class Model:
    def __init__(self, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        d = SHAPE.d_model
        self.embed = rand(VOCAB, d).bfloat16()
        self.gammas = [torch.ones(d, device="cuda") for _ in range(LAYERS)]
        self.gamma_out = torch.ones(d, device="cuda")
        self.head_w = (0.02 * rand(VOCAB, d)).bfloat16()
        self.weights = [W.make_layer(SHAPE, layer=i) for i in range(LAYERS)]
        self.routers = [lw.w_router.cuda() for lw in self.weights]
        self.biases = [lw.b_router.cuda() for lw in self.weights]
        self.experts = [[t.cuda() for t in (lw.w_gate, lw.w_up, lw.w_down)] for lw in self.weights]
        # the perplexity signal, written by eat_ppl_update and read by the layers' routing
        self.ppl = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda")
        self.sign = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.accounts = None
        self.layers = []
        self.make_layers()
        self.head = eat.EatHead(self.head_w, BATCH, grad=True)  # w may change in place
        self.head8, self.trained = None, False

    def make_layers(self):
        """Layer handles for the present routers (a handle's weights do not change while it lives);
        the expert accounts go on."""
        old = [layer.accounts() for layer in self.layers]
        for layer in self.layers:
            layer.close()
        self.layers = []
        for i in range(LAYERS):
            p = eat.eat_layer_policy(i, LAYERS, eat.eat_default_params(
                SHAPE.max_k, temperature=SHAPE.temperature))
            layer = eat.EatLayer(self.routers[i], self.biases[i], *self.experts[i], BATCH, p)
            if old:
                layer.set_accounts(*old[i])
            eat.eat_set_ppl_sign_source(layer.h, self.sign)
            self.layers.append(layer)

    def body(self, tokens):
        """(x, residual) before the final norm, and each layer's input and selected experts."""
        x, h, seen = self.embed[tokens], None, []
        for gamma, layer in zip(self.gammas, self.layers):
            x, h = eat.rms_norm(x, gamma, EPS, residual=h)
            out, idx, _, _ = layer.forward(x, 0, with_routing=True)
            seen.append((x, idx))
            x = out
        return x, h, seen

    def score(self, tokens, targets):
        """Token NLLs through the e4m3 head, and the perplexity signal of this window."""
        self.update_head8()
        x, h, _ = self.body(tokens)
        q, scale, _ = eat.rms_norm_fp8(x, self.gamma_out, EPS, residual=h)
        nll, _ = self.head8.nll(q, targets, x_scale=scale)
        eat.eat_ppl_update(nll, nll.numel(), self.ppl, self.sign)
        return nll

    def update_head8(self):
        """The e4m3 head of the present vocabulary matrix; after a training step its rows are written
        in place (a handle's w may change between calls)."""
        if self.head8 is None:
            self.w8, self.w8_scale = e4m3_rows(self.head_w)
            self.head8 = eat.EatHead(self.w8, BATCH, w_scale=self.w8_scale)
        elif self.trained:
            for mine, now in zip((self.w8, self.w8_scale), e4m3_rows(self.head_w)):
                mine.copy_(now)
        self.trained = False

    def train_step(self, tokens, targets, mask, lr=0.5, balance=0.05):
        """One step on the tokens that count; (mean NLL, balance losses, expert counts)."""
        x, h, seen = self.body(tokens)
        y, h = eat.rms_norm(x, self.gamma_out, EPS, residual=h)
        target = torch.where(mask, targets, -1)
        g = mask.float() / mask.sum()
        nll, _, dy, dw = self.head.nll_grad(y, target, g)
        _, dgamma = eat.rms_norm_grad(h, self.gamma_out, EPS, dy)
        losses, all_counts = [], []
        weight = torch.full((1,), balance, device="cuda")
        for i, (x, idx) in enumerate(seen):
            logits = (x.float() @ self.routers[i].T + self.biases[i]) / SHAPE.temperature
            loss, counts, n = eat.balance_loss(logits, idx, mask=mask)
            dlogits = eat.balance_grad(logits, counts, n, weight, mask=mask)
            step = dlogits.T @ x.float() / SHAPE.temperature
            self.routers[i] = self.routers[i] - lr * step
            losses.append(loss)
            all_counts.append(counts)
        self.gamma_out -= lr * dgamma
        self.head_w -= lr * dw
        self.trained = True
        self.make_layers()
        return (nll * g).sum(), losses, all_counts

    def close(self):
        for layer in self.layers:
            layer.close()
        self.head.close()
        if self.head8 is not None:
            self.head8.close()


def batch(seed):
    """Tokens whose successors are a fixed function of them, with some noise; 5 % padding."""
    g = torch.Generator("cuda").manual_seed(seed)
    tokens = torch.randint(0, 64, (BATCH,), generator=g, device="cuda")
    targets = (tokens * 31 + 7) % VOCAB
    mask = torch.rand(BATCH, generator=g, device="cuda") >= 0.05
    return tokens, targets.to(torch.int32), mask


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=12)
    a = ap.parse_args(argv)
    model = Model()
    history = []
    for step in range(a.steps):
        tokens, targets, mask = batch(step)
        nll, losses, counts = model.train_step(tokens, targets, mask)
        history.append(float(nll))
        print(f"step {step}: nll {history[-1]:.4f}  balance "
              + " ".join(f"{float(v):.3f}" for v in losses)
              + f"  busiest expert {int(counts[0].max())} of {int(counts[0].sum())}")
    for step in range(3):
        tokens, targets, _ = batch(100 + step)
        nll = model.score(tokens, targets)
        print(f"score {step}: perplexity {float(nll.mean().exp()):.3f} (e4m3 head), "
              f"sign {int(model.sign)}")
    model.close()
    return history


if __name__ == "__main__":
    main()
