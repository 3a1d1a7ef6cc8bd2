"""A training step in few bits on one GPU: products of 4-bit matrices forward and backward, moments in 8 bits.

A perceptron (784-256-256-10, the smallest benchmark configuration) learns which of ten directions a sample is nearest to.  Every step:

    mc_mx_quantize of the layers' weights (from the 16-bit copy) and inputs, along rows and along columns
    -> mc_mx_matmul with the bias: logits -> mc_token_logp, mc_policy_loss: loss and d loss / d logits (with advantages of 1 and the
       present policy for the old one that is the cross entropy's gradient)
    -> for every layer, last first: mc_mx_quantize of its outputs' gradient, mc_mx_matmul by the weights' columns and with the inputs' columns
    -> mc_grad_norm, clipped to MAX_NORM -> mc_adamw8, which writes the 16-bit copy

Run from the repository's root:  python examples/lowbit_step.py [--steps 200]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2103_15195_amd import mx as X  # noqa: E402
from paper_2103_15195_amd import step as S  # noqa: E402

DEV = "cuda:0"
SIZES, BATCH = (784, 256, 256, 10), 512
MAX_NORM, LR, BETAS, DECAY = 1.0, 2e-3, (0.9, 0.95), 0.01


class Layer:
    """y = x W^T + b with W and x in 4 bits; what the backward pass needs is laid out in the forward one."""

    def __init__(self, mx, inputs, outputs, gen):
        self.mx = mx
        self.weight = torch.randn(outputs, inputs, device=DEV, generator=gen) * inputs ** -0.5
        self.bias = torch.zeros(outputs, device=DEV)
        self.model = self.weight.bfloat16()          # what is quantised: mc_adamw8 keeps it
        self.bias_model = self.bias.bfloat16()
        self.dweight, self.dbias = torch.zeros_like(self.weight), torch.zeros_like(self.bias)
        self.w_rows, self.w_cols = X.MxMatrix(outputs, inputs), X.MxMatrix(inputs, outputs)
        self.x_rows, self.x_cols = X.MxMatrix(BATCH, inputs), X.MxMatrix(inputs, BATCH)
        self.d_rows, self.d_cols = X.MxMatrix(BATCH, outputs), X.MxMatrix(outputs, BATCH)
        self.y, self.dx = torch.empty(BATCH, outputs, device=DEV), torch.empty(BATCH, inputs, device=DEV)

    def forward(self, x):
        self.mx.mc_mx_quantize(self.model, self.w_rows, self.w_cols)
        self.mx.mc_mx_quantize(x, self.x_rows, self.x_cols)
        self.mx.mc_mx_matmul(self.x_rows, self.w_rows, self.y, bias=self.bias)
        return self.y

    def backward(self, dy, first):
        self.mx.mc_mx_quantize(dy, self.d_rows, self.d_cols)
        self.mx.mc_mx_matmul(self.d_cols, self.x_cols, self.dweight)
        torch.sum(dy, 0, out=self.dbias)
        if not first:
            self.mx.mc_mx_matmul(self.d_rows, self.w_cols, self.dx)
        return self.dx


class Training:
    """The model, its optimizer's lists and the scratch of the calls."""

    def __init__(self, seed=0):
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(seed)
        self.mx, self.loss = X.Mx(), S.PolicyLoss()
        self.layers = [Layer(self.mx, a, b, self.gen) for a, b in zip(SIZES[:-1], SIZES[1:])]
        both = lambda a, b: [t for l in self.layers[::-1] for t in (getattr(l, a).view(-1), getattr(l, b))]  # noqa: E731
        params, grads, model = both("weight", "bias"), both("dweight", "dbias"), both("model", "bias_model")
        numel, still = [p.numel() for p in params], [False, True] * len(self.layers)
        self.norm_of = S.Step(numel)
        self.norm_of.bind(grads=grads)
        self.update = X.Step8(numel, model_dtype="bfloat16", no_decay=still)
        self.moments = self.update.moments()
        self.update.bind(params=params, grads=grads, model=model, **self.moments)
        self.norm, self.sums = torch.empty(2, device=DEV), torch.empty(8, device=DEV)
        self.logp, self.slopes = torch.empty(BATCH, device=DEV), torch.empty(BATCH, SIZES[-1], device=DEV)
        self.ones, self.weights = torch.ones(BATCH, device=DEV), torch.full((BATCH,), 1.0 / BATCH, device=DEV)
        self.steps = 0

    def gradients(self, x, labels):
        """Logits, and the gradients in the layers' dweight and dbias."""
        for i, layer in enumerate(self.layers):
            x = layer.forward(x)
            if i + 1 < len(self.layers):
                x = torch.relu(x)
        self.loss.mc_token_logp(x, labels, self.logp)
        self.loss.mc_policy_loss(x, labels, self.logp, self.ones, sums=self.sums, weights=self.weights, dlogits=self.slopes)
        dy = self.slopes
        for i in range(len(self.layers) - 1, -1, -1):
            dy = self.layers[i].backward(dy, i == 0)
            if i:
                dy = torch.where(self.layers[i - 1].y > 0, dy, 0.0)
        return x

    def step(self, x, labels):
        logits = self.gradients(x, labels)
        self.steps += 1
        self.norm_of.mc_grad_norm(MAX_NORM, self.norm)
        self.update.mc_adamw8(self.steps, LR, BETAS, weight_decay=DECAY, coef=self.norm[1:])
        return logits

    def close(self):
        for handle in (self.mx, self.loss, self.norm_of, self.update):
            handle.close()


def train(steps=200, seed=0, log=lambda line: None):
    """Accuracy and mean log-probability of every step's samples."""
    t = Training(seed)
    teacher = torch.randn(SIZES[0], SIZES[-1], device=DEV, generator=t.gen)
    history = []
    for i in range(steps):
        x = torch.randn(BATCH, SIZES[0], device=DEV, generator=t.gen)
        labels = (x @ teacher).argmax(1)
        logits = t.step(x, labels)
        history.append((float((logits.argmax(1) == labels).float().mean()), float(t.logp.mean())))
        if i % 20 == 19:
            log(f"step {i + 1}: accuracy {history[-1][0]:.3f}, log-probability {history[-1][1]:.3f}, norm {float(t.norm[0]):.3f}")
    t.close()
    return history


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=200)
    train(parser.parse_args().steps, log=print)
