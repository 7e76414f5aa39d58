#!/usr/bin/env python3
"""An image network from pixels to answers: the 13-layer VGG-16 convolution stack (F(m x m, 3 x 3), ReLU and max-pool fused), the three fully connected
layers behind it with 4-bit weights, and the log probabilities of the 1000 classes with their entropy and the best five; then the gradient of
the answers' log probabilities back through the three layers to the features, as adapters or a saliency map take it.  Random He-normal weights, N(0,1)
images, binary16.

    python vgg16_classify.py [--m 8] [--batch 32] [--points nova] [--group 128] [--reps 10]

Prints one JSON line: times of the stack, the layers, the log probabilities and the gradient, of one image or a batch; the whole forward pass as calls and as one
graph.
"""
import argparse
import json
import os
import sys

import torch

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2512_18453_amd import nova, synth  # noqa: E402

DEV = "cuda:0"
CLASSES, HIDDEN, TOP = 1000, 4096, 5


def he_normal(gen, outputs, *inputs):
    fan_in = 1
    for n in inputs:
        fan_in *= n
    return (torch.randn((outputs,) + inputs, device=DEV, generator=gen) * (2.0 / fan_in) ** 0.5).half()


class Stack:
    """The convolutions: transformed filters, one workspace, one output per layer."""

    def __init__(self, gen, batch, size, m, points):
        self.t = nova.nova_make_transforms(synth.point_set(points, m), m, 3)
        self.layers, bytes_needed = [], 0
        for idx, (cin, cout) in enumerate(synth.VGG16_LAYERS, start=1):
            flags = nova.NOVA_FLAG_RELU | (nova.NOVA_FLAG_POOL2 if idx in synth.VGG16_POOL_AFTER else 0)
            out = size // 2 if flags & nova.NOVA_FLAG_POOL2 else size
            bytes_needed = max(bytes_needed, nova.nova_conv2d_workspace_bytes(batch, cin, size, size, cout, m, nova.NOVA_F16, flags))
            y = torch.empty((batch, cout, out, out), dtype=torch.float16, device=DEV)
            self.layers.append((nova.nova_filter_transform(self.t, he_normal(gen, cout, cin, 3, 3)), cout, y, flags))
            size = out
        self.features = cout * size * size
        self.workspace = torch.empty(bytes_needed, dtype=torch.uint8, device=DEV)

    def __call__(self, x):
        for U, cout, y, flags in self.layers:
            x = nova.nova_winograd_conv2d(self.t, x, U, cout, y=y, flags=flags, workspace=self.workspace)
        return x.view(x.shape[0], -1)


class Head:
    """The fully connected layers in 4 bits, laid out for both directions, and the log probabilities."""

    def __init__(self, gen, batch, features, group):
        self.group, self.layers = group, []
        sizes = [features, HIDDEN, HIDDEN, CLASSES]
        for i, (K, N) in enumerate(zip(sizes, sizes[1:])):
            w = he_normal(gen, N, K)
            forward, backward = (nova.nova_q4_quantize(w, group, d) for d in (nova.NOVA_Q4_FORWARD, nova.NOVA_Q4_BACKWARD))
            y, dx = (torch.empty((batch, n), dtype=torch.float16, device=DEV) for n in (N, K))
            need = max(nova.nova_q4_linear_workspace_bytes(batch, N, K, group, torch.float16, d) for d in (nova.NOVA_Q4_FORWARD, nova.NOVA_Q4_BACKWARD))
            self.layers.append(dict(N=N, K=K, forward=forward, backward=backward, bias=(0.1 * torch.randn(N, device=DEV, generator=gen)).half(), y=y, dx=dx,
                                    flags=nova.NOVA_FLAG_RELU if i < 2 else 0, workspace=torch.empty(need, dtype=torch.uint8, device=DEV)))
        self.workspace = torch.empty(nova.nova_logprobs_workspace_bytes(batch, CLASSES, TOP, torch.float16), dtype=torch.uint8, device=DEV)
        self.dlogits = torch.empty((batch, CLASSES), dtype=torch.float16, device=DEV)

    def logits(self, x):
        for L in self.layers:
            x = nova.nova_q4_linear(x, L["forward"], L["N"], self.group, bias=L["bias"], y=L["y"], flags=L["flags"], workspace=L["workspace"])
        return x

    def answers(self, logits, labels):
        return nova.nova_logprobs(logits, labels, top=TOP, workspace=self.workspace)

    def gradient(self, logits, labels, answers, g_logprob):
        d = nova.nova_logprobs_backward(logits, answers.stats, labels, g_logprob=g_logprob, dlogits=self.dlogits)
        for L in reversed(self.layers):
            d = nova.nova_q4_linear_backward(d, L["backward"], L["K"], self.group, y=L["y"] if L["flags"] else None, dx=L["dx"], workspace=L["workspace"])
        return d


def timed(f, reps):
    for _ in range(3):
        f()
    torch.cuda.synchronize()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(reps):
        f()
    end.record()
    torch.cuda.synchronize()
    return round(start.elapsed_time(end) / reps, 4)


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--m", type=int, default=8, choices=(2, 4, 6, 8))
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--size", type=int, default=224)
    ap.add_argument("--points", default="nova")
    ap.add_argument("--group", type=int, default=128, choices=(32, 64, 128))
    ap.add_argument("--reps", type=int, default=10)
    args = ap.parse_args(argv)
    gen = torch.Generator(device=DEV).manual_seed(16)
    images = torch.randn((args.batch, 3, args.size, args.size), device=DEV, generator=gen).half()
    labels = torch.randint(0, CLASSES, (args.batch,), device=DEV, generator=gen)
    stack = Stack(gen, args.batch, args.size, args.m, args.points)
    head = Head(gen, args.batch, stack.features, args.group)
    g = torch.full((args.batch,), -1.0 / args.batch, device=DEV)            # of the mean negative log probability

    def forward():
        return head.answers(head.logits(stack(images)), labels)
    features = stack(images)
    logits = head.logits(features)
    answers = head.answers(logits, labels)
    gradient = head.gradient(logits, labels, answers, g)
    times = dict(stack=timed(lambda: stack(images), args.reps), layers=timed(lambda: head.logits(features), args.reps),
                 log_probabilities=timed(lambda: head.answers(logits, labels), args.reps),
                 gradient=timed(lambda: head.gradient(logits, labels, answers, g), args.reps), forward=timed(forward, args.reps))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = forward()
    times["forward_as_graph"] = timed(graph.replay, args.reps)
    print(json.dumps({
        "workload": f"VGG-16, batch {args.batch}, {args.size}x{args.size}, F({args.m},3), {args.points} points, fp16; fully connected layers in 4 bits, groups of {args.group}",
        "ms": times, "entropy": round(answers.entropy.mean().item(), 4), "log_probability": round(answers.logprob.mean().item(), 4),
        "best_of_first_image": answers.top_ids[0].tolist(), "finite": bool(torch.isfinite(gradient).all().item()),
    }))
    return dict(features=features, logits=logits, labels=labels, answers=answers, gradient=gradient, replayed=replayed, head=head, g=g)


if __name__ == "__main__":
    main()
