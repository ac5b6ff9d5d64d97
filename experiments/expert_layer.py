"""Experts in 8-bit block-scaled products, trained for a few steps and then served token by token: the calls of `scaled` and
`experts` together, timed.  Synthetic data; the target is another, random layer.

    python experiments/expert_layer.py [--tokens 4096] [--width 2048] [--inner 1024] [--experts 16] [--topk 2] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_13778_amd import experts, ozdgemm  # noqa: E402


def main():
    p = argparse.ArgumentParser()
    for name, value in (("tokens", 4096), ("width", 2048), ("inner", 1024), ("experts", 16), ("topk", 2), ("steps", 20)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    h = ozdgemm.Handle(0)
    r = torch.Generator(device="cuda").manual_seed(1)

    def weights(scale):
        return [torch.randn(s, generator=r, device="cuda") * scale * s[-1] ** -0.5 for s in ((a.experts, a.inner, a.width), (a.experts, a.width, a.inner))]

    layer, target = experts.ExpertLayer(h, *weights(1.0)), experts.ExpertLayer(h, *weights(1.0))
    router = torch.randn((a.width, a.experts), generator=r, device="cuda") * a.width ** -0.5

    def route(x):
        top, ids = (x.float() @ router).topk(a.topk, dim=1)
        return ids, top.softmax(dim=1)

    def ms(f):
        s, e = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        s.record()
        out = f()
        e.record()
        e.synchronize()
        return out, s.elapsed_time(e)

    for step in range(a.steps):
        x = torch.randn((a.tokens, a.width), generator=r, device="cuda").bfloat16()
        ids, p = route(x)
        want = target.serve(x, ids, p)
        (y, kept), forward = ms(lambda: layer.forward(x, ids, p))
        dy = (y - want) * (2.0 / a.tokens)
        (_, _, dw1, dw2), backward = ms(lambda: layer.backward(dy, kept))
        loss = (y.float() - want.float()).square().sum(1).mean().item() / a.width
        for w, d in ((layer.w1, dw1), (layer.w2, dw2)):          # a step of 3 % of the weights' size down the gradient
            w -= d * (0.03 * w.norm() / d.norm())
        _, prepare = ms(layer.prepare_weights)
        if step % 5 == 0 or step == a.steps - 1:
            print("step %2d  loss %.4f  forward %.3f ms  backward %.3f ms  weights to 8 bits %.3f ms" % (step, loss, forward, backward, prepare), flush=True)
    for tokens in (1, 8, 64):
        x = torch.randn((tokens, a.width), generator=r, device="cuda").bfloat16()
        ids, w = route(x)
        for _ in range(3):
            layer.serve(x, ids, w)
        _, t = ms(lambda: [layer.serve(x, ids, w) for _ in range(50)])
        print("serving %2d token(s): %.1f us a step" % (tokens, t * 20))
    h.close()


if __name__ == "__main__":
    main()
