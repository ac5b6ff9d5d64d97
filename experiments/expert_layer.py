"""A router and experts in 8-bit block-scaled products, trained for a few steps and then served token by token, also with weights in 4 bits: the
calls of `experts`, `scaled`, `packed` and `orthogonal` together, timed.  Synthetic data; the target is another, random layer.

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
    router, of_target = (torch.randn((a.width, a.experts), generator=r, device="cuda") * a.width ** -0.5 for _ in range(2))

    def ms(f):
        s, e = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        s.record()
        out = f()
        e.record()
        e.synchronize()
        return out, s.elapsed_time(e)

    for step in range(a.steps):
        x = torch.randn((a.tokens, a.width), generator=r, device="cuda").bfloat16()
        chosen = experts.choose(h, x.float() @ of_target, a.topk, balance=False)
        want = target.serve(x, chosen.ids, chosen.weights)
        scores = x.float() @ router
        choice, choosing = ms(lambda: experts.choose(h, scores, a.topk))
        (y, kept), forward = ms(lambda: layer.forward(x, choice.ids, choice.weights))
        dy = (y - want) * (2.0 / a.tokens / a.width)
        (_, dp, dw1, dw2), backward = ms(lambda: layer.backward(dy, kept))
        router -= 0.3 * (x.float().T @ experts.choose_backward(h, scores, choice, dp, 0.01))
        loss = (y.float() - want.float()).square().mean().item()
        _, update = ms(lambda: layer.update(dw1, dw2, 0.05))
        if step % 5 == 0 or step == a.steps - 1:
            print("step %2d  loss %.4f  balance %.3f  choice %.3f ms  forward %.3f ms  backward %.3f ms  update, weights to 8 bits %.3f ms"
                  % (step, loss, choice.loss.item(), choosing, forward, backward, update), flush=True)
    layer.pack_weights()
    for tokens in (1, 8, 64):
        x = torch.randn((tokens, a.width), generator=r, device="cuda").bfloat16()
        for name, serve in (("8", layer.serve), ("4", layer.serve_packed)):
            def token():
                c = experts.choose(h, x.float() @ router, a.topk, balance=False)
                return serve(x, c.ids, c.weights)
            for _ in range(3):
                token()
            _, t = ms(lambda: [token() for _ in range(50)])
            print("serving %2d token(s), weights in %s bits: %.1f us a step" % (tokens, name, t * 20))
    h.close()


if __name__ == "__main__":
    main()
