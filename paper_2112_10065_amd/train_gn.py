"""A small group-normalised image classifier, trained and evaluated with this library's layers: the operators of a training step
as they are used together.

  python -m paper_2112_10065_amd.train_gn --steps 60 --batch 16 --state q8

  conv 3x3 (3 -> 32), group norm + ReLU, 2x2 max-pool, conv 3x3 (32 -> 64), group norm + SiLU, 2x2 max-pool, dense

The norm's statistics are those of one sample, so the network computes the same function at every per-GPU batch.  The first
norm's ReLU is differentiated by the layer behind it (DP_RELU_IN), so its backward call gets a masked gradient; the
second norm differentiates its own SiLU.  All parameters are in one list: one call for the norm of all gradients, one for the
AdamW step, which takes the clipping factor from device memory (and skips the step if a gradient is not finite).
Evaluation: log-probability of the label, entropy and the likeliest classes of each image.

Images are synthetic: one random pattern per class plus noise.  PyTorch supplies device memory and streams only.
"""
import argparse
import json
import math

import torch

from . import binding as dp

IMAGE, CHANNELS, GROUPS, EPS = 32, (3, 32, 64), 8, 1e-5


class GroupNormNet:
    def __init__(self, batch, classes, state=dp.DP_STATE_F32, lr=1e-3, weight_decay=0.05, max_norm=1.0, seed=0, device="cuda:0"):
        self.n, self.classes, self.lr, self.max_norm, self.steps, self.seed = batch, classes, lr, max_norm, 0, seed
        self.weight_decay = weight_decay
        dev = torch.device(device)
        gen = torch.Generator(dev).manual_seed(seed)
        bf, f32 = torch.bfloat16, torch.float32

        def empty(*shape, dtype=bf):
            return torch.empty(shape, dtype=dtype, device=dev)

        c0, c1, c2 = CHANNELS
        h1, h2, h3 = IMAGE, IMAGE // 2, IMAGE // 4
        feats = h3 * h3 * c2
        self.params = []

        def param(shape, scale, decays):
            w = torch.randn(shape, generator=gen, device=dev) * scale
            return self._add(w, decays, state)

        self.w1 = param((c1, 3, 3, c0), math.sqrt(2 / (9 * c0)), True)
        self.g1, self.b1 = self._add(torch.ones(c1, device=dev), False, state), self._add(torch.zeros(c1, device=dev), False, state)
        self.w2 = param((c2, 3, 3, c1), math.sqrt(2 / (9 * c1)), True)
        self.g2, self.b2 = self._add(torch.ones(c2, device=dev), False, state), self._add(torch.zeros(c2, device=dev), False, state)
        self.w3, self.b3 = param((classes, feats), math.sqrt(1 / feats), True), self._add(torch.zeros(classes, device=dev), False, state)
        self.list = dp.param_list([{k: v for k, v in p.items() if k != "view"} for p in self.params], state)

        self.conv1 = dp.conv_desc(batch, h1, h1, c0, c1, 3, 3, (1, 1), (1, 1), dp.DP_BF16, 0)
        # the input of the second convolution is a pooled ReLU output: its backward-data masks by it
        self.conv2 = dp.conv_desc(batch, h2, h2, c1, c2, 3, 3, (1, 1), (1, 1), dp.DP_BF16, dp.DP_RELU_IN)
        self.conv2_fwd = dp.conv_desc(batch, h2, h2, c1, c2, 3, 3, (1, 1), (1, 1), dp.DP_BF16, 0)
        self.norm1 = dp.group_norm_desc(batch, h1, h1, c1, GROUPS, dp.DP_BF16, dp.DP_RELU, EPS)
        self.norm2 = dp.group_norm_desc(batch, h2, h2, c2, GROUPS, dp.DP_BF16, dp.DP_SILU, EPS)
        self.dense = dp.linear_desc(batch, feats, classes, dp.DP_BF16, dp.DP_BIAS)
        self.scores = dp.logprobs_desc(batch, classes, min(5, classes), dp.DP_BF16)

        self.x = empty(batch, h1, h1, c0)
        self.u1, self.y1, self.p1 = empty(batch, h1, h1, c1), empty(batch, h1, h1, c1), empty(batch, h2, h2, c1)
        self.u2, self.y2, self.p2 = empty(batch, h2, h2, c2), empty(batch, h2, h2, c2), empty(batch, feats)
        self.z, self.dz, self.loss = empty(batch, classes), empty(batch, classes), empty(4, dtype=f32)
        self.du1, self.dp1 = torch.empty_like(self.u1), torch.empty_like(self.p1)
        self.du2, self.dp2 = torch.empty_like(self.u2), torch.empty_like(self.p2)
        self.mean1, self.rstd1, self.mean2, self.rstd2 = (empty(batch, GROUPS, dtype=f32) for _ in range(4))
        self.norm = empty(4, dtype=f32)
        k = min(5, classes)
        self.logp, self.entropy, self.lse = (empty(batch, dtype=f32) for _ in range(3))
        self.top_logp, self.top_ids = empty(batch, k, dtype=f32), empty(batch, k, dtype=torch.int32)
        need = [dp.dp_conv2d_workspace_bytes(d, p) for d in (self.conv1, self.conv2, self.conv2_fwd) for p in range(3)]
        need += [dp.dp_group_norm_workspace_bytes(d, p) for d in (self.norm1, self.norm2) for p in (dp.DP_PASS_FWD, dp.DP_PASS_DGRAD)]
        need += [dp.dp_linear_workspace_bytes(self.dense), dp.dp_grad_norm_workspace_bytes(self.list), dp.dp_logprobs_workspace_bytes(self.scores)]
        self.ws = torch.empty(max(need) + 256, dtype=torch.uint8, device=dev)

    def _add(self, w, decays, state):
        """A parameter with its gradient, bf16 copy and optimizer states; weights decay, norms and biases do not."""
        w = w.contiguous()
        flat = w.view(-1)
        q8 = state == dp.DP_STATE_Q8
        blocks = -(-flat.numel() // 256)
        p = dict(view=w, w32=flat, grad=torch.zeros_like(flat), w_bf16=flat.to(torch.bfloat16), weight_decay=self.weight_decay if decays else 0.0,
                 m=torch.zeros(flat.numel(), dtype=torch.uint8 if q8 else torch.float32, device=w.device))
        p["v"] = torch.zeros_like(p["m"])
        if q8:
            p["m_scale"], p["v_scale"] = (torch.zeros(blocks, device=w.device) for _ in range(2))
        self.params.append(p)
        return p

    def forward(self):
        n, ws = self.n, self.ws
        h1, h2 = IMAGE, IMAGE // 2
        dp.dp_conv2d_fwd(self.conv1, self.x, self.w1["w_bf16"], None, self.u1, ws)
        dp.dp_group_norm_fwd(self.norm1, self.u1, self.g1["w32"], self.b1["w32"], self.y1, self.mean1, self.rstd1, ws)
        dp.dp_maxpool2x2_fwd(n, h1, h1, CHANNELS[1], dp.DP_BF16, self.y1, self.p1)
        dp.dp_conv2d_fwd(self.conv2_fwd, self.p1, self.w2["w_bf16"], None, self.u2, ws)
        dp.dp_group_norm_fwd(self.norm2, self.u2, self.g2["w32"], self.b2["w32"], self.y2, self.mean2, self.rstd2, ws)
        dp.dp_maxpool2x2_fwd(n, h2, h2, CHANNELS[2], dp.DP_BF16, self.y2, self.p2)
        dp.dp_linear_fwd_bwd(self.dense, x=self.p2, W=self.w3["w_bf16"], bias=self.b3["w32"], y=self.z, ws=ws)

    def backward(self):
        """From self.dz to every parameter's gradient."""
        n, ws = self.n, self.ws
        h1, h2 = IMAGE, IMAGE // 2
        dp.dp_linear_fwd_bwd(self.dense, x=self.p2, W=self.w3["w_bf16"], dy=self.dz, dx=self.dp2, dW=self.w3["grad"], dbias=self.b3["grad"], ws=ws)
        dp.dp_maxpool2x2_bwd(n, h2, h2, CHANNELS[2], dp.DP_BF16, self.y2, self.dp2, self.du2)
        dp.dp_group_norm_bwd(self.norm2, self.u2, self.du2, None, self.g2["w32"], self.b2["w32"], self.mean2, self.rstd2, self.du2, self.g2["grad"],
                             self.b2["grad"], ws)
        dp.dp_conv2d_bwd_filter(self.conv2, self.p1, self.du2, None, self.w2["grad"], None, ws)
        dp.dp_conv2d_bwd_data_relu(self.conv2, self.du2, None, self.w2["w_bf16"], self.p1, self.dp1, ws)
        dp.dp_maxpool2x2_bwd(n, h1, h1, CHANNELS[1], dp.DP_BF16, self.y1, self.dp1, self.du1)
        dp.dp_group_norm_bwd(self.norm1, self.u1, self.du1, None, self.g1["w32"], self.b1["w32"], self.mean1, self.rstd1, self.du1, self.g1["grad"],
                             self.b1["grad"], ws)
        dp.dp_conv2d_bwd_filter(self.conv1, self.x, self.du1, None, self.w1["grad"], None, ws)

    def train_step(self, labels):
        """One step on self.x; the loss is in self.loss[0], the gradients' norm in self.norm[0], both on the device."""
        self.forward()
        dp.dp_softmax_xent(self.n, self.classes, dp.DP_BF16, self.z, labels, self.loss, self.dz)
        self.backward()
        self.steps += 1
        dp.dp_grad_norm(self.list, self.max_norm, self.norm, self.ws)
        hyper = dp.adamw_hyper(self.lr, step=self.steps, seed=self.seed + self.steps)
        dp.dp_adamw_step(self.list, hyper, self.norm[1:])

    def evaluate(self, labels):
        """Forward on self.x; log-probability of the labels, entropy and likeliest classes in self.logp, .entropy, .top_ids."""
        self.forward()
        dp.dp_logprobs_fwd(self.scores, self.z, labels, self.logp, self.entropy, self.lse, self.top_logp, self.top_ids, self.ws)


class Patterns:
    """Labelled images: a random pattern per class plus noise."""

    def __init__(self, classes, seed=0, device="cuda:0"):
        self.gen = torch.Generator(torch.device(device)).manual_seed(seed)
        self.device, self.classes = torch.device(device), classes
        self.proto = torch.randn((classes, IMAGE, IMAGE, CHANNELS[0]), generator=self.gen, device=self.device)

    def batch(self, n):
        labels = torch.randint(0, self.classes, (n,), generator=self.gen, device=self.device)
        x = self.proto[labels] + 0.7 * torch.randn((n, IMAGE, IMAGE, CHANNELS[0]), generator=self.gen, device=self.device)
        return x.to(torch.bfloat16), labels.to(torch.int32)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--classes", type=int, default=20)
    ap.add_argument("--state", choices=("f32", "q8"), default="f32", help="optimizer states in 32 or in 8 bits")
    ap.add_argument("--max-norm", type=float, default=1.0, help="clip the gradients' norm (inf: do not)")
    a = ap.parse_args(argv)
    net = GroupNormNet(a.batch, a.classes, dp.DP_STATE_Q8 if a.state == "q8" else dp.DP_STATE_F32, max_norm=a.max_norm)
    data = Patterns(a.classes)
    for step in range(1, a.steps + 1):
        x, labels = data.batch(a.batch)
        net.x.copy_(x)
        net.train_step(labels)
        if step == 1 or step % 20 == 0 or step == a.steps:
            print(f"step {step}: loss {float(net.loss[0]):.4f}, gradient norm {float(net.norm[0]):.3f}", flush=True)
    logp = entropy = top1 = top5 = 0.0
    rounds = 8
    for _ in range(rounds):
        x, labels = data.batch(a.batch)
        net.x.copy_(x)
        net.evaluate(labels)
        hit = net.top_ids == labels[:, None]
        logp, entropy = logp + float(net.logp.mean()) / rounds, entropy + float(net.entropy.mean()) / rounds
        top1, top5 = top1 + float(hit[:, 0].float().mean()) / rounds, top5 + float(hit.any(dim=1).float().mean()) / rounds
    result = {"steps": a.steps, "state": a.state, "loss": -logp, "entropy": entropy, "top1": top1, "top5": top5}
    print(json.dumps(result))
    return result


if __name__ == "__main__":
    main()
