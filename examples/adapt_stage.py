"""Tunes what surrounds two frozen int8 convolutions against a teacher's top logits.

Two 3x3 layers of a quantized network stay as they are; between them a group norm with ReLU hands on int8 activations.
Behind them a group norm with SiLU, whose weight and bias are trained, then a shared projection to the classes with a
low-rank adapter for each of four tasks, trained as well, their images mixed in one batch.  The loss is the divergence
from ten stored logits of a teacher, with the rest of its mass as one more outcome.

    python examples/adapt_stage.py [steps]

needs the built library and a GPU, and prints the loss.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2407_02913_amd import adapt, binding, layers, synth  # noqa: E402

IMAGES, CHANNELS, EDGE, GROUPS = 64, 64, 14, 8
CLASSES, TASKS, RANK, TOP, TEMPERATURE = 1000, 4, 8, 10, 2.0


class Stage:
    """The frozen part: int8 maps in, float32 planes out."""

    def __init__(self):
        shape = synth.LayerShape("stage", IMAGES, CHANNELS, CHANNELS, EDGE, EDGE, "relu", True, 3)
        data = [synth.make_layer(shape, extra=k) for k in range(2)]
        self.convs = [layers.Layer(shape, d, out="f32") for d in data]
        self.x = torch.from_numpy(data[0]["x"]).cuda()
        self.workspace = binding.device_buffer(max(c.workspace_bytes for c in self.convs))
        g = torch.Generator(device="cuda").manual_seed(1)
        self.weight = 1 + 0.1 * torch.randn(CHANNELS, generator=g, device="cuda")
        self.bias = 0.1 * torch.randn(CHANNELS, generator=g, device="cuda")

    def __call__(self, x):
        first, second = self.convs
        y = first.new_output()
        first.run(x, y, self.workspace)
        # the next layer's activations, at the scale it was calibrated for
        q = adapt.group_norm_i8(y, GROUPS, self.weight, self.bias, activation="relu", y_scale=second.x_scale)
        z = second.new_output()
        second.run(q, z, self.workspace)
        return z

    def close(self):
        for c in self.convs:
            c.close()


def head(maps, tasks, p):
    """Logits of each image by its task's adapter."""
    z = adapt.group_norm(maps, GROUPS, p["weight"], p["bias"], activation="silu")
    features = z.mean((2, 3))
    return adapt.adapters(features @ p["shared"].t(), features, tasks, p["down"], p["up"], p["scale"])


def parameters(seed, spread):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    shared = torch.randn(CLASSES, CHANNELS, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda")
    return {"weight": 1 + spread * 0.3 * normal(CHANNELS), "bias": spread * 0.3 * normal(CHANNELS), "shared": shared,
            "down": normal(TASKS, RANK, CHANNELS) * CHANNELS ** -0.5, "up": spread * normal(TASKS, CLASSES, RANK),
            "scale": torch.full((TASKS,), 1.0, device="cuda")}


def main(steps=60):
    stage = Stage()
    maps = stage(stage.x)
    tasks = (torch.arange(IMAGES, device="cuda") * TASKS // IMAGES).to(torch.int32)
    with torch.no_grad():  # the teacher, of whom ten logits an image are stored
        log_p = torch.log_softmax(head(maps, tasks, parameters(7, 1.0)) / TEMPERATURE, 1)
        values, index = torch.topk(log_p, TOP, 1)
    p = parameters(3, 0.0)  # adapters that add nothing yet, a plain norm
    trained = [p[k].requires_grad_(True) for k in ("weight", "bias", "down", "up")]
    optimizer = torch.optim.Adam(trained, lr=0.03)
    losses = []
    for _ in range(steps):
        optimizer.zero_grad(set_to_none=True)
        loss = adapt.distill(head(maps, tasks, p), values, index, temperature=TEMPERATURE, tail=True).mean()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    stage.close()
    return losses


if __name__ == "__main__":
    curve = main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    for k in range(0, len(curve), max(1, len(curve) // 6)):
        print(f"step {k:4d}  loss {curve[k]:.4f}")
    print(f"step {len(curve) - 1:4d}  loss {curve[-1]:.4f}")
