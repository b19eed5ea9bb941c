"""A training loop on distances: labelling images from one mark in each object.

Every image shows bright discs on noise; a user has put one mark (a pixel) into each of them.  A small network labels
the pixels as object or background:

  - attention over image patches, with a learned bias by the distance between two patches (``relative_bias``);
  - a learned prior by the distance to the nearest mark (``distance_transform_edt``, then ``distance_bias``), added to
    the logits;
  - a loss of the labels' log-probabilities and of the expected signed distance of each class
    (``signed_distance_transform``, then ``label_log_probs``): probability far on the wrong side of a border costs more.

    python examples/train_marks.py [--steps 60] [--batch 8] [--size 128]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_24738_amd import binding, training  # noqa: E402

PATCH = 8


def make_images(gen, batch, size, count=3):
    """(images, labels, marks): labels 1 inside the discs, marks 0 at each disc's centre and 1 elsewhere."""
    dev = gen.device
    axis = torch.arange(size, device=dev)
    labels = torch.zeros((batch, size, size), dtype=torch.uint8, device=dev)
    marks = torch.ones((batch, 1, size, size), dtype=torch.uint8, device=dev)
    for _ in range(count):
        radius = (0.06 + 0.1 * torch.rand(batch, generator=gen, device=dev)) * size
        y = torch.randint(size // 8, size - size // 8, (batch,), generator=gen, device=dev)
        x = torch.randint(size // 8, size - size // 8, (batch,), generator=gen, device=dev)
        square = (axis[None, :, None] - y[:, None, None]) ** 2 + (axis[None, None, :] - x[:, None, None]) ** 2
        labels |= (square <= (radius * radius)[:, None, None]).to(torch.uint8)
        marks[torch.arange(batch, device=dev), 0, y, x] = 0
    images = labels[:, None].float() + torch.randn((batch, 1, size, size), generator=gen, device=dev)
    return images, labels, marks


class Network(torch.nn.Module):
    def __init__(self, size, width=32, heads=4, buckets=16):
        super().__init__()
        self.heads, self.grid = heads, (size // PATCH, size // PATCH)
        self.embed = torch.nn.Linear(PATCH * PATCH, width)
        self.qkv = torch.nn.Linear(width, 3 * width)
        self.decode = torch.nn.Linear(width, 2 * PATCH * PATCH)
        # learned by bucket of distance: between patches for each head, to the nearest mark for each class
        self.position = torch.nn.Parameter(torch.zeros(buckets, heads))
        self.prior = torch.nn.Parameter(torch.zeros(buckets, 2))
        self.register_buffer("patch_edges", training.distance_edges(buckets, size / PATCH))
        self.register_buffer("mark_edges", training.distance_edges(buckets, size / 2))

    def forward(self, images, marks):
        b, _, n, _ = images.shape
        gh, gw = self.grid
        patches = images.reshape(b, gh, PATCH, gw, PATCH).transpose(2, 3).reshape(b, gh * gw, PATCH * PATCH)
        x = self.embed(patches)
        q, k, v = self.qkv(x).reshape(b, gh * gw, 3, self.heads, -1).permute(2, 0, 3, 1, 4).unbind(0)
        scores = q @ k.transpose(-1, -2).contiguous() * q.shape[-1] ** -0.5
        scores = training.relative_bias(self.position, self.patch_edges, self.grid, self.grid, add=scores)
        x = x + (scores.softmax(-1) @ v).transpose(1, 2).reshape(b, gh * gw, -1)
        logits = self.decode(x).reshape(b, gh, gw, 2, PATCH, PATCH).permute(0, 3, 1, 4, 2, 5).reshape(b, 2, n, n)
        distance = binding.distance_transform_edt(marks)[:, 0]
        return training.distance_bias(distance, self.prior, self.mark_edges, add=logits.contiguous())


def losses(logits, labels):
    """(label loss, boundary loss, mean entropy).  The signed distance is positive inside, so an expected value of the
    true class's field as large as possible keeps the border in place."""
    inside = binding.signed_distance_transform(labels[:, None])
    field = torch.cat([-inside, inside], 1)
    got = training.label_log_probs(logits, labels, entropy=True, field=field)
    return -got.log_probs.mean(), -got.field_mean.mean(), got.entropy.mean()


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--batch", type=int, default=8)
    parser.add_argument("--size", type=int, default=128)
    parser.add_argument("--quiet", action="store_true")
    args = parser.parse_args(argv)
    if args.size % PATCH:
        parser.error("--size must be a multiple of %d" % PATCH)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(0)
    torch.manual_seed(0)
    network = Network(args.size).to(dev)
    optimizer = torch.optim.Adam(network.parameters(), lr=0.01)
    history = []
    for step in range(args.steps):
        images, labels, marks = make_images(gen, args.batch, args.size)
        label_loss, boundary_loss, entropy = losses(network(images, marks), labels)
        optimizer.zero_grad(set_to_none=True)
        # with one GPU, handing a pass over to autograd's own thread and back takes longer than its launches
        with torch.autograd.set_multithreading_enabled(False):
            (label_loss + 0.02 * boundary_loss).backward()
        optimizer.step()
        history.append(float(label_loss.detach()))
        if not args.quiet and step % 10 == 0:
            print("step %3d  label loss %.4f  boundary loss %8.3f  entropy %.4f" % (
                step, history[-1], float(boundary_loss.detach()), float(entropy.detach())), flush=True)
    with torch.no_grad():
        images, labels, marks = make_images(gen, args.batch, args.size)
        got = training.label_log_probs(network(images, marks), labels, top_k=1)
        right = float((got.top_indices[:, 0] == labels).float().mean())
    if not args.quiet:
        print("pixels labelled as they are: %.1f %%" % (100 * right))
    return history, right, network


if __name__ == "__main__":
    main()
