"""A student that reads records at a low scan group learns from a teacher that reads all of them.

One decode gives the student's pictures, an upgrade on top of it the teacher's.  Both go through a small transformer encoder: patch rows with their
positions (patch_rows), attention within each picture whose queries and keys are normalised and turned by row and column (norm_rotate), a mean and a
linear layer over the classes.  The teacher keeps its top logits; the student's loss is taken against these and the record's labels (distill_loss).

    python examples/distill_fidelity.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1911_00472_amd as pcr  # noqa: E402
import pcrgen  # noqa: E402

MEAN, INV_STD = (0.485, 0.456, 0.406), (1 / 0.229, 1 / 0.224, 1 / 0.225)
PATCH, WIDTH, HEADS, DIM, CLASSES, TOP = 16, 128, 4, 32, 100, 8
LOW, FULL = 2, 10                                          # scan groups


class Encoder(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.embed = torch.nn.Linear(3 * PATCH * PATCH, WIDTH)
        self.qkv = torch.nn.Linear(WIDTH, 3 * HEADS * DIM)
        self.q_weight = torch.nn.Parameter(torch.ones(DIM))
        self.k_weight = torch.nn.Parameter(torch.ones(DIM))
        self.out = torch.nn.Linear(HEADS * DIM, WIDTH)
        self.classes = torch.nn.Linear(WIDTH, CLASSES)
        # positions are (frame, row, column): no pair goes to the frame of a single picture, half of them to each of the others
        frequency, axis = pcr.axis_frequencies((0, DIM // 4, DIM // 4), 100.0, each=True)
        self.register_buffer("frequency", frequency)
        self.register_buffer("axis", axis)

    def forward(self, rows, positions, bounds):
        x = self.embed(rows)
        q, k, v = self.qkv(x).unflatten(-1, (3, HEADS, DIM)).unbind(1)      # [rows, heads, dim], views of one projection's output
        q, k = pcr.norm_rotate(q, k, self.q_weight, self.k_weight, positions, self.frequency, self.axis)
        mixed = []
        for a, b in zip(bounds[:-1], bounds[1:]):                           # a picture at a time
            weight = torch.softmax(torch.matmul(q[a:b].transpose(0, 1), k[a:b].permute(1, 2, 0).contiguous()) * DIM ** -0.5, -1)
            mixed.append(torch.matmul(weight, v[a:b].transpose(0, 1).contiguous()).transpose(0, 1).flatten(1))
        x = x + self.out(torch.cat(mixed))
        return self.classes(torch.stack([x[a:b].mean(0) for a, b in zip(bounds[:-1], bounds[1:])]))


def run(steps=40, images=48, say=print):
    """The student's mean loss of every step."""
    torch.manual_seed(0)
    data = pcrgen.make_workload("imagenet_like", limit=images)[0][0]
    teacher, student = Encoder().cuda().requires_grad_(False), Encoder().cuda()
    with torch.no_grad():
        teacher.classes.weight.mul_(8)                     # (a teacher with opinions)
    train = torch.optim.AdamW(student.parameters(), 2e-3)
    losses = []
    with pcr.pcr_open(data, 0) as record:
        layout = record.patch_layout(PATCH)
        bounds = layout[2].tolist()
        labels = torch.tensor([record.image_info(i)[3] % CLASSES for i in range(record.n)], device="cuda")
        low = pcr.patch_rows(record.decode_batch(LOW), *layout, PATCH, MEAN, INV_STD, dtype=torch.float32)
        full = pcr.patch_rows(record.upgrade_batch(FULL), *layout, PATCH, MEAN, INV_STD, dtype=torch.float32)
        with torch.no_grad():
            top_logits, top_index = teacher(*full, bounds).topk(TOP, 1)
        for step in range(steps):
            logits = student(*low, bounds)
            loss = pcr.distill_loss(logits, top_index, top_logits, labels, temperature=2.0, distill_part=0.9, label_part=0.1).mean()
            train.zero_grad()
            loss.backward()
            train.step()
            losses.append(loss.detach().item())
            if step % 10 == 0 or step == steps - 1:
                say("step %3d   loss %.4f" % (step, losses[-1]))
    return losses


if __name__ == "__main__":
    run(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
