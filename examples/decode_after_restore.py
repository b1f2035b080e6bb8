"""One attention layer over a paged 8-bit cache whose prefix comes back from its objects: append, attend, save, restore, go on.

Two sequences' prompts are appended to e4m3 blocks in chunks (tutti_kv_append, rotated by their places) while each chunk's queries
attend over what is there (tutti_kv_attend).  The blocks are saved as one layer's objects (tutti_layer_save), and so are their scales,
whose planes are a second pool with blocks of `stride` floats.  Both are restored into other blocks (tutti_layer_restore), and
the sequences go on token by token, there and in the blocks they came from: the results are the same to the last bit.

    python examples/decode_after_restore.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_03375_amd import binding as B  # noqa: E402

T, H, HQ, D = 16, 8, 32, 128          # block tokens, KV heads, query heads, head size
STAGE_ADDR, SGL_ID = 1 << 40, 3


def angles(positions, device):
    half = D // 2
    a = torch.arange(positions, dtype=torch.float64, device=device).unsqueeze(1)
    a = a * 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
    return torch.cat([a.cos(), a.sin()], 1).float()


class Cache:
    """A pool of e4m3 blocks with its scales, and where the sequences' blocks are."""

    def __init__(self, blocks, table, device):
        self.codes = [torch.zeros(blocks * T * H * D, dtype=torch.uint8, device=device) for _ in range(2)]
        self.scale = [torch.zeros(blocks, H, device=device) for _ in range(2)]       # rows of 32 bytes
        self.pool = B.make_pool(*self.codes, num_blocks=blocks, block_tokens=T, num_kv_heads=H, head_dim=D, elt_bytes=1)
        self.scales = B.make_scales(*self.scale)
        # the same planes of scales as blocks that the object calls move: one "token" of H values of 4 bytes
        self.scale_pool = B.make_pool(*self.scale, num_blocks=blocks, block_tokens=1, num_kv_heads=1, head_dim=H, elt_bytes=4)
        self.table = table


class Layer:
    """Appends a step's tokens and attends; `cache` says where."""

    def __init__(self, cos_sin, device):
        self.rope = B.make_rope(cos_sin, D)
        self.attn = B.make_attn(HQ, B.BF16, 1.0 / math.sqrt(D))
        self.device, self.work = device, None

    def step(self, cache, qkv, new, held, table_off):
        """qkv [rows, HQ + 2H, D] of all sequences' new tokens, sequence after sequence; held: tokens with the new ones."""
        row0 = [sum(new[:i]) for i in range(len(new))]
        seqs = torch.tensor(list(zip(row0, new, held, table_off)), dtype=torch.int32, device=self.device)
        batch = B.make_batch(seqs, len(new), max(new), cache.table, cache.table.numel(), qkv.shape[0])
        q = torch.empty(qkv.shape[0], HQ, D, dtype=qkv.dtype, device=self.device)
        out = torch.empty_like(q)
        status = torch.zeros(1, dtype=torch.int32, device=self.device)
        need = B.tutti_kv_attend_work_bytes(cache.pool, batch, self.attn)
        if self.work is None or self.work.numel() < need:
            self.work = torch.empty(need, dtype=torch.uint8, device=self.device)
        B.tutti_kv_append(cache.pool, cache.scales, batch, self.rope, B.make_rows(qkv[:, :HQ]), B.make_rows(q),
                          B.make_rows(qkv[:, HQ:HQ + H]), B.make_rows(qkv[:, HQ + H:]), HQ, B.BF16, status)
        B.tutti_kv_attend(cache.pool, cache.scales, batch, self.attn, B.make_rows(q), B.make_rows(out), None, self.work,
                          self.work.numel(), status)
        assert int(status.item()) == 0
        return out


def move(pool, n_blocks, table, stage, device, save):
    """The blocks of a layer's sequences to their objects in `stage`, or back."""
    n = len(n_blocks)
    cfg = B.make_cfg(4096, 2 << 20, 1)
    d_n, files = (torch.tensor(x, dtype=torch.int32, device=device) for x in (n_blocks, list(range(n))))
    extents = torch.zeros(32 * n, dtype=torch.uint8, device=device)
    totals = torch.zeros(2, dtype=torch.int64, device=device)
    entries = torch.zeros(64 * 64, dtype=torch.uint8, device=device)
    status = torch.zeros(1, dtype=torch.int32, device=device)
    call = B.tutti_layer_save if save else B.tutti_layer_restore
    call(pool, cfg, d_n, n, table, table.numel(), files, 0, stage, stage.numel(), STAGE_ADDR, SGL_ID, extents, totals, entries, 64, 0,
         status)
    assert int(status.item()) == 0


def run(prompts=(700, 333), chunk=256, steps=20, seed=0, device="cuda:0"):
    """Outputs of the decoded tokens where the prompts were, and where they were restored: two tensors [steps, sequences, HQ, D]."""
    torch.cuda.set_device(device)
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    n_seq, most = len(prompts), [p + steps for p in prompts]
    need = [-(-m // T) for m in most]
    off = [sum(need[:i]) for i in range(n_seq)]
    blocks = 2 * sum(need) + 5
    order = torch.randperm(blocks, generator=gen, device=device).to(torch.int32)
    here, there = Cache(blocks, order[:sum(need)], device), Cache(blocks, order[sum(need):2 * sum(need)], device)
    layer = Layer(angles(max(most), device), device)

    def qkv(rows):
        return torch.randn(rows, HQ + 2 * H, D, generator=gen, device=device).to(torch.bfloat16)

    held = [0] * n_seq
    while any(h < p for h, p in zip(held, prompts)):         # the prompts, chunk by chunk
        new = [min(chunk, p - h) for h, p in zip(held, prompts)]
        held = [h + n for h, n in zip(held, new)]
        layer.step(here, qkv(sum(new)), new, held, off)

    full = [-(-p // T) for p in prompts]                     # blocks that hold something
    table = {}
    for name, cache in (("here", here), ("there", there)):
        table[name] = torch.cat([cache.table[o:o + f] for o, f in zip(off, full)])
    for pool, size in (("pool", T * H * D), ("scale_pool", 4 * H)):
        stage = torch.zeros(sum(2 * -(-f * size // 4096) * 4096 for f in full), dtype=torch.uint8, device=device)
        move(getattr(here, pool), full, table["here"], stage, device, save=True)
        move(getattr(there, pool), full, table["there"], stage, device, save=False)

    got = [[], []]
    for _ in range(steps):
        held = [h + 1 for h in held]
        x = qkv(n_seq)
        for i, cache in enumerate((here, there)):
            got[i].append(layer.step(cache, x, [1] * n_seq, held, off))
    return torch.stack(got[0]), torch.stack(got[1])


if __name__ == "__main__":
    a, b = run()
    assert torch.equal(a, b)
    print(f"{a.shape[0]} steps of {a.shape[1]} sequences over a restored prefix: the same as where the prefix was, "
          f"|out| up to {float(a.float().abs().max()):.3f}")
