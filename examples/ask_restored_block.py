"""A block of text is read once, saved, restored into other pages, and asked a question.

The model is a toy with random weights (two layers, 8 query heads on 2 key heads of 64 dimensions); what it shows is
the order of the calls.  For every layer: gk_append writes the new tokens' keys and values behind those that are in the
cache and rotates the queries, gk_attention lets them attend to everything before them.  Between the two runs lie
gk_pack and gk_restore: the answer's states after restoring the block have the same bits as without.

    python examples/ask_restored_block.py [--fp8]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2609_39358_b200 as gk

LAYERS, HQ, H, D, T, WIDTH = 2, 8, 2, 64, 16, 512


def make_cache(pages: int, fp8: bool) -> gk.Cache:
    slab = T * H * D * (1 if fp8 else 2)
    data = torch.zeros(LAYERS * 2 * pages * slab, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(LAYERS, 2, pages, H, device="cuda") if fp8 else None
    return gk.Cache(data, pages, 2 * pages * slab, pages * slab, slab, scales, 8 * pages * H if fp8 else 0,
                    4 * pages * H if fp8 else 0, 4 * H if fp8 else 0)


class Toy:
    def __init__(self, ctx: gk.Context, rope: gk.Rope, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.rope = ctx, rope
        self.qkv = [(torch.randn(WIDTH, (HQ + 2 * H) * D, device="cuda", generator=g) / WIDTH ** 0.5).to(torch.bfloat16)
                    for _ in range(LAYERS)]
        self.out = [(torch.randn(HQ * D, WIDTH, device="cuda", generator=g) / (HQ * D) ** 0.5).to(torch.bfloat16)
                    for _ in range(LAYERS)]

    def forward(self, x: torch.Tensor, cache: gk.Cache, batch: gk.Batch) -> torch.Tensor:
        """x: the new tokens' states, [n_tokens, WIDTH]."""
        n = x.shape[0]
        for layer in range(LAYERS):
            qkv = (x @ self.qkv[layer]).view(n, HQ + 2 * H, D)
            q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:]
            self.ctx.gk_append(cache, layer, batch, k, v, q, None, self.rope)      # q is rotated in place
            y = torch.empty(n, HQ, D, dtype=torch.bfloat16, device="cuda")
            self.ctx.gk_attention(cache, layer, batch, q, y)
            x = x + y.view(n, HQ * D) @ self.out[layer]
        return x


def batch_of(pages: torch.Tensor, total: int, new: int) -> gk.Batch:
    return gk.Batch(pages[None], torch.tensor([total], dtype=torch.int32, device="cuda"),
                    torch.tensor([0, new], dtype=torch.int32, device="cuda"), new, new)


def main(fp8: bool = False, block: int = 333, question: int = 21, steps: int = 5) -> int:
    geom = gk.Geom(LAYERS, H, D, T, gk.GK_FP8_E4M3 if fp8 else gk.GK_BF16, 2 if fp8 else 0)
    with gk.Context(geom, 0) as ctx:
        angle = torch.arange(1024, device="cuda")[:, None] * 1e4 ** (-torch.arange(D // 2, device="cuda") / (D // 2))
        model = Toy(ctx, gk.Rope(torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()), 7)
        g = torch.Generator(device="cuda").manual_seed(1)
        states = torch.randn(block + question + steps, WIDTH, device="cuda", generator=g).to(torch.bfloat16)
        need = -(-(block + question + steps) // T)

        def ask(cache, pages):
            """The question behind the block, then single steps."""
            got = [model.forward(states[block:block + question], cache, batch_of(pages, block + question, question))]
            kv = torch.tensor([block + question], dtype=torch.int32, device="cuda")
            step = gk.Batch(pages[None], kv)
            for i in range(block + question, block + question + steps):
                kv += 1
                got.append(model.forward(states[i:i + 1], cache, step))
            return torch.cat(got)

        # read the block; save its record before the question is written behind it
        first, home = make_cache(64, fp8), torch.randperm(64, device="cuda")[:need].to(torch.int32)
        model.forward(states[:block], first, batch_of(home, block, block))
        n_bytes, n_pages = gk.gk_blob_size(geom, block)
        blob = torch.zeros(n_bytes, dtype=torch.uint8, device="cuda")
        sums = torch.zeros(n_pages, dtype=torch.int64, device="cuda")
        ctx.gk_pack(first, home, block, blob, sums)
        want = ask(first, home)

        # another cache, other pages
        second, away = make_cache(96, fp8), torch.randperm(96, device="cuda")[:need].to(torch.int32)
        mask, bad = torch.full((1,), 255, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        ctx.gk_restore([gk.Job(blob, sums, away, block)], second, mask, bad)
        got = ask(second, away)
        torch.cuda.synchronize()
        same = int(mask[0]) == gk.JOB_OK and torch.equal(want, got)
        print(f"{'fp8' if fp8 else 'bf16'}: {block} tokens restored, {question} asked, {steps} steps: "
              f"{'the same bits as without restoring' if same else 'DIFFERENT'}")
        return 0 if same and bool(torch.isfinite(want.float()).all()) else 1


if __name__ == "__main__":
    sys.exit(main("--fp8" in sys.argv))
