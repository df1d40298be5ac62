"""Generation after compression, layer by layer as a model runs it: at the end of prefill some layers' caches are compressed
(MixKV) and kept, the others are kept whole; both go into paged 4-bit caches that every new token's keys and values are
appended to.  Compressed layers attend over all of their pages, whole ones over the pages that the query selects.

    python examples/paged_decode.py [tokens]

Random keys, values and queries stand in for a model's projections.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_20707_b200 import binding  # noqa: E402

LAYERS, WHOLE = 4, (0, 3)          # layers of the model, and those whose cache is not compressed
H, G, L, BUDGET = 4, 7, 4096, 256
PAGE, TOP = 64, 16                 # rows of a page; pages that a whole layer's query reads


def rotation(length, dim=128, base=10000.0):
    angle = torch.arange(length, device="cuda").double().unsqueeze(1) * base ** (
        -torch.arange(dim // 2, device="cuda").double() / (dim // 2))
    return angle.cos().float(), angle.sin().float()


def prefill(gen):
    """Keys (rotated already), values and window queries of one layer."""
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    K = (rand(H, L, 128) + 0.8 * rand(H, 1, 128)).bfloat16()
    return K, rand(H, L, 128).bfloat16(), rand(1, H * G, 32, 128).bfloat16()


def build_caches(gen, tokens):
    params = binding.Params(kv_heads=H, gqa_ratio=G, budget=BUDGET, budget_mode=1)     # head-adaptive budgets
    caches, compact = [], []
    for layer in range(LAYERS):
        K, V, Q = prefill(gen)
        if layer in WHOLE:
            pages = binding.new_pages(1, H, L + tokens, PAGE, bounds=True)
            pages.rows += L
            offsets = torch.tensor([0, L], dtype=torch.int32, device="cuda")
            binding.paged_append(pages, K.transpose(0, 1), V.transpose(0, 1), offsets=offsets, max_new=L)
            compact.append(None)
        else:
            out = binding.compress_layer(K, V, Q, params)
            offsets = out["out_row_offsets"]
            most = H * BUDGET                                  # adaptive: a head may keep what others give up
            pages = binding.new_pages(1, H, most + tokens, PAGE)
            pages.rows += offsets.diff().view(1, H)
            binding.paged_append(pages, out["K_out"], out["V_out"], offsets=offsets, max_new=most)
            compact.append(out)
        caches.append(pages)
    return caches, compact


def decode(caches, gen, tokens):
    """`tokens` steps; returns the attention outputs of the last one, a tensor per layer."""
    cos, sin = rotation(L + tokens)
    most = [int(p.rows.max()) for p in caches]                 # (once; a step makes it one more)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    space = [binding.paged_workspace(p, rand(1, 1, H * G, 128)) for p in caches]
    outs = []
    for step in range(tokens):
        position = torch.tensor([L + step], dtype=torch.int32, device="cuda")     # in the sequence, not in the cache
        outs = []
        for layer, pages in enumerate(caches):
            q, k, v = rand(1, 1, H * G, 128), rand(1, H, 128), rand(1, H, 128)
            pages.rows += 1
            binding.paged_append(pages, k, v, cos=cos, sin=sin, positions=position, status=status)
            if layer in WHOLE:
                out, _, _ = binding.paged_sparse_attention(pages, q, TOP, most[layer] + step + 1, workspace=space[layer])
            else:
                out = binding.paged_attention(pages, q, most[layer] + step + 1, workspace=space[layer])
            outs.append(out)
    assert status.item() == 0
    return outs


def main(tokens=32):
    gen = torch.Generator(device="cuda").manual_seed(0)
    caches, compact = build_caches(gen, tokens)
    # how far 4 bits are from the compact rows themselves
    q = torch.randn((1, 1, H * G, 128), generator=gen, device="cuda").bfloat16()
    errors = []
    for layer, out in enumerate(compact):
        if out is not None:
            rows = int(out["out_row_offsets"].diff().max())
            full = binding.decode_attention(out["K_out"].unsqueeze(0), out["V_out"].unsqueeze(0),
                                            out["out_row_offsets"].unsqueeze(0), q, H, G, rows)
            four = binding.paged_attention(caches[layer], q).float()
            errors.append(((four - full).norm() / full.norm()).item())
    outs = decode(caches, gen, tokens)
    held = sum(p.pool.numel() for p in caches)
    print(f"{LAYERS} layers, {tokens} tokens; attention over 4 bits is {max(errors):.3f} off bf16 rows; "
          f"pools {held / 2 ** 20:.1f} MiB, a whole bf16 cache {LAYERS * H * (L + tokens) * 512 / 2 ** 20:.1f} MiB")
    return errors, outs


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 32)
