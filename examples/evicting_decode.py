"""Generation over a cache that stays small: the prompt's cache is compressed (MixKV), its rows go into a paged 8-bit cache, and from
then on every row keeps count of the attention it gets; whenever a head has outgrown its budget, the rows that got least are thrown
away.  One layer; the others of a model are the same.

    python examples/evicting_decode.py [tokens]

Random keys, values and queries stand in for a model's projections.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_20707_b200 import binding  # noqa: E402

H, G, L = 4, 7, 4096
BUDGET, SLACK, PAGE = 256, 16, 64         # rows of a head after an eviction, and how many more set off the next; rows of a page
SINKS, RECENT = 4, 32                     # rows that are kept whatever they got: the first, the newest


def compress(gen):
    """Keys, values and window queries of a prompt; of every head the rows that the compression keeps."""
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    K = (rand(H, L, 128) + 0.8 * rand(H, 1, 128)).bfloat16()
    params = binding.Params(kv_heads=H, gqa_ratio=G, budget=BUDGET)
    return binding.compress_layer(K, rand(H, L, 128).bfloat16(), rand(1, H * G, 32, 128).bfloat16(), params)


def main(tokens=200):
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    out = compress(gen)
    # two caches in turn: an eviction writes what it keeps to the pages of the other
    here, there = (binding.new_cache8(1, H, BUDGET + SLACK, PAGE, mass=True) for _ in range(2))
    here.rows += BUDGET
    binding.cache8_append(here, out["K_out"], out["V_out"], offsets=out["out_row_offsets"], max_new=BUDGET)
    q = rand(1, 1, H * G, 128)
    full = binding.decode_attention(out["K_out"].unsqueeze(0), out["V_out"].unsqueeze(0), out["out_row_offsets"].unsqueeze(0), q, H, G, BUDGET)
    error = ((binding.cache8_attention(here, q).float() - full).norm() / full.norm()).item()
    space = binding.cache8_workspace(here, q, accumulate=True)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    outs, held, rows, evictions = [], [], BUDGET, 0
    for _ in range(tokens):
        here.rows += 1
        rows += 1
        binding.cache8_append(here, rand(1, H, 128), rand(1, H, 128), status=status)
        outs.append(binding.cache8_attention(here, rand(1, 1, H * G, 128), rows, accumulate=True, workspace=space))
        if rows == BUDGET + SLACK:
            binding.cache8_evict(here, there, BUDGET, keep_first=SINKS, keep_last=RECENT, max_rows=rows, status=status)
            here, there, rows, evictions = there, here, BUDGET, evictions + 1
        held.append(rows)
    assert status.item() == 0 and (here.rows == rows).all()
    print(f"{tokens} tokens, {evictions} evictions, {rows} rows a head; attention over 8 bits is {error:.4f} off bf16 rows")
    return error, outs, held, evictions


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
