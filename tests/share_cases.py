"""Calls of dsi_attend that run every variant of the shared prefix's kernel, in
several stages and chunks: the GPU tests run them, the host tests check that
they are what runs."""

# query heads, KV heads, head dim, windows, rows, shared positions, max_len,
# query tiles of 32 per workgroup, keys per chunk
CASES = [
    # more than 128 queries: chunks of 128 keys up to 2048, of 192 beyond
    (32, 8, 128, 7, 6, 2047, 4300, 8, 128),
    (32, 8, 128, 7, 6, 2048, 4300, 8, 128),
    (32, 8, 128, 7, 6, 2081, 4300, 8, 192),
    (32, 8, 128, 7, 6, 4100, 4300, 8, 192),
    (32, 8, 64, 7, 6, 2081, 4300, 8, 192),
    (24, 8, 96, 8, 6, 2047, 4300, 8, 128),
    (24, 8, 96, 8, 6, 2500, 4300, 8, 192),
    (32, 8, 32, 5, 7, 3333, 4300, 8, 192),
    # six stages a chunk, and two tiles of 256 queries, of which the second is mostly empty
    (32, 8, 128, 8, 8, 12289, 12500, 8, 384),
    (16, 4, 64, 8, 9, 5003, 5200, 8, 192),
    # 65 to 128 queries
    (32, 8, 128, 4, 6, 8191, 8300, 4, 256),
    (16, 4, 64, 3, 10, 4999, 5200, 4, 128),
    (12, 4, 96, 5, 7, 9001, 9200, 4, 192),
    (32, 16, 32, 8, 5, 8000, 8200, 4, 512),
    # up to 64
    (40, 40, 128, 6, 7, 8191, 8300, 2, 1408),
    (32, 32, 64, 2, 8, 5000, 5100, 2, 640),
    (24, 24, 96, 3, 3, 6011, 6100, 2, 640),
    (16, 16, 32, 2, 1, 9001, 9100, 2, 576),
]
