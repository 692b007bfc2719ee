"""Calls in which a workgroup's and a wave's part of shared attention is long: 256 layers and
KV heads, a workgroup for each, so that page ids are looked up again and again on the way."""
LAYERS, HEADS = 32, 8

# dtype, head dim, query heads of a KV head, page, shared rows, own rows of each sequence, (sinks, window)
COMMON = [("bf16", 128, 4, 16, 2501, (3, 20), w) for w in ((0, 0), (70, 2200))] + \
         [("bf16", 64, 16, 32, 3333, (0, 31, 5, 64, 17), w) for w in ((0, 0), (3, 3000))] + \
         [("f32", 64, 16, 16, 2501, (3, 20), w) for w in ((0, 0), (70, 2200))] + \
         [("f32", 128, 16, 16, 2333, (9, 0, 33), w) for w in ((0, 0), (1, 2201))] + \
         [("f32", 128, 16, 64, 2333, (0, 31, 5, 64, 17), w) for w in ((0, 0), (40, 2250))] + \
         [("f32", 64, 8, 16, 2203, (12, 1, 40, 7), w) for w in ((0, 0), (5, 2150))]
OWN = [("bf16", 64, 4, 16, 40, (3000, 5000, 2101), w) for w in ((0, 0), (4, 2900))] + \
      [("bf16", 128, 7, 64, 33, (9001,), w) for w in ((0, 0), (20, 8500))] + \
      [("f32", 64, 2, 16, 77, (100, 6003, 2900, 33), w) for w in ((0, 0), (90, 4000))] + \
      [("f32", 128, 1, 32, 0, (5003, 4000), w) for w in ((0, 0), (0, 3500))]
