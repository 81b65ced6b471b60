"""Products of 8-bit operands that are split along k: (m, n, k, splits of each kind of sum in turn:
power-of-two scales and 16-bit results, the same with fp32 results, fp32 scales with each)."""
SPLIT = [(200, 301, 1900, (1, 2, 1, 2)), (35, 67, 2100, (4,) * 4), (301, 299, 8200, (8,) * 4), (65, 131, 16500, (15,) * 4),
         (99, 65, 20001, (16,) * 4)]
# linear layers of 33 tokens and more, fp16 and fp32, whose product is split
SPLIT_LINEAR = [(64, 501, 4096), (130, 97, 5001)]
