"""Losses of a last layer whose signal comes in several pieces of the classes, so that dx is added up over launches: type, rows, in, classes, and columns
between a row's end and the next row (with three, rows start on no 16-byte boundary).  On the GPU test_gpu_linear_xent_pieces.py runs them, on the host
test_loss_plan_pieces.py sees what they are cut into."""
PIECES = [("bf16", 972, 80, 127153, 0), ("bf16", 577, 140, 178951, 3), ("bf16", 12288, 512, 12001, 0), ("bf16", 8195, 1016, 16391, 0),
          ("bf16", 20001, 1500, 6000, 0), ("bf16", 4097, 1000, 50003, 0), ("bf16", 12000, 16, 30001, 8),
          ("f32", 20000, 300, 4001, 0), ("f32", 3000, 64, 40001, 3), ("f32", 1500, 100, 70003, 0), ("f32", 40000, 24, 2100, 0)]
