"""Point-wise products on either side of what 32-bit offsets reach: planes of 2^24 pixels, images of 2^31 bytes; gp is fp32 with bf16 storage too."""
F32, BF16 = 0, 1
REGISTERS = r"strip_(back_)?kernel"             # offsets of 32 bits, the input channels in registers
STREAMED = r"14product_kernel.*Lb0EEEvN"        # offsets of 32 bits
ADDRESSES = r"14product_kernel.*Lb1EEEvN"       # a 64-bit address for each pixel
# dtype, K, M, H, W, act; which kernels take the forward pass, gp and grad_x
CASES = [(F32, 31, 3, 4096, 4096, "none", REGISTERS, REGISTERS), (F32, 31, 3, 4096, 4097, "none", ADDRESSES, ADDRESSES), (F32, 31, 3, 4096, 4096, "gelu", REGISTERS, REGISTERS),
         (F32, 3, 31, 4096, 4096, "gelu", REGISTERS, REGISTERS), (F32, 3, 32, 4096, 4096, "gelu", ADDRESSES, ADDRESSES), (F32, 32, 3, 4096, 4096, "none", ADDRESSES, ADDRESSES),
         (F32, 200, 40, 1638, 1638, "silu", STREAMED, f"{STREAMED}|{REGISTERS}"), (F32, 200, 40, 1638, 1640, "silu", ADDRESSES, ADDRESSES),
         (BF16, 24, 130, 2048, 2010, "gelu", REGISTERS, REGISTERS), (BF16, 24, 130, 2048, 2020, "gelu", REGISTERS, ADDRESSES),
         (BF16, 63, 20, 4096, 4096, "none", REGISTERS, REGISTERS), (BF16, 64, 20, 4096, 4096, "none", ADDRESSES, ADDRESSES)]
