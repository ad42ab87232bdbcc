"""Sizes at which the decoder layer's operators take each of their kernels: what test_gpu_layer_ops_edges.py compares with the definitions, and
test_layer_ops_plans.py holds to reaching every one of them."""
# channels, contraction, tokens; bf16 W and X: tiles of 256, 128 and 64, whole and in parts of the contraction, up to 16 and up to 32 tokens
LINEAR_BF16 = [(1133, 75, 7729), (545, 5548, 7717), (2304, 264, 2049), (408, 7865, 376), (129, 257, 130), (300, 2000, 200), (40, 700, 5), (40, 700, 20)]
# an fp32 operand: tiles of 128 x 128, 128 x 64 and 64 x 64, whole and in parts
LINEAR_F32 = [(3831, 823, 1013), (3179, 5242, 95), (489, 1688, 19909), (5126, 2117, 1), (65, 33, 200), (700, 600, 70)]
# channels and tokens: columns of 16 bytes a workgroup (16, 8, 4, 2, 1) by rows a thread (16, 8, 4, 2)
NORM_TOKENS = {"bf16": {16: 40001, 8: 17001, 4: 5001, 2: 2501, 1: 131}, "f32": {16: 17001, 8: 9001, 4: 2501, 2: 1301, 1: 131}}
NORM = {dt: [(rows * 1000 // ct + (ct == 1), T) for ct, T in by.items() for rows in (16, 8, 4, 2)] for dt, by in NORM_TOKENS.items()}
NORM_TALL = [(16400, 37), (20001, 131)]
# entries, tokens, alternatives: eight wavefronts a token and one; in the last a part of the vocabulary's maxima that does not fit registers
LOGPROBS = [(5000, 2048, 5), (5000, 2049, 5), (131000, 2100, 16)]
