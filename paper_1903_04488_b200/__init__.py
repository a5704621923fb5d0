"""B200-native Sketched-SGD compression step (CUDA, sm_100a) behind a C-ABI library.

`from paper_1903_04488_b200 import ssgd` gives the thin binding over the library; `workloads` holds the
seeded synthetic gradient generators.  `train_ops` and `autograd` are the operators of the training step around
the compression (layer norm, log probabilities of given tokens, AdamW); `train_lm` uses them all together.
"""
