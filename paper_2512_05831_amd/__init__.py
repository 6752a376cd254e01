"""Embedding Bag forward (arXiv 2512.05831) for AMD Instinct MI355X.

``eb``        -- binding of the C ABI in include/eb.h (libeb.so, HIP / gfx950).
``experts``   -- binding of include/eb_experts.h: a mixture of experts on the
                 pooled vectors (routing, 8-bit quantisation and products).
``train``     -- binding of include/eb_train.h: what trains a mixture of experts
                 (layer norm, activations from 8-bit checkpoints, sorting by
                 expert, weight gradients).
``workloads`` -- seeded synthetic inputs (tables, lengths, offsets, indices).
``build``     -- compiles libeb.so in tree.
"""
