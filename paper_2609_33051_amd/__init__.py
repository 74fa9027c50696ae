"""SketchSSM decode hot path for MI355X (gfx950).

Submodules:
  binding  -- ctypes binding of the C-ABI library libsketchssm.so
              (sketchssm_update / sketchssm_decode / sketchssm_full_read_baseline)
  layer    -- device buffers of one linear-attention layer and its decode loop
  ops      -- the operators around the recurrence of a Mamba-2 mixer layer: conv,
              conv_token, scan, norm and matmul_fp8 on torch tensors
  mixer    -- such a layer served end to end: prompts, then single tokens
  attention -- a softmax attention layer between mixer layers, over a paged cache in 4 bits (its
              operators in ops: rotary, cache_append, cache_read and attention)
  inputs   -- seeded synthetic workloads
  traffic  -- byte accounting (the paper's model and this implementation's)

Nothing is imported eagerly: importing the package does not load the HIP library.
"""
