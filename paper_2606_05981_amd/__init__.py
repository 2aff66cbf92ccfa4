"""MI355X (gfx950) multimodal text-encoder prefill: HIP kernels behind a C ABI.

``binding`` mirrors the headers under include/ one to one; ``encoder`` wraps the
encoders for torch tensors and ``conditioning`` the operators that read what they
return; ``build`` compiles libmte.so. Importing any of the three requires the built
library.
"""
