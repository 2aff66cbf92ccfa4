"""MI355X (gfx950) multimodal text-encoder prefill: HIP kernels behind a C ABI.

``binding`` mirrors the headers under include/ one to one; ``encoder`` wraps the
encoders for torch tensors, ``projections`` the linear layers and rotary positions
that turn what they return into queries and keys, and ``conditioning`` the operators that read
it; ``build`` compiles libmte.so. Importing any of the four requires the built library.
"""
