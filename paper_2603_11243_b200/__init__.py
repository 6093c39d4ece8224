"""B200-native decision kernels for CTC-draft self-speculative decoding of LLM-based ASR.

`binding` exposes the C ABI of libssd (ssd_ctc_draft, ssd_entropy_gate, ssd_verify; for draft trees
ssd_tree_attention, ssd_verify_tree, ssd_cache_append, ssd_cache_weights, ssd_cache_evict);
`synth` holds the seeded synthetic workloads; `build` compiles the library for sm_100a.
"""
__all__ = ["binding", "synth", "build"]
