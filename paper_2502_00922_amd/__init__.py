"""MI355X-native Huff-LLM: lossless bf16 weight compression with decoding
fused into the decode-step GEMV on gfx950, the operators between the products
of a decoder layer (norm, attention over a shared prefix, eviction from the
cache), and a step's 4-bit forms and end (a cache held in 4 bits, products of
4-bit weights, sampling)."""
from .hufflm import (AttentionResult, Codebook, DeviceTensor, EvictResult, HLError, NormResult, SampleResult,
                     build_codebook, cache4_row_bytes, cache_evict, cache_read4, cache_write4, default_grp_rows,
                     default_seg_len, encode, gemv4, gemv_bf16, gemv_multi, lib, prefix_attention, prefix_attention4,
                     rms_norm, sample, status_str, validate)

__all__ = ["AttentionResult", "Codebook", "DeviceTensor", "EvictResult", "HLError", "NormResult", "SampleResult",
           "build_codebook", "cache4_row_bytes", "cache_evict", "cache_read4", "cache_write4", "default_grp_rows",
           "default_seg_len", "encode", "gemv4", "gemv_bf16", "gemv_multi", "lib", "prefix_attention",
           "prefix_attention4", "rms_norm", "sample", "status_str", "validate"]
