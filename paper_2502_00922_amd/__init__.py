"""MI355X-native Huff-LLM: lossless bf16 weight compression with decoding
fused into the decode-step GEMV on gfx950, and the operators between the
products of a decoder layer (norm, attention over a shared prefix, eviction
from the cache)."""
from .hufflm import (AttentionResult, Codebook, DeviceTensor, EvictResult, HLError, NormResult, build_codebook,
                     cache_evict, default_grp_rows, default_seg_len, encode, gemv_bf16, gemv_multi, lib,
                     prefix_attention, rms_norm, status_str, validate)

__all__ = ["AttentionResult", "Codebook", "DeviceTensor", "EvictResult", "HLError", "NormResult", "build_codebook",
           "cache_evict", "default_grp_rows", "default_seg_len", "encode", "gemv_bf16", "gemv_multi", "lib",
           "prefix_attention", "rms_norm", "status_str", "validate"]
