"""KVBuffer-style Gated DeltaNet decoding for AMD MI355X (gfx950).

``kvb``      ctypes binding of the C-ABI library (kvb_decode / kvb_flush /
             kvb_verify / kvb_direct, kvb_scan / kvb_scan_backward over whole
             sequences, kvb_accept for drafts); loads libkvb.so on first use and raises if
             it has not been built.
``synth``    seeded synthetic workloads.
``traffic``  algorithmic HBM byte counts per call (the roofline denominators).
"""
__all__ = ["kvb", "synth", "traffic"]
