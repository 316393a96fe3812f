"""MI355X-native search path of sparsity-aware IVF-PQ (JUNO, arxiv 2312.01712).

`binding` holds the thin ctypes front end of the C-ABI library built from
`csrc/`; `kv` that of the paged 4-bit key/value cache; `workloads` holds the seeded synthetic inputs and the offline trainer.
"""
