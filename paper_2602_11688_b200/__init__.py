"""B200-native population replay of the GORGO routing cost model.

``paper_2602_11688_b200.binding`` exposes the C-ABI entry points of ``libgorgo_b200.so``
(it raises if the library has not been built); ``paper_2602_11688_b200.workloads``
generates the seeded synthetic traces; ``paper_2602_11688_b200.service`` measures the constants of the
service model with the paged key-value cache and its attention.
"""
__all__ = ["binding", "workloads", "service", "build"]
