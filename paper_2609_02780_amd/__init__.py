"""MI355X (gfx950) implementation of ShallowStream's query-time evidence
retrieval over a shallow-layer key index.

The work runs in ``libshallowstream.so`` (HIP kernels behind the C ABI of
``include/shallowstream.h``); this package only marshals arguments.
"""
from ._lib import SSError, lib  # noqa: F401
from .index import (HistoryAttention, LongClusters, PooledRanker, Retriever, ShallowIndex,  # noqa: F401
                    assemble_evidence, sample_plan, set_profile_events)
from .paged import PagedBatch, PagedCache, Rotary  # noqa: F401

__all__ = ["ShallowIndex", "Retriever", "PooledRanker", "LongClusters", "HistoryAttention", "Rotary", "PagedCache",
           "PagedBatch", "assemble_evidence", "SSError", "sample_plan", "set_profile_events", "lib"]
