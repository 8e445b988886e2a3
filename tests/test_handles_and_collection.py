"""Handles go with their context however the two are collected: from a cycle of references (a caught exception's frames make one), where weak
references are gone before anything is finalised, the context may come first."""
import gc

import pytest
import torch

import paper_2202_02365_b200 as mg
from paper_2202_02365_b200 import inputs


class Library:
    """What frees, in the order it was asked for."""

    def __init__(self):
        self.freed = []

    def __getattr__(self, name):
        if not name.startswith("mg_"):
            raise AttributeError(name)
        return lambda handle: self.freed.append((name, handle.value)) or 0


def make(lib, first):
    """A context and four handles of it in one cycle of references, finalised in an order that `first` turns round."""
    from paper_2202_02365_b200 import api
    ctx = object.__new__(api.Context)
    ctx.lib, ctx._owned, ctx._keep, ctx.handle = lib, {}, {}, api.C.c_void_p(1)
    kinds = [api.Dense, api.Model, api.GatModel, api.LpBatch]
    owned = []
    for i, kind in enumerate(kinds):
        o = object.__new__(kind)
        o._own(ctx)
        o.handle.value = 10 + i
        owned.append(o)
    ring = [ctx] + owned if first else owned + [ctx]
    for o in ring:
        o.__dict__["ring"] = ring


@pytest.mark.parametrize("context_first", [True, False])
def test_everything_is_freed_once_and_the_context_last(context_first):
    lib = Library()
    make(lib, context_first)
    gc.collect()
    assert sorted(lib.freed[:-1]) == [("mg_dense_free", 10), ("mg_gat_model_free", 12), ("mg_lp_free", 13), ("mg_model_free", 11)]
    assert lib.freed[-1] == ("mg_destroy", 1)


@pytest.mark.gpu
def test_collected_with_their_context():
    g = inputs.erdos_renyi_graph(2_000, 20_000, seed=1)
    for _ in range(5):
        ctx = mg.Context(0)
        ctx.load_graph(g.row_offsets.cuda(), g.nbrs.cuda())
        ctx.load_features(torch.zeros(2_000, 8, device="cuda"))
        ids = torch.arange(50, dtype=torch.int32)
        ring = [ctx, ctx.lp_prepare(ids, ids, ids + 100, 2, 10, seed=1), ctx.sample(ids, [3], 1), ctx.model(inputs.random_bias_layers([8, 8], seed=1))]
        ring.append(ring)
        del ctx, ring
        gc.collect()
    torch.cuda.synchronize()
