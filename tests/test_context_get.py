"""Context.get on the CPU: views of a workspace's regions have the shapes that the library's sizes say, or are refused."""
import pytest
import torch

import paper_2503_09304_amd as q
from paper_2503_09304_amd import binding as b

E, K, H, F, N = 6, 2, 64, 128, 10
SIZES = {"logits": N * E * 4, "topk_idx": N * K * 4, "topk_w": N * K * 4, "counts": E * 8, "offsets": (2 * E + 1) * 4, "perm": N * K * 4, "inv": N * K * 4,
         "expert_out": N * K * H * 4, "act": N * K * F * 2, "units": 7 * 16}
SHAPES = {"logits": (N, E), "topk_idx": (N, K), "topk_w": (N, K), "counts": (E, 2), "offsets": (2 * E + 1,), "perm": (N * K,), "inv": (N * K,),
          "expert_out": (N * K, H), "act": (N * K, F), "units": (7, 4)}


@pytest.fixture
def context(monkeypatch):
    """A context without a GPU: its workspace in host memory, a stand-in for moe_get that gives the size the library would."""
    c = object.__new__(q.Context)
    c.cfg, c.N, c.h = q.MoeConfig(E, K, H, F, q.MOE_BF16, 16, 64, 0), N, None
    c.ws = torch.arange(1 << 18, dtype=torch.int32).view(torch.uint8)
    c._ws_at, c._typed = c.ws.data_ptr(), None

    class Library:
        def moe_get(self, h, what, p, nb):
            p._obj.value, nb._obj.value = c._ws_at + 4096, dict(SIZES, **c.sizes)[next(n for n, i in b.GET.items() if i == what)]
            return q.MOE_OK

    c.sizes = {}
    monkeypatch.setattr(b, "lib", Library)
    return c


@pytest.mark.parametrize("name", SIZES)
def test_views_have_the_regions_sizes(name, context):
    t = context.get(name)
    assert t.shape == SHAPES[name] and t.is_contiguous() and t.nbytes == SIZES[name] and t.data_ptr() == context._ws_at + 4096


@pytest.mark.parametrize("name", ["logits", "topk_idx", "topk_w", "expert_out", "act", "counts", "units"])
@pytest.mark.parametrize("factor", [0.5, 1.5, 2])
def test_a_region_of_another_size_is_refused(name, factor, context):
    """The context was driven past the binding (with another number of tokens): no view of rows that are not there, or of a part of them."""
    context.sizes[name] = int(SIZES[name] * factor) + (4 if name == "units" else 0)
    with pytest.raises(RuntimeError):
        context.get(name)
