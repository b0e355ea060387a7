"""Gradients of whole numbers, whose sums are exact in fp32 in any order: equal
to the 64-bit results, so that no row may be missing or counted twice anywhere
(tests/test_tokens_util.py shows that the check notices one)."""
from __future__ import annotations

import pytest
import torch

from paper_2007_13005_amd import tokens
from tests import tokens_util as ref
from tests.gpu_util import note
from tests.test_gpu_tokens_launches import launches

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SENTINEL = -77.0


# n, c, h, w, p, dim, nhwc; threads of a workgroup of the 16-bit products (512:
# tiles of 256). Rows that end inside a step of 64 (and of 32, fp32), parts of
# the rows of unequal length, columns and values that end inside a tile.
PATCHES = [((201, 3, 224, 224, 16, 780, False), 512), ((150, 3, 210, 224, 14, 1000, True), 512),
           ((193, 3, 224, 238, 14, 772, False), 512), ((431, 3, 128, 128, 16, 1024, False), 512),
           ((33, 3, 160, 176, 16, 1000, False), 256), ((61, 3, 112, 120, 14, 776, True), 256),
           ((97, 3, 70, 84, 9, 130, False), 256), ((7, 2, 63, 70, 7, 264, False), 256),
           ((3, 3, 65, 97, 16, 4, False), 256), ((1, 3, 32, 32, 16, 64, False), 256)]


@pytest.mark.parametrize("case, threads", PATCHES)
@pytest.mark.parametrize("image, dtype", [(F16, BF16), (F16, F16), (BF16, BF16), (F32, F32),
                                          (F32, F16)])
def test_patch_gradient_of_whole_numbers(case, threads, image, dtype):
    note(f"patch grad whole {case} {image} {dtype}")
    n, c, h, w, p, dim, nhwc = case
    g = torch.Generator().manual_seed(dim)
    img = ref.whole(g, *((n, h, w, c) if nhwc else (n, c, h, w)), dtype=image).cuda()
    t = (h // p) * (w // p)
    dy = ref.whole(g, n, t, dim, dtype=dtype).cuda()
    layout = tokens.LAYOUT_NHWC if nhwc else tokens.LAYOUT_NCHW
    shapes = ((dim, p, p, c) if nhwc else (dim, c, p, p)), (dim,), (t, dim)
    a, d = ref.patches(img.double(), p, nhwc).reshape(n * t, -1), dy.double()
    d2 = d.reshape(n * t, dim)
    want = (torch.mm(d2.t().contiguous(), a).reshape(shapes[0]), d2.sum(0), d.sum(0))
    assert 4 * n * t < 2 ** 24
    names = "weight", "bias", "pos"
    got = [torch.full(s, SENTINEL, device="cuda") for s in shapes]
    room = torch.empty(tokens.patch_embed_workspace_bytes(img, got[0], dtype, layout),
                       dtype=torch.uint8, device="cuda")
    found = launches(lambda: tokens.patch_embed_backward(dy, img, *got, layout=layout,
                                                         workspace=room))
    assert found[0][1] == (threads if dtype != F32 and image != F32 else 256)
    for x in got:
        x.fill_(SENTINEL)
    tokens.patch_embed_backward(dy, img, *got, layout=layout, workspace=room)
    for x, e, name in zip(got, want, names):
        ref.same(x, e, name)
    # added to what is there; grad_out a slice of a longer sequence
    old = [ref.whole(g, *s, dtype=F32, most=100).cuda() for s in shapes]
    got = [o.clone() for o in old]
    seq = torch.full((n, t + 2, dim + 1), SENTINEL, dtype=dtype, device="cuda")
    seq[:, 1:1 + t, 1:] = dy
    tokens.patch_embed_backward(seq[:, 1:1 + t, 1:], img, *got, layout=layout, accumulate=True,
                                workspace=room)
    for x, e, o, name in zip(got, want, old, names):
        ref.same(x, e + o.double(), f"{name} added")


TYPES = [F32, F16, BF16]


def zipf(g, n, vocab, holes):
    """Frequent low ids: the most frequent of 300 is named by 12 % of the rows."""
    u = torch.rand(n, generator=g, dtype=torch.float64)
    ids = (torch.exp(u * torch.log(torch.tensor(vocab + 1.0))) - 1).long().clamp_(0, vocab - 1)
    ids[torch.rand(n, generator=g) < holes] = -1
    return ids


@pytest.mark.parametrize("n, kernels", [(900, 1), (4000, 3), (7000, 3), (20000, 4)])
@pytest.mark.parametrize("dim", [5, 72, 1030])
@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("act", TYPES)
def test_table_gradient_of_whole_numbers(n, kernels, dim, grad, act):
    """Every pair of types on every way of summing (one launch; ids counted;
    ids sorted by one digit), with ids that reach over many pieces of the rows:
    the exact sum rounded once, overwritten and added."""
    note(f"embed grad whole n={n} dim={dim} {act} {grad}")
    vocab = 300
    g = torch.Generator().manual_seed(n + dim)
    ids = zipf(g, n, vocab, 0.1)
    piece = 1 if kernels == 1 else 8 if n <= 4096 else 32  # rows; more than 16 pieces
    assert int((ids == 0).sum()) > 17 * piece
    dy = ref.whole(g, n, dim, dtype=act)
    some = ids >= 0
    want = torch.zeros((vocab, dim), dtype=torch.float64).index_add_(0, ids[some],
                                                                     dy[some].double())
    dev_ids, dev_dy = ids.cuda(), dy.cuda()
    out = torch.full((vocab, dim), SENTINEL, dtype=grad, device="cuda")
    room = torch.empty(tokens.embed_workspace_bytes(n, vocab, dim), dtype=torch.uint8,
                       device="cuda")
    assert len(launches(lambda: tokens.embed_backward(dev_dy, dev_ids, out, 0.5,
                                                      workspace=room))) == kernels
    out.fill_(SENTINEL)
    tokens.embed_backward(dev_dy, dev_ids, out, 0.5, workspace=room)
    ref.same(out, want * 0.5, "table")
    old = ref.whole(g, vocab, dim, dtype=grad, most=64)
    wide = torch.full((vocab, dim + 3), SENTINEL, dtype=grad, device="cuda")
    wide[:, 1:1 + dim] = old.cuda()
    tokens.embed_backward(dev_dy, dev_ids, wide[:, 1:1 + dim], 2.0, padding=1, accumulate=True,
                          workspace=room)
    want[1] = 0
    ref.same(wide[:, 1:1 + dim], want * 2 + old.double(), "added")
    assert bool((wide[:, 0] == SENTINEL).all()) and bool((wide[:, 1 + dim:] == SENTINEL).all())
