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
