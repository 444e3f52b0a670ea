"""Every kernel that the grouped products and their weight gradients choose among, each at a size that takes it:
ragged groups, edges inside tiles, several steps of the reduction, more tiles than workgroups, entries without a row.

The sizes follow the rules that choose (``describe_grouped_matmul``, ``describe_grouped_weight_grad``): a change of
the rules that moves one of these sizes to another kernel fails here by name, and wants another size for it."""
from __future__ import annotations

import math

import pytest
import torch

from tests import ops_ref as ref
from tests.conftest import flush_print

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
F8 = torch.float64

TILES = {"bf16": ("32x128", "64x128", "128x128", "256x256"), "f32": ("32x128", "64x128", "128x128", "64x64")}
PRODUCTS = {  # kernel: entries, groups, k, n
    "few<bf16,aligned>": (37, 11, 1032, 250), "few<bf16,unaligned>": (37, 11, 1031, 250),
    "few<f32,aligned>": (37, 26, 516, 131), "few<f32,unaligned>": (37, 26, 514, 131),
    "tiles<bf16,32x128,direct,w_nk>": (413, 29, 304, 2568), "tiles<bf16,32x128,direct,w_kn>": (385, 28, 392, 2784),
    "tiles<bf16,32x128,registers,w_nk>": (404, 31, 558, 2775), "tiles<bf16,32x128,registers,w_kn>": (433, 24, 365, 2857),
    "tiles<bf16,64x128,direct,w_nk>": (1572, 28, 288, 2448), "tiles<bf16,64x128,direct,w_kn>": (1198, 31, 288, 2736),
    "tiles<bf16,64x128,registers,w_nk>": (1409, 30, 277, 2479), "tiles<bf16,64x128,registers,w_kn>": (1631, 30, 334, 2295),
    "tiles<bf16,128x128,direct,w_nk>": (18202, 24, 272, 392), "tiles<bf16,128x128,direct,w_kn>": (2145, 27, 280, 2824),
    "tiles<bf16,128x128,registers,w_nk>": (2277, 26, 293, 2869), "tiles<bf16,128x128,registers,w_kn>": (22842, 28, 284, 269),
    "tiles<bf16,256x256,direct,w_nk>": (10701, 20, 280, 2128), "tiles<bf16,256x256,direct,w_kn>": (9945, 1, 272, 2448),
    "tiles<f32,32x128,direct,w_nk>": (548, 30, 176, 2208), "tiles<f32,32x128,direct,w_kn>": (414, 28, 144, 2848),
    "tiles<f32,32x128,registers,w_nk>": (469, 31, 158, 2726), "tiles<f32,32x128,registers,w_kn>": (408, 29, 233, 2645),
    "tiles<f32,64x128,direct,w_nk>": (22364, 1, 144, 143), "tiles<f32,64x128,direct,w_kn>": (2164, 20, 136, 1744),
    "tiles<f32,64x128,registers,w_nk>": (23122, 5, 153, 137), "tiles<f32,64x128,registers,w_kn>": (22755, 31, 141, 131),
    "tiles<f32,128x128,direct,w_nk>": (28861, 21, 140, 273), "tiles<f32,128x128,direct,w_kn>": (30098, 18, 136, 280),
    "tiles<f32,128x128,registers,w_nk>": (27626, 11, 155, 262), "tiles<f32,128x128,registers,w_kn>": (27813, 3, 146, 287),
    "tiles<f32,64x64,direct,w_nk>": (18488, 6, 240, 72), "tiles<f32,64x64,direct,w_kn>": (18272, 9, 232, 72),
    "tiles<f32,64x64,registers,w_nk>": (18608, 2, 230, 70), "tiles<f32,64x64,registers,w_kn>": (18115, 2, 242, 65),
}
GRADS = {  # kernel, whether the entries are split: entries, groups, k, n
    ("tiles<bf16,256x256,direct>", False): (4100, 30, 600, 616), ("tiles<bf16,256x256,direct>", True): (13000, 8, 600, 616),
    ("tiles<bf16,128x128,direct>", False): (4100, 150, 104, 304), ("tiles<bf16,128x128,direct>", True): (80000, 3, 104, 304),
    ("tiles<bf16,128x128,registers>", False): (4100, 150, 101, 303), ("tiles<bf16,128x128,registers>", True): (80000, 3, 101, 303),
    ("tiles<bf16,64x64,direct>", False): (900, 7, 104, 304), ("tiles<bf16,64x64,direct>", True): (6000, 3, 104, 304),
    ("tiles<bf16,64x64,registers>", False): (900, 7, 101, 303), ("tiles<bf16,64x64,registers>", True): (6000, 3, 101, 303),
    ("tiles<f32,128x128,direct>", False): (4100, 150, 104, 304), ("tiles<f32,128x128,direct>", True): (40000, 3, 104, 304),
    ("tiles<f32,128x128,registers>", False): (4100, 150, 101, 303), ("tiles<f32,128x128,registers>", True): (40000, 3, 101, 303),
    ("tiles<f32,64x64,direct>", False): (900, 7, 104, 304), ("tiles<f32,64x64,direct>", True): (6000, 3, 104, 304),
    ("tiles<f32,64x64,registers>", False): (900, 7, 101, 303), ("tiles<f32,64x64,registers>", True): (6000, 3, 101, 303),
}


def test_every_kernel_has_a_size():
    """The kernels that are built: 256 x 256 tiles for whole vectors in bf16 only, the few-entries form for W as [n, k]."""
    whole = {f"few<{t},{a}>" for t in DT for a in ("aligned", "unaligned")}
    whole |= {f"tiles<{t},{s},{how},{w}>" for t in DT for s in TILES[t] for how in ("direct", "registers")
              for w in ("w_nk", "w_kn") if s != "256x256" or how == "direct"}
    assert set(PRODUCTS) == whole
    grads = {f"tiles<{t},{s},{how}>" for t in DT for s in ("64x64", "128x128") for how in ("direct", "registers")}
    assert set(GRADS) == {(g, split) for g in grads | {"tiles<bf16,256x256,direct>"} for split in (False, True)}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(DT[dtype])


def _groups(gen, E, G):
    """Ragged offsets of E entries, the second group empty, two entries behind the last group."""
    pick = torch.randint(0, G, (E - 2,), generator=gen, device="cuda").cpu()
    if G > 2:
        pick[pick == 1] = 0
    return torch.cat((torch.zeros(1, dtype=torch.int64), torch.bincount(pick, minlength=G).cumsum(0))).to(torch.int32).cuda()


def _product(x, w, offsets, index, transpose):
    """z in float64 in grouped order and its fp32 error (2 U a term: the matrix cores may truncate), on the GPU."""
    index = index.long()
    there = (index >= 0) & (index < x.shape[0])
    xs = torch.where(there[:, None], x[index.clamp(0, x.shape[0] - 1)].to(F8), 0.0)
    N, K = (w.shape[2], w.shape[1]) if transpose else w.shape[1:]
    z = torch.zeros((index.numel(), N), dtype=F8, device="cuda")
    err = torch.zeros_like(z)
    for g, (a, b) in enumerate(zip(offsets.tolist(), offsets[1:].tolist())):
        m = (w[g] if transpose else w[g].T).to(F8).contiguous()
        z[a:b] = xs[a:b] @ m
        err[a:b] = (2 * K + 4) * ref.U * (xs[a:b].abs() @ m.abs())
    return z, err


def _act(z, name):
    """Either GELU and its derivative in float64."""
    if name == "gelu":
        phi = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        share, d_share = 0.5 * torch.erfc(-z * math.sqrt(0.5)), phi
    else:
        c = 2 * math.sqrt(2 / math.pi)
        share = torch.sigmoid(c * (z + 0.044715 * z ** 3))
        d_share = share * torch.sigmoid(-c * (z + 0.044715 * z ** 3)) * c * (1 + 0.134145 * z * z)
    return z * share, share + z * d_share


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", list(PRODUCTS))
def test_products(fff_lib, kernel):
    E, G, K, N = PRODUCTS[kernel]
    t, transpose = "bf16" if "bf16" in kernel else "f32", "w_kn" in kernel
    gen = _gen(E + G + K + N)
    offsets = _groups(gen, E, G)
    used = int(offsets[-1])
    w = (_randn(gen, G, *((K, N) if transpose else (N, K)), dtype="f32") * K ** -0.5).to(DT[t])
    x = _randn(gen, E, K, dtype=t)
    index, place = (torch.randperm(E, generator=gen, device="cuda").to(torch.int32) for _ in range(2))
    index[used // 3], index[2 * used // 3], place[used // 2] = -1, E, E + 5  # two entries without a row, one without a place
    kept = place < E
    kept[used:] = False
    kw = {"x_index": index, "transpose_w": transpose}
    assert fff_lib.describe_grouped_matmul(x, w, offsets, **kw).split(" ")[0] == kernel
    z64, ez = _product(x, w, offsets, index, transpose)
    flush_print(f"[gpu] {kernel} {E} x {G}, {K} -> {N}")
    for yt, act in (("f32", "identity"), ("bf16", "gelu"), ("f32", "gelu"), ("f32", "gelu_tanh"), ("bf16", "gelu_tanh")):
        y, z = (torch.full((E, N), -7.0, dtype=DT[yt], device="cuda") for _ in range(2))
        fff_lib.grouped_matmul(x, w, offsets, y=y, y_index=place, act=act, z_out=z, **kw)
        ref.check(z[:used], z64[:used].cpu(), ez[:used].cpu(), f"z {yt}")
        want, err = z64, ez
        if act != "identity":
            want = _act(z64, act)[0]
            err = 1.13 * ez + (16 + 2 * z64 ** 2) * ref.U * want.abs()  # 1.13: the largest derivative of either
        ref.check(y[place[kept].long()], want[kept].cpu(), err[kept].cpu(), f"y {yt} {act}")
        free = torch.ones(E, dtype=torch.bool, device="cuda")
        free[place[kept].long()] = False
        assert (y[free] == -7).all() and (z[used:] == -7).all(), "rows that no entry names are left as they were"
    for zt, act in (("f32", "gelu"), ("bf16", "gelu_tanh")):
        z_in = (2 * _randn(gen, E, N, dtype="f32")).to(DT[zt])
        d = _act(z_in.to(F8), act)[1]
        zi = z_in.to(F8)
        # the derivative's own error: z enters the exponential squared, a few roundings each, sizes up to 1 + |z|
        ed = (16 + 2 * zi ** 2) * ref.U * (1 + zi.abs()) * torch.exp(-zi ** 2 / 2).clamp_min(1e-30) + 8 * ref.U * d.abs()
        want = z64 * d
        err = ez * d.abs() + z64.abs() * ed + ez * ed + 2 * ref.U * want.abs()
        for yt in ("f32", "bf16"):
            y = torch.full((E, N), -7.0, dtype=DT[yt], device="cuda")
            fff_lib.grouped_matmul(x, w, offsets, y=y, act=act, z_in=z_in, **kw)
            ref.check(y[:used], want[:used].cpu(), err[:used].cpu(), f"gradient {yt} {act}")
            assert (y[used:] == -7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,split", list(GRADS))
def test_weight_gradients(fff_lib, kernel, split):
    E, G, K, N = GRADS[kernel, split]
    t = "bf16" if "bf16" in kernel else "f32"
    gen = _gen(E + G + K)
    offsets = _groups(gen, E, G)
    used = int(offsets[-1])
    dy, x = _randn(gen, E, N, dtype=t), _randn(gen, E, K, dtype=t)
    index, place = (torch.randperm(E, generator=gen, device="cuda").to(torch.int32) for _ in range(2))
    index[used // 3], index[2 * used // 3], place[used // 2] = -1, E, E + 5
    kw = {"dy_index": place, "x_index": index}
    plan = fff_lib.describe_grouped_weight_grad(dy, x, offsets, **kw).split(" ")
    assert plan[0] == kernel and (plan[1] != "splits=1") == split
    flush_print(f"[gpu] weight gradient {kernel} {E} x {G}, {K} x {N}, split {split}")
    there = (index >= 0) & (index < E) & (place < E)
    dys = torch.where(there[:, None], dy[place.long().clamp(0, E - 1)].to(F8), 0.0)
    xs = torch.where(there[:, None], x[index.long().clamp(0, E - 1)].to(F8), 0.0)
    want = torch.zeros((G, N, K), dtype=F8, device="cuda")
    err = torch.zeros_like(want)
    for g, (a, b) in enumerate(zip(offsets.tolist(), offsets[1:].tolist())):
        if b > a:
            left = dys[a:b].T.contiguous()
            want[g] = left @ xs[a:b]
            err[g] = (2 * (b - a) + 4) * ref.U * (left.abs() @ xs[a:b].abs())
    dw = fff_lib.grouped_weight_grad(dy, x, offsets, **kw)
    ref.check(dw, want.cpu(), err.cpu(), "dw")
    assert torch.equal(dw, fff_lib.grouped_weight_grad(dy, x, offsets, **kw))
    base = _randn(gen, G, N, K, dtype="f32")
    got = fff_lib.grouped_weight_grad(dy, x, offsets, dw=base.clone(), accumulate=True, **kw)
    ref.check(got, (want + base.to(F8)).cpu(), (err + ref.U * (want.abs() + base.to(F8).abs())).cpu(), "accumulated")


@pytest.mark.gpu
@pytest.mark.parametrize("t,k", [("bf16", 8), ("f32", 4)])
def test_more_tiles_than_the_few_entries_form_launches(fff_lib, t, k):
    """2^23 groups of an entry: more workgroups than the few-entries form may launch, so tiles take them."""
    import ctypes

    from paper_2311_10770_amd import ops

    P, buf = 1 << 40, ctypes.create_string_buffer(256)  # addresses that nothing reads: a description only
    for n_groups, form in ((1 << 22, "few"), (1 << 23, "tiles")):
        a = ops.FffGroupedMatmulArgs(x=P, w=2 * P, offsets=3 * P, y=4 * P, n_entries=n_groups, x_rows=n_groups, y_rows=n_groups,
                                     n_groups=n_groups, k=k, n=16, x_div=1, x_dtype=int(t == "bf16"), w_dtype=int(t == "bf16"))
        assert ops._lib().fff_describe_grouped_matmul(ctypes.addressof(a), buf, len(buf)) == 0
        flush_print(f"[gpu] {n_groups} groups {t}: {buf.value.decode()}")
        assert buf.value.decode().startswith(form + "<")
