"""Scaffolding of the tests of the target's cache, tree attention and distributions: device buffers, the calls, their contents decoded."""
import numpy as np

from oracle import target as orc
from paper_2410_05589_amd import binding as B
from paper_2410_05589_amd import verify as VF


def torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def np64(t):
    return t.detach().double().cpu().numpy()


def places(kind, d):
    t, j = np.meshgrid(np.arange(32), np.arange(d), indexing="ij")
    return orc.place(kind, t, j).reshape(-1)


class Cache:
    """A cache of sequences with `capacity` positions each (multiples of 32), its codes and scales random bytes at first: nothing of it
    has to be initialised.  `lead` blocks in front belong to nobody."""

    def __init__(self, heads, d, capacity, seed=0, lead=1, scales=None):
        import torch
        self.heads, self.d = heads, d
        self.offsets = [32 * lead]
        for c in capacity:
            self.offsets.append(self.offsets[-1] + c)
        blocks = self.offsets[-1] // 32 + 1
        g = torch.Generator().manual_seed(seed)
        self.codes = {n: torch.randint(0, 256, (blocks, heads, 32 * d), generator=g, dtype=torch.uint8).cuda() for n in "kv"}
        self.scales = {n: (torch.randn((blocks, heads), generator=g) if scales is None else torch.full((blocks, heads), scales)).cuda() for n in "kv"}
        self.struct = VF.make_cache(heads, d, self.codes["k"].data_ptr(), self.codes["v"].data_ptr(),
                                    self.scales["k"].data_ptr(), self.scales["v"].data_ptr(), self.offsets)

    def decoded(self, kind):
        """(values [blocks, heads, 32, d] without scales, scales [blocks, heads]) in float64"""
        codes = self.codes[kind].cpu().numpy()
        return orc.VALUES[codes[:, :, places(kind, self.d)]].reshape(*codes.shape[:2], 32, self.d), np64(self.scales[kind])

    def write_args(self, k, v, kv_len, dtype, n_seq=None, stride=0):
        a = VF.make_cache_write_args(self.struct, k.shape[1], dtype, kv_len, n_seq)
        a.k_rows, a.v_rows, a.row_stride = k.data_ptr(), v.data_ptr(), stride
        return a

    def write(self, k, v, kv_len, dtype, n_seq=None, stride=0, **pointers):
        a = self.write_args(k, v, kv_len, dtype, n_seq, stride)
        for n, x in pointers.items():
            setattr(a, n, x if isinstance(x, int) else x.data_ptr())
        st = VF.ps_cache_write(a, stream())
        assert st == B.PS_OK, B.ps_draft_strerror(st)

    def read(self, k, v, start, dtype, n_seq=None, stride=0):
        a = VF.make_cache_read_args(self.struct, (k if k is not None else v).shape[1], dtype, start, n_seq)
        a.k_rows, a.v_rows, a.row_stride = k.data_ptr() if k is not None else None, v.data_ptr() if v is not None else None, stride
        st = VF.ps_cache_read(a, stream())
        assert st == B.PS_OK, B.ps_draft_strerror(st)


def normal(shape, seed, dtype, gain=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * gain).to(torch_dtype(dtype)).cuda()


def strided(x, stride, lead=0):
    """The rows [batch, rows, heads, d] of x, `stride` elements apart, `lead` elements behind the start of an allocation."""
    import torch
    b, n, h, d = x.shape
    mem = torch.full((lead + b * n * stride,), float("nan"), dtype=x.dtype, device=x.device)
    view = mem[lead:].as_strided((b, n, h, d), (n * stride, stride, d, 1))
    view.copy_(x)
    return view


def workspace(need, fill=0xA5):
    """(memory, its aligned address)"""
    import torch
    x = torch.full((need + 512,), fill, dtype=torch.uint8, device="cuda:0")
    return x, (x.data_ptr() + 255) & ~255
