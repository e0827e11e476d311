"""Helpers of the tests of language-model layers: inputs from a seed, tolerances."""
import numpy as np
import torch

from paper_1908_05033_amd import binding as B

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                     # half a step of binary32, relative


def host(t):
    """A tensor's values in float64."""
    return t.detach().double().cpu().numpy()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half the distance of the smallest numbers of a type."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def normal(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def assert_within(got, want, bound, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    off = np.abs(got - want)
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d values off, worst %.3e with a bound of %.3e (value %.3e)" % (
        what, bad.sum(), bad.size, off[bad].max(), np.broadcast_to(bound, off.shape)[bad][np.argmax(off[bad])],
        want[bad][np.argmax(off[bad])])


def random_w4(seed, N, K, group):
    """Codes, scales (float16 numbers) and zero points on the host."""
    rs = np.random.RandomState(seed)
    G = -(-K // group)
    return (rs.randint(0, 16, (N, K)).astype(np.uint8), (0.01 * np.exp(0.5 * rs.randn(N, G))).astype(np.float16).astype(np.float32),
            rs.randint(0, 16, (N, G)).astype(np.uint8))


def pack(codes, scale, zero, group, w=None):
    """Packed weights and scales on the GPU."""
    N, K = (codes if codes is not None else w).shape
    wp = torch.full((B.dsq_w4_packed_bytes(N, K),), 0xAB, dtype=torch.uint8, device="cuda")
    sp = torch.full((B.dsq_w4_scale_bytes(N, K, group),), 0xAB, dtype=torch.uint8, device="cuda")
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    B.dsq_pack_weights_w4(dev(w), dev(codes), dev(scale), dev(zero), N, K, group, wp, sp)
    return wp, sp


def code_rows(seed, M, K, junk=False):
    """int8 rows with their pitch, and their scales; `junk`: what lies behind a row's end is not 0."""
    rs = np.random.RandomState(seed)
    q = np.zeros((M, B.dsq_code_row_bytes(K)), np.int8)
    q[:, :K] = np.clip(np.rint(rs.randn(M, K) * 40), -127, 127)
    if junk:
        q[:, K:] = 77
    s = (0.02 * np.exp(0.5 * rs.randn(M))).astype(np.float32)
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda()
