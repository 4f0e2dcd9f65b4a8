"""Helpers for the GPU parity tests: moving checkpoint arrays between numpy
(fp32 arrays, or uint16 arrays of raw bfloat16 patterns) and torch device
tensors, and the merge tolerance."""

import numpy as np


def to_dev(a, dtype, device="cuda"):
    import torch
    if dtype == "bf16":
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(device)


def to_pinned(a, dtype):
    """A new pinned host tensor holding the array (allocated pinned, never
    registered after the fact)."""
    import torch
    if dtype == "bf16":
        t = torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16)
    else:
        t = torch.from_numpy(np.ascontiguousarray(a, np.float32))
    return t.pin_memory()


def to_host(t):
    import torch
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    return t.cpu().numpy()


def gather_blocks(t, blocks, ids):
    """Copy the listed blocks of a device checkpoint into one compact host
    array; returns (array, doff) with doff the element offset of each block."""
    import torch
    idx = np.concatenate([np.arange(blocks.off[g], blocks.off[g] + blocks.len[g]) for g in ids])
    sel = t[torch.from_numpy(idx).to(t.device)]
    doff = np.concatenate([[0], np.cumsum(blocks.len[ids])[:-1]]).astype(np.int64)
    return to_host(sel), doff


def assert_merge_equal(got, want, base, dtype, what=""):
    """The merge tolerance: fp32 |g - o| <= 1e-6 * max(|o|, |base|); bf16 at
    most 1 ulp apart after the final rounding.  Returns the number of
    elements that are not bitwise equal."""
    got = np.asarray(got)
    want = np.asarray(want)
    assert got.shape == want.shape
    if dtype == "bf16":
        g = got.view(np.int16).astype(np.int32)
        w = want.view(np.int16).astype(np.int32)
        # ulp distance on the sign-magnitude patterns
        gm = np.where(g < 0, -(g & 0x7FFF), g)
        wm = np.where(w < 0, -(w & 0x7FFF), w)
        dist = np.abs(gm - wm)
        bad = dist > 1
        assert not bad.any(), f"{what}: {int(bad.sum())} bf16 elements differ by > 1 ulp (max {int(dist.max())})"
        return int((got != want).sum())
    gf = got.astype(np.float64)
    wf = want.astype(np.float64)
    bf = np.asarray(base).astype(np.float64)
    tol = 1e-6 * np.maximum(np.abs(wf), np.abs(bf))
    bad = np.abs(gf - wf) > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} fp32 elements outside 1e-6 relative"
    return int((got.view(np.uint32) != want.view(np.uint32)).sum())


def side_streams_from_the_first_beside():
    """Advances torch's pool of side streams so that the next torch.cuda.Stream() is the first of the pool that
    runs beside the default stream.

    torch hands out its 32 side streams in turn, so that which one a test gets depends on the tests before it,
    and HIP spreads a process's streams over 4 hardware queues: the work of streams on one queue runs in order,
    whatever it is.  Every fourth stream of the pool waits for the default stream that way.  Which, is seen with a
    small torch kernel that has to end while eight passes over a GiB still run on the default stream."""
    import torch
    busy, small = torch.zeros(1 << 30, dtype=torch.uint8, device="cuda"), torch.zeros(64, device="cuda")
    pool = [torch.cuda.Stream()]
    while len(pool) == 1 or (pool[-1].cuda_stream != pool[0].cuda_stream and len(pool) < 64):
        pool.append(torch.cuda.Stream())
    for s in pool[1:]:  # the next stream of the pool is pool[1]
        early = 0
        for _ in range(4):  # the first brings what a first launch needs
            done = torch.cuda.Event()
            for _ in range(8):
                busy.add_(1)
            done.record()
            with torch.cuda.stream(s):
                small.add_(1)
            s.synchronize()
            early += not done.query()
            torch.cuda.synchronize()
        if early >= 3:
            return
        torch.cuda.Stream()
