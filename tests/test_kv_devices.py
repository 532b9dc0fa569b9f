"""A coded KV cache whose pools, or a workspace, are not on the rows' GPU is refused before any
call: the library would take the addresses for device memory."""

import pytest


def cpu_cache(nq, torch):
    pools = [torch.zeros(2 * 2 * 16 * n, dtype=torch.int32) if n else torch.zeros(64) for n in (8, 1, 0)] * 2
    return nq.kv_cache(heads=2, dim=64, page=16, pools=pools), pools


def test_pools_on_the_host():
    import torch
    import paper_2502_09720_amd as nq
    x = torch.zeros(3, 2, 64)
    index = torch.zeros(3, dtype=torch.int32)
    for c in (cpu_cache(nq, torch)[0], nq.kv_cache(2, 2, 64, 16, device="cpu")):
        with pytest.raises(ValueError, match="pools"):
            nq.kv_append(c, x, x, x, index.long())
        with pytest.raises(ValueError, match="pools"):
            nq.attend(c, x, index.view(3, 1), index)


def test_pools_on_two_devices():
    import torch
    import paper_2502_09720_amd as nq
    _, pools = cpu_cache(nq, torch)
    for i in range(6):
        moved = list(pools)
        moved[i] = pools[i].to("meta")
        with pytest.raises(ValueError, match="device"):
            nq.kv_cache(heads=2, dim=64, page=16, pools=moved)


@pytest.mark.gpu
def test_arguments_on_the_host():
    import torch
    import paper_2502_09720_amd as nq
    c = nq.kv_cache(2, 2, 64, 16)
    x, y = torch.zeros(3, 2, 64), torch.zeros(3, 2, 64, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64)
    for rows in ((x, y, y), (y, x, y), (y, y, x)):
        with pytest.raises(ValueError):
            nq.kv_append(c, *rows, slots.cuda())
    for more in (dict(out=x), dict(k_norm=torch.ones(64)),
                 dict(cos=torch.zeros(4, 32), sin=torch.zeros(4, 32, device="cuda"), positions=slots.int().cuda())):
        with pytest.raises(ValueError):
            nq.kv_append(c, y, y, y, slots.cuda(), **more)
    with pytest.raises(ValueError):
        nq.kv_append(c, y, y, y, slots)
    table, lengths = (torch.zeros(3, 1, dtype=torch.int32, device="cuda"),
                      torch.zeros(3, dtype=torch.int32, device="cuda"))
    for args in ((x, table, lengths), (y, table.cpu(), lengths), (y, table, lengths.cpu())):
        with pytest.raises(ValueError):
            nq.attend(c, *args)
    wide = torch.empty(64, 2, dtype=torch.uint8, device="cuda")[:, 0]
    for more in (dict(out=x), dict(lse=torch.zeros(3, 2)), dict(workspace=torch.empty(1 << 20, dtype=torch.uint8)),
                 dict(workspace=wide), dict(starts=torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(ValueError):
            nq.attend(c, y, table, lengths, **more)
