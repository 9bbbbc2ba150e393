"""An attention block behind a convolutional stem, over the voxels of a volume as tokens.

    python -m paper_1606_05688_amd.volume_block

A stem (3^3 kernels) makes f maps of a grey volume, three banks of 1^3 kernels make queries, keys and values of every voxel.
Read voxel by voxel, x slowest, the maps are a sequence: every token gets the rotary positions of its three coordinates
and attends to the tokens of the slabs before it and to the first ones.  The same block also runs as a scan does it: slabs
come one after the other, their keys and values go into an 8-bit cache, and the new tokens attend over what it holds.
"""
import torch

from . import binding as znni

PAGE = znni.KV8_PAGE


class VolumeBlock:
    """Random weights of a block with Hq query heads and Hk key and value heads of D elements on f maps.  `slabs` whole planes
    of voxels before a token's own are surely in its window, `sinks` first tokens always."""

    def __init__(self, f=16, Hq=8, Hk=2, D=32, slabs=2, sinks=4, dtype=torch.float32, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)

        def bank(fo, fi, k):
            return torch.randn((fo, fi, k, k, k), generator=g, device=device) * (fi * k ** 3) ** -0.5

        self.f, self.Hq, self.Hk, self.D, self.slabs, self.sinks, self.dtype = f, Hq, Hk, D, slabs, sinks, dtype
        self.stem, self.bias = bank(f, 1, 3), torch.zeros(f, device=device)
        self.wq, self.wk, self.wv = 2 * bank(Hq * D, f, 1), 2 * bank(Hk * D, f, 1), bank(Hk * D, f, 1)
        a = D // 2 // 3
        self.sections = (D // 2 - 2 * a, a, a)                    # pairs of a head for x, y and z
        self.freq = torch.cat([100.0 ** (-torch.arange(n, device=device) / n) for n in self.sections]).float()

    def heads(self, volume, x0=0):
        """volume [1, 1, nx + 2, ny, nz] -> (q, k, v, planes): heads of the voxels of nx planes that begin at plane x0 of the
        whole map, queries and keys with their positions, and the voxels of a plane."""
        maps = znni.znni_conv3d(volume, self.stem, self.bias, relu=True)
        nx, ny, nz = maps.shape[2:]

        def tokens(w, H):
            y = znni.znni_conv3d(maps, w)[0]                      # [H D, nx, ny, nz]
            return y.reshape(H, self.D, -1).permute(2, 0, 1).contiguous().to(self.dtype)

        grid = torch.meshgrid(*(torch.arange(n, device=maps.device) for n in (nx, ny, nz)), indexing="ij")
        pos = torch.stack([grid[0] + x0, grid[1], grid[2]], -1).reshape(-1, 3).to(torch.int32)
        q, k = znni.znni_rope_axes(tokens(self.wq, self.Hq), tokens(self.wk, self.Hk), pos, self.freq, self.sections)
        return q, k, tokens(self.wv, self.Hk), ny * nz

    def whole(self, volume):
        """The block on a whole volume: [voxels, Hq, D]."""
        q, k, v, plane = self.heads(volume)
        cu = torch.tensor([0, q.shape[0]], dtype=torch.int32, device=q.device)
        return znni.znni_attn_window(q, k, v, cu, cu, q.shape[0], q.shape[0], left=self.slabs * plane, sinks=self.sinks)

    def scan(self, volume, planes):
        """The same, `planes` planes at a time, over a cache of 8 bits a value.  Yields the outputs of the voxels as they come.  Pages
        that the window has left behind (but for those of the first tokens) go back and are used again."""
        device, held, free, table, cache = volume.device, 0, [], [], None
        nx = volume.shape[2] - 2
        for x0 in range(0, nx, planes):
            x1 = min(nx, x0 + planes)
            q, k, v, plane = self.heads(volume[:, :, x0:x1 + 2].clone(), x0)
            new = q.shape[0]
            if cache is None:                                     # window, newest slab, first tokens, two pages cut open
                pages = -(-(self.slabs * plane + planes * plane) // PAGE) + -(-self.sinks // PAGE) + 3
                cache, free = znni.kv8_alloc(pages, self.Hk, self.D, device), list(range(pages))
            while len(table) * PAGE < held + new:
                table.append(free.pop())
            at = torch.tensor([table], dtype=torch.int32, device=device)
            start = torch.tensor([held], dtype=torch.int32, device=device)
            znni.znni_kv8_append(*cache, k, v, at, torch.tensor([0, new], dtype=torch.int32, device=device), start, new)
            held += new
            yield znni.znni_kv8_attn(q[None], *cache, at, start + new, held, left=self.slabs * plane, sinks=self.sinks)[0]
            for i in range(-(-self.sinks // PAGE), max(0, held - self.slabs * plane) // PAGE):
                if table[i] >= 0:
                    free.append(table[i])
                    table[i] = -1                                 # no row will look there again


def main():
    block = VolumeBlock(dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(1)
    volume = torch.rand((1, 1, 34, 18, 18), generator=g, device="cuda")
    whole = block.whole(volume).float()
    parts = torch.cat(list(block.scan(volume, 1))).float()
    off = ((parts - whole).norm() / whole.norm()).item()
    print(f"{whole.shape[0]} voxels, {block.Hq} heads of {block.D}: plane by plane over the 8-bit cache, {100 * off:.1f} % off the whole volume's")


if __name__ == "__main__":
    main()
