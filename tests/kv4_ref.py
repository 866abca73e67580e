"""The 4-bit rows by their definition, in plain torch: least value, scale and codes of both halves of a head."""
import torch


def quantise(x):
    """bf16 [..., D] -> scale, least [..., 2] (bf16 values as float32) and codes [..., 2, D/2] (int)."""
    y = x.float().reshape(*x.shape[:-1], 2, x.shape[-1] // 2)
    least, top = y.amin(-1), y.amax(-1)
    span = top - least
    good = torch.isfinite(y).all(-1) & torch.isfinite(span)
    scale = (span / torch.full_like(span, 15.0)).to(torch.bfloat16).float()
    scale = torch.where(scale < 2.0 ** -100, 0.0, scale)
    least, scale = torch.where(good, least, torch.nan), torch.where(good, scale, torch.nan)
    quotient = (y - least[..., None]) / torch.where(scale > 0, scale, 1.0)[..., None]
    codes = torch.where((scale > 0)[..., None], quotient.round(), 0.0).nan_to_num(0.0).clamp(0, 15).int()
    return scale, least, codes


def pool4(x):
    """A 16-bit pool [pages][page][H][D] as a 4-bit pool [pages][H][page * (D/2 + 8)]."""
    pages, page, h, d = x.shape
    scale, least, codes = quantise(x.permute(0, 2, 1, 3))
    byte = (codes[..., 0, :] | codes[..., 1, :] << 4).to(torch.uint8).reshape(pages, h, page * (d // 2))
    four = torch.stack([scale[..., 0], least[..., 0], scale[..., 1], least[..., 1]], -1).to(torch.bfloat16).contiguous()
    return torch.cat([byte, four.view(torch.uint8).reshape(pages, h, page * 8)], -1).contiguous()


def parts(pool, page, d):
    """Codes [pages][page][H][2][D/2], scale and least [pages][page][H][2] of a 4-bit pool."""
    pages, h, _ = pool.shape
    byte = pool[:, :, : page * (d // 2)].reshape(pages, h, page, d // 2).permute(0, 2, 1, 3)
    four = pool[:, :, page * (d // 2):].contiguous().view(torch.bfloat16).float().reshape(pages, h, page, 2, 2).permute(0, 2, 1, 3, 4)
    return torch.stack([byte & 15, byte >> 4], -2), four[..., 0], four[..., 1]


def values(pool, page, d):
    """What a 4-bit pool stands for: [pages][page][H][D], 64 bits."""
    codes, scale, least = parts(pool, page, d)
    v = codes.double() * scale.double()[..., None] + least.double()[..., None]
    return v.reshape(*v.shape[:3], d)
