"""Layers for the kernels of the attention over 8-bit rows that none in mx_util.SHAPES reaches."""
import mx_util as M

WIDTHS = {
    "k64c512": M.shape(8, 1, 1, 64, 512), "k64c512q16": M.shape(16, 1, 2, 64, 256), "k128c512": M.shape(4, 1, 1, 128, 512),
    "k128c512q16": M.shape(16, 2, 1, 64, 512), "k256c512": M.shape(2, 1, 2, 256, 256), "k256c512q16": M.shape(16, 2, 1, 128, 512),
    "k256c1024": M.shape(4, 2, 1, 128, 1024), "k256c1024q16": M.shape(16, 4, 2, 64, 512),
    # slices: two and three of 512 or 1024 latents, in the middle of a latent and between two
    "k64c1536": M.shape(4, 1, 1, 64, 1536), "k128c1536": M.shape(6, 2, 3, 64, 512), "k256c2048": M.shape(4, 2, 1, 128, 2048),
    "k512c2048": M.shape(8, 4, 2, 128, 1024), "k1024c2048": M.shape(8, 8, 2, 128, 1024),
}
