"""Sizes of the feed-forward block that meet every form of its kernels, and which form each product has there: of tiles of 256 x 256 (L) or 128 x 128 (S) in
bf16, D: some have a workgroup each, P: some are cut along k into pieces, R: what is left of those is shared out; in fp32 0, 1, 2: 32 x 32 tiles
whose k eight waves divide, 64 x 64 tiles whose k four groups divide, 64 x 64 tiles.  The sizes leave remainders in every direction."""
PRODUCTS = ("gate", "down", "dgate", "dx", "weights")

# rows, width, inner, form of each product; "few": few rows
BF16 = [
    (1, 40, 24, "few few SD SD SD"), (17, 2100, 130, "few few SD SD SD"), (61, 2056, 2600, "few few SD SP LD"), (190, 77, 2003, "few few SD SP SD"),
    (289, 8, 16, "SD SD SD SD SD"), (216, 9, 12, "SD SD SD SD SD"), (1463, 8, 5592, "LD SP LD SP SP"), (1232, 9, 6825, "LD SP LD SP SP"),
    (32999, 144, 8, "SD LD SD LD SPR"), (33518, 131, 9, "SD LD SD LD SPR"), (11251, 141, 2705, "LD LP LD LP LP"), (10981, 144, 3464, "LD LP LD LP LP"),
    (65659, 168, 464, "LD LDP LD LDP LPR"), (6966, 2316, 642, "LD LDP SD LDP LPR"), (3107, 792, 3488, "LD SPR LD SPR SDP"), (4380, 286, 7485, "LD SPR LD SPR SDP"),
    (3865, 2056, 1576, "LD SDP SD SDP LD"), (3909, 2143, 1610, "LD SDP SD SDP LD"), (4537, 1056, 4608, "LD LPR LD LPR LDP"), (3644, 1346, 4517, "LD LPR LD LPR LDP"),
    (3285, 776, 8240, "LD SPR LD LPR LDPR"), (2964, 1083, 6497, "LD LP LD LP LDPR"), (7554, 592, 5456, "LD SPR LD LPR SDPR"), (7460, 623, 5401, "LD SPR LD LPR SDPR"),
    (26142, 272, 3760, "LD LD LD SDPR SPR"), (27396, 262, 3908, "LD LD LD SDPR SPR"), (33340, 528, 1568, "LD LD LD LDPR LP"), (32941, 575, 1476, "LD LD LD LDPR LPR"),
    (51005, 272, 3000, "LD SDPR LD SDPR LPR"), (51027, 263, 3861, "LD SDPR LD LDPR SPR"), (32768, 768, 2048, "LD LDP LD LDP LPR"), (32767, 763, 2045, "LD LDP LD LDP LPR"),
]
F32 = [
    (1, 40, 24, "0 0 0 0 0"), (33, 1400, 2840, "0 0 0 0 2"), (300, 100, 130, "0 0 0 0 0"), (701, 890, 697, "0 0 0 0 1"), (1500, 1100, 1300, "1 1 1 1 2"),
    (1333, 1027, 901, "1 1 1 1 2"), (1900, 1110, 1203, "2 2 2 2 2"), (2001, 1160, 1288, "2 2 2 2 2"),
]
